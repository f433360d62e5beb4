// Attention of rows that share a prefix, over a paged cache: every row of a sequence reads its group's
// prefix and, causally, its sequence's own keys; grouped-query heads map query head i to kv head
// i / (Hq / Hkv).  prefix_plan.cuh says how the work of larger calls is cut; here are the kernel for few query
// vectors per entry, the kernel that joins the segments, and the kernel that takes smaller calls by itself.
//
// Score s_k = scale <q, K_k>, m = max s_k, l = sum exp(s_k - m), o = sum exp(s_k - m) V_k / l, one pass over
// the keys with the running m, l and o in fp32; exponentials in base 2 with scale log2(e) folded into the
// scores.  P is rounded to bf16 for the second product (relative 2^-9 of each weight, the operand's type),
// the sum l takes the unrounded weights.  A row without a visible key has l = 0: zeros out, lse -infinity.
#include <algorithm>
#include <cmath>

#include "internal.h"
#include "prefix_plan.cuh"

namespace sp {

namespace {

SP_DEVINL float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

SP_DEVINL void cp_async16(uint32_t dst, const void* src, int bytes) {  // bytes 16, or 0: zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
SP_DEVINL void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
SP_DEVINL void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

SP_DEVINL void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
SP_DEVINL void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// c += a b, 16 x 8 x 16, bf16 in, fp32 sums
SP_DEVINL void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// --------------------------------------------------------------- few query vectors per entry
// A worker is one warp with its own ring of key tiles in shared memory: 16 query vectors against 16 keys at
// a time (a tile never crosses a page, whose size is a multiple of 16), no barrier between warps.  Bound by
// the cache's bytes: the products are padded to 16 rows, which the memory's pace leaves room for.  Measured: 89 MB
// (four beams each of 16 prefixes, 32 heads of 128) in 22 us, of which 3 are the start; 8 KB take a warp some 2,300
// cycles, with eight warps per SM 28 bytes a cycle, near what HBM gives an SM.  Twelve warps with two tiles in
// flight instead of eight with three made no difference.
constexpr int WK_WARPS = 8, WK_NT = WK_WARPS * 32, WK_KEYS = 16, WK_ROWS = 16;

template <int DH>
struct WkCfg {
  static constexpr int ROW = DH * 2;                     // bytes of a key's row
  static constexpr int STAGE = 2 * WK_KEYS * ROW;        // K tile, V tile
  static constexpr int NS = DH == 128 ? 3 : 6;           // tiles in flight per warp: 24 KB
  static constexpr size_t SMEM = (size_t)WK_WARPS * NS * STAGE;
};

// (200 registers a thread leave room for a CTA of the merge beside this kernel's, which then waits on the SM instead
// of being launched when it ends: 11.3 us instead of 12.6 for four beams, when they went this way)
template <int DH>
__global__ void __maxnreg__(200) prefix_warp_kernel(const PrefixArgs a, const PlanArgs p, int late) {
  using C = WkCfg<DH>;
  constexpr int CPR = DH / 8;  // 16-byte chunks of a row
  extern __shared__ __align__(128) uint8_t ring_all[];
  __shared__ PlanShared plan;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int E = a.n_groups + a.B, G = a.Hq / a.Hkv;
  // Behind prefix_tc_kernel (late) nothing here reads or overwrites what that writes, and what came before it was
  // complete when it let this kernel start: only the merge has to find both complete, so the wait is at the end and
  // SMs that the other kernel has left are used meanwhile.
  if (!late) pdl_wait();
  pdl_trigger();
  build_plan<WK_NT>(a, p, plan, blockIdx.x == 0);
  if (warp == WK_WARPS - 1) write_rows(a, p, plan, lane, 32);  // (the warp with the least to do)
  const int N = plan.unit0[E], P = N > 0 ? plan_workers(p, N) : 0;
  // a short list goes to different SMs first; behind the other kernel to few, those that one has left idle
  const int w = late ? blockIdx.x * WK_WARPS + warp : blockIdx.x + warp * gridDim.x;
  int t0 = 0, t1 = 0;
  if (w < P) part_of_worker(N, P, w, t0, t1);
  TileCursor put, get;
  bool more = w < P && get.seek(plan, p, E, a.Hkv, t0, t1);
  put = get;
  bool more_put = more;

  const uint32_t ring = smem_u32(ring_all) + warp * C::NS * C::STAGE;
  const size_t W = (size_t)a.Hkv * DH;
  const size_t plane = ((size_t)a.n_pages << a.page_shift) * W;

  // A tile to be loaded: its page is looked up when the one before it is loaded, which hides the lookup.
  struct Ahead {
    int page, row, n, kvh;  // page, its first key's row there, keys, kv head
    bool some;
  };
  auto look = [&]() {
    Ahead h;
    h.some = more_put;
    if (!more_put) return h;
    const bool pre = put.e < a.n_groups;
    const int k0 = put.j * WK_KEYS;
    const int* tb = pre ? a.ptable + (size_t)put.e * a.pmax_pages : a.table + (size_t)(put.e - a.n_groups) * a.max_pages;
    h.page = __ldg(tb + (k0 >> a.page_shift));
    h.row = k0 & ((1 << a.page_shift) - 1);
    h.n = min(WK_KEYS, plan.keys[put.e] - k0);
    h.kvh = put.kvh;
    more_put = put.next(plan, p, a.Hkv, t1);
    return h;
  };
  // one tile into ring slot `slot`: lane = 16-byte chunk of a row, rows in turn; rows past the keys are zeros
  auto load_tile = [&](const Ahead& h, int slot) {
    int page = h.page;
    const bool ok = page >= 0 && page < a.n_pages;
    if (!ok) {
      if (lane == 0) set_error(a.err, SP_DEVERR_INDEX);
      page = 0;
    }
    const uint32_t dst = ring + slot * C::STAGE;
    const int c = lane % CPR;
    const __nv_bfloat16* src = a.kv + (((size_t)page << a.page_shift) + h.row) * W + h.kvh * DH + c * 8;
#pragma unroll
    for (int r0 = 0; r0 < WK_KEYS; r0 += 32 / CPR) {
      const int r = r0 + lane / CPR;
      const bool in = ok && r < h.n;
      const __nv_bfloat16* s = src + (in ? r : 0) * W;
      const uint32_t d = dst + r * C::ROW + ((c ^ (r & 7)) << 4);
      cp_async16(d, s, in ? 16 : 0);
      cp_async16(d + WK_KEYS * C::ROW, s + plane, in ? 16 : 0);
    }
  };

  Ahead first[C::NS - 1], ahead;
#pragma unroll
  for (int s = 0; s < C::NS - 1; ++s) first[s] = look();
  ahead = look();
#pragma unroll
  for (int s = 0; s < C::NS - 1; ++s) {
    if (first[s].some) load_tile(first[s], s);
    cp_async_commit();
  }

  uint32_t qf[DH / 16][4];
  float o[DH / 8][4];
  float m[2], l[2];
  int lim[2];
  bool fresh = true;
  int slot = 0, slot_put = C::NS - 1;
  const int row_a = lane >> 2, col = (lane & 3) * 2;

  while (more) {
    if (fresh) {  // a new segment: its query vectors, empty statistics
      const int M = plan.rows[get.e] * G;
      const int keys = plan.keys[get.e], R = plan.rows[get.e];
      const bool pre = get.e < a.n_groups;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int mr = row_a + 8 * h, mv = get.rt * p.tile_rows + mr;
        const int r = mv / G, g = mv - r * G;
        const bool have = mr < p.tile_rows && mv < M;
        lim[h] = have ? (pre ? keys : min(max(keys - R + r + 1, 0), keys)) : 0;
        const __nv_bfloat16* qr = a.q + (have ? (plan.row0[get.e] + r) * a.ld_q + (get.kvh * G + g) * DH : 0) + col;
#pragma unroll
        for (int kk = 0; kk < DH / 16; ++kk) {
          qf[kk][h] = have ? __ldg(reinterpret_cast<const unsigned int*>(qr + kk * 16)) : 0u;
          qf[kk][h + 2] = have ? __ldg(reinterpret_cast<const unsigned int*>(qr + kk * 16 + 8)) : 0u;
        }
        m[h] = -INFINITY;
        l[h] = 0.f;
      }
#pragma unroll
      for (int n = 0; n < DH / 8; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][c] = 0.f;
      fresh = false;
    }
    if (ahead.some) {
      load_tile(ahead, slot_put);
      ahead = look();
    }
    cp_async_commit();
    if (++slot_put == C::NS) slot_put = 0;
    cp_async_wait<C::NS - 1>();
    __syncwarp();  // every lane's copies of this tile have landed and are visible to the warp

    const uint32_t kt = ring + slot * C::STAGE, vt = kt + WK_KEYS * C::ROW;
    float s[2][4];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[n][c] = 0.f;
    {
      const int r = (lane >> 4) * 8 + (lane & 7), cb = (lane >> 3) & 1;
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk) {
        uint32_t b[4];
        ldsm4(kt + r * C::ROW + (((2 * kk + cb) ^ (r & 7)) << 4), b);
        mma16816(s[0], qf[kk], b[0], b[1]);
        mma16816(s[1], qf[kk], b[2], b[3]);
      }
    }
    const int k0 = get.j * WK_KEYS;
    uint32_t pf[4];
    float corr[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float x[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int key = k0 + (c >> 1) * 8 + col + (c & 1);
        x[c] = key < lim[h] ? s[c >> 1][2 * h + (c & 1)] * a.scale_log2 : -INFINITY;
      }
      float mx = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
      const float mn = fmaxf(m[h], mx);
      const float mz = mn == -INFINITY ? 0.f : mn;
      corr[h] = ex2(m[h] - mz);  // (0 while m is -infinity)
      m[h] = mn;
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = ex2(x[c] - mz);
      l[h] = l[h] * corr[h] + ((x[0] + x[1]) + (x[2] + x[3]));
      pf[h] = pack_bf16x2(x[0], x[1]);
      pf[h + 2] = pack_bf16x2(x[2], x[3]);
    }
    if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
      for (int n = 0; n < DH / 8; ++n) {
        o[n][0] *= corr[0];
        o[n][1] *= corr[0];
        o[n][2] *= corr[1];
        o[n][3] *= corr[1];
      }
    }
    {
      const int r = ((lane >> 3) & 1) * 8 + (lane & 7), cb = lane >> 4;
#pragma unroll
      for (int nn = 0; nn < DH / 16; ++nn) {
        uint32_t b[4];
        ldsm4_t(vt + r * C::ROW + (((2 * nn + cb) ^ (r & 7)) << 4), b);
        mma16816(o[2 * nn], pf, b[0], b[1]);
        mma16816(o[2 * nn + 1], pf, b[2], b[3]);
      }
    }
    __syncwarp();  // the tile is read before a lane's next copies overwrite it
    if (++slot == C::NS) slot = 0;

    const TileCursor now = get;
    more = get.next(plan, p, a.Hkv, t1);
    if (!more || get.item != now.item) {  // the segment ends
      const int M = plan.rows[now.e] * G;
      const size_t base = ((size_t)now.item + w) * p.slot_rows;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = l[h];
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
        const int mr = row_a + 8 * h;
        if (mr < p.tile_rows && now.rt * p.tile_rows + mr < M) {
          float* po = p.part_o + (base + mr) * DH + col;
#pragma unroll
          for (int n = 0; n < DH / 8; ++n)
            *reinterpret_cast<float2*>(po + n * 8) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
          if ((lane & 3) == 0) p.part_ml[base + mr] = make_float2(m[h], sum);
        }
      }
      fresh = true;
    }
  }
  cp_async_wait<0>();
  if (late) pdl_wait();
}

// --------------------------------------------------------------- joining the segments
// One warp per row and VC query heads of a kv head: the segments of their prefix item and of their own item, in key
// order, up to 32 of them at a time.  Bound by latency, so the chain of dependent accesses is short: where the
// row's items lie (both at once), every segment's (max, sum), a lane each, then the values with the weights known.
// It adds 5 us to a call of few rows, 13 to one of 512 rows of 28 heads (21 MB of segments).
template <int DH, int VC>
__global__ void __launch_bounds__(256, 4) prefix_merge_kernel(const PrefixArgs a, const PlanArgs pp, const PlanArgs po) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int E = a.n_groups + a.B, G = a.Hq / a.Hkv;
  const int per = (G + VC - 1) / VC;  // warps per kv head
  const int row = blockIdx.x, task = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (task >= a.Hkv * per) return;
  int4 place[2];
  int total[2];
  place[0] = pp.prefix ? __ldcg(pp.rows_prefix + row) : make_int4(0, 0, 0, 0);
  place[1] = po.own ? __ldcg(po.rows_own + row) : make_int4(0, 0, 0, 0);
  total[0] = pp.prefix ? __ldcg(pp.unit0 + E) : 0;
  total[1] = po.own ? __ldcg(po.unit0 + E) : 0;
  if (row < row_begin(a, 0) || row >= row_begin(a, a.B)) return;
  const int kvh = task / per, g0 = (task - kvh * per) * VC, nv = min(VC, G - g0);
  int n[2];           // segments of the prefix item, of the own item
  size_t first[2];    // slot row of the first one's first vector
#pragma unroll
  for (int side = 0; side < 2; ++side) {
    const PlanArgs& p = side == 0 ? pp : po;
    const int unit0 = place[side].x, len = place[side].y, N = total[side];
    n[side] = 0;
    first[side] = 0;
    if (len == 0) continue;
    const int mv = place[side].w + g0;
    const int rt = mv / p.tile_rows, mr = mv - rt * p.tile_rows;
    const int in = rt * a.Hkv + kvh;
    // the workers that have key tiles of the item, units u0 .. u1: a lane tries each of 32 candidates, from a little
    // before where u0's worker is estimated
    const int u0 = unit0 + in * len + p.over, u1 = unit0 + in * len + len - 1;
    const int P = plan_workers(p, N);
    int from = max((int)((float)u0 / (float)N * (float)P) - 2, 0);
    while (from > 0 && part_begin(N, P, from) > u0) --from;
    int w0 = from, w1 = from;
    for (int c = from;; c += 32) {
      const int begin = c + lane < P ? part_begin(N, P, c + lane) : 0x7fffffff;
      const unsigned int upto0 = __ballot_sync(0xffffffffu, begin <= u0), upto1 = __ballot_sync(0xffffffffu, begin <= u1);
      if (upto0) w0 = c + 31 - __clz(upto0);
      if (upto1) w1 = c + 31 - __clz(upto1);
      if (upto1 != 0xffffffffu) break;
    }
    n[side] = w1 - w0 + 1;
    first[side] = ((size_t)(place[side].z + in) + w0) * p.slot_rows + mr;
  }
  constexpr int V = DH / 32;
  float acc[VC][V], mm[VC], ll[VC];
#pragma unroll
  for (int x = 0; x < VC; ++x) {
    mm[x] = -INFINITY;
    ll[x] = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) acc[x][v] = 0.f;
  }
  for (int s0 = 0; s0 < n[0] + n[1]; s0 += 32) {
    const int s = s0 + lane, there = min(32, n[0] + n[1] - s0);
    const float* o = nullptr;  // the lane's segment: values and (max, sum) of the first vector
    const float2* ml_at = nullptr;
    if (s < n[0]) {
      const size_t at = first[0] + (size_t)s * pp.slot_rows;
      ml_at = pp.part_ml + at;
      o = pp.part_o + at * DH;
    } else if (s < n[0] + n[1]) {
      const size_t at = first[1] + (size_t)(s - n[0]) * po.slot_rows;
      ml_at = po.part_ml + at;
      o = po.part_o + at * DH;
    }
    float2 ml[VC];
    float cb[VC];
#pragma unroll
    for (int x = 0; x < VC; ++x) {
      ml[x] = make_float2(-INFINITY, 0.f);
      if (ml_at && x < nv) ml[x] = __ldcg(ml_at + x);
    }
#pragma unroll
    for (int x = 0; x < VC; ++x) {
      const float mn = fmaxf(mm[x], warp_max(ml[x].x));
      const float mz = mn == -INFINITY ? 0.f : mn;
      const float ca = ex2(mm[x] - mz);  // (0 while mm is -infinity)
      cb[x] = ex2(ml[x].x - mz);
      ll[x] = ll[x] * ca + warp_sum(ml[x].y * cb[x]);
#pragma unroll
      for (int v = 0; v < V; ++v) acc[x][v] *= ca;
      mm[x] = mn;
    }
#pragma unroll(VC == 1 ? 4 : 2)
    for (int i = 0; i < there; ++i) {
      const float* src = reinterpret_cast<const float*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(o), i)) + lane * V;
      float y[VC][V];
#pragma unroll
      for (int x = 0; x < VC; ++x) {
        if (x >= nv) continue;
        if (V == 4) *reinterpret_cast<float4*>(y[x]) = __ldcg(reinterpret_cast<const float4*>(src + x * DH));
        else *reinterpret_cast<float2*>(y[x]) = __ldcg(reinterpret_cast<const float2*>(src + x * DH));
      }
#pragma unroll
      for (int x = 0; x < VC; ++x) {
        const float c = __shfl_sync(0xffffffffu, cb[x], i);
        if (x >= nv) continue;
        if (c != 0.f) {  // (a segment that saw no key of this vector may hold anything)
#pragma unroll
          for (int v = 0; v < V; ++v) acc[x][v] += y[x][v] * c;
        }
      }
    }
  }
#pragma unroll
  for (int x = 0; x < VC; ++x) {
    if (x >= nv) continue;
    const int h = kvh * G + g0 + x;
    const float inv = ll[x] == 0.f ? 0.f : 1.f / ll[x];  // (NaN stays NaN)
    __nv_bfloat16* d = a.out + row * a.ld_out + (long long)h * DH + lane * V;
    if (V == 4)
      *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16x2(acc[x][0] * inv, acc[x][1] * inv),
                                                pack_bf16x2(acc[x][V - 2] * inv, acc[x][V - 1] * inv));
    else
      *reinterpret_cast<uint32_t*>(d) = pack_bf16x2(acc[x][0] * inv, acc[x][1] * inv);
    if (a.lse && lane == 0)
      a.lse[(size_t)row * a.Hq + h] = ll[x] == 0.f ? -INFINITY : (mm[x] + log2f(ll[x])) * 0.69314718055994531f;
  }
}

template <int DH>
cudaError_t launch_merge(const PrefixArgs& a, const PlanArgs& pp, const PlanArgs& po, cudaStream_t st) {
  // four heads per warp where there are warps enough all the same (24 per SM): fewer chains; above 16 heads per kv
  // head a row's vectors may lie in two row tiles, so one
  const int G = a.Hq / a.Hkv, four = (G + 3) / 4;
  const bool many = G > 1 && G <= 16 && (long long)a.T_cap * a.Hkv * four >= 24ll * device_sm_count();
  const dim3 grid(a.T_cap, (a.Hkv * (many ? four : G) + 7) / 8);
  return launch_pdl(many ? prefix_merge_kernel<DH, 4> : prefix_merge_kernel<DH, 1>, grid, dim3(256), 0, st, a, pp, po);
}

// --------------------------------------------------------------- few tiles per row, joined in a CTA
// One CTA per R consecutive rows and kv head, its warps in turn over the 16-key tiles of the rows' prefixes (one that
// several of the rows share is read once for them) and own keys, and the join in shared memory: one launch, no plan,
// no workspace.  The R G <= 8 query vectors are the product's N: S^T = K Q^T and O^T = V^T P^T, so half the registers
// of the other form hold Q and O; a tile counts for the vectors of its rows.
// Measured: four beams (32 heads of 128, 240 + 20 keys) 5.8 us instead of 11.1 by plan and merge; 64 beams of 16 prefixes
// of 300 keys (89 MB) 20.5 instead of 28.5.  With few CTAs bound by the chain of a tile, some 330 instructions that a warp
// issues at 0.47 a cycle and scheduler together with 2 or 3 others (a tile takes a warp 1 us); 14 warps with two tiles in
// flight each fill the shared memory and the registers (nine with three took 31 us where these take 24: 4,000 keys).
// With many CTAs bound by HBM: 64 rows of 500 keys of their own, 540 MB, 95.7 us (5.6 TB/s).
constexpr int RK_VECS = 8, RK_NS = 2;  // vectors; tiles of a warp in flight

template <int DH>
struct RkCfg {
  static constexpr int ROW = DH * 2, HALF = WK_KEYS * ROW, STAGE = 2 * HALF;  // K tile, V tile
  static constexpr int WARPS = DH == 128 ? 14 : 12;                           // of a CTA at most
  static constexpr int SM_WARPS = DH == 128 ? 14 : 24;                        // of an SM, by shared memory and registers
};

SP_DEVINL uint32_t transpose8(uint32_t x) {  // an 8 x 8 matrix of 16-bit elements, a row's pair per lane
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int DH>
__global__ void __launch_bounds__(RkCfg<DH>::WARPS * 32, RkCfg<DH>::SM_WARPS / RkCfg<DH>::WARPS)
prefix_row_kernel(const PrefixArgs a, int R, int rows) {
  using C = RkCfg<DH>;
  constexpr int CPR = DH / 8;
  extern __shared__ __align__(256) uint8_t row_ring[];  // [warps][RK_NS][STAGE]; then the warps' O, [8][DH] each
  __shared__ float2 ml_s[C::WARPS][RK_VECS];
  static_assert(RK_VECS * DH * 4 <= RK_NS * C::STAGE, "a warp's O in its ring");
  pdl_wait();
  pdl_trigger();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  const int G = a.Hq / a.Hkv, kvh = blockIdx.x, r0 = blockIdx.y * R, nr = min(R, rows - r0);
  const int cap = a.max_pages << a.page_shift, pcap = a.pmax_pages << a.page_shift;
  // Lane i < 8 stands for the prefix that row r0 + i is the first of the rows to read, lane 8 + i for the sequence whose
  // first row here is r0 + i.  First lane i's and lane 8 + i's row, its sequence b (-1: none), that one's rows, its group g
  // (-1: none): the last that begins at or before, if it reaches it.
  const int my = r0 + min(lane & 7, nr - 1);
  int b = -1, g = -1, b_from = my, b_rows = 1;
  // (A round's offsets are loaded in the one before it.)
  int own_len = 0;
  if (!a.cu_rows) {
    if (my < a.B) own_len = __ldg(a.lens + (b = my));
  }
  auto group_at = [&](int i) { return i <= a.n_groups ? __ldg(a.group_cu + i) : 0; };
  int g_from = a.n_groups ? group_at(lane) : 0, g_to = a.n_groups ? group_at(lane + 1) : 0;
  if (a.cu_rows) {
    auto row_at = [&](int i) { return row_begin(a, min(i, a.B)); };
    int from = row_at(lane), to = row_at(lane + 1);
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int from_next = row_at(b0 + 32 + lane), to_next = row_at(b0 + 33 + lane);
      for (int j = 0; j < nr; ++j) {
        const unsigned int all = __ballot_sync(0xffffffffu, from <= r0 + j && r0 + j < to);
        const int at = all ? 31 - __clz(all) : 0, f = __shfl_sync(0xffffffffu, from, at), n = __shfl_sync(0xffffffffu, to, at) - f;
        if (all && my == r0 + j) {
          b = b0 + at;
          b_from = f;
          b_rows = n;
        }
      }
      from = from_next;
      to = to_next;
    }
    if (b >= 0) own_len = __ldg(a.lens + b);
  }
  for (int g0 = 0; g0 < a.n_groups; g0 += 32) {
    const int from_next = group_at(g0 + 32 + lane), to_next = group_at(g0 + 33 + lane);
    for (int j = 0; j < nr; ++j) {
      const int bj = __shfl_sync(0xffffffffu, b, j);
      const unsigned int all = __ballot_sync(0xffffffffu, g0 + lane < a.n_groups && g_from <= bj && bj < g_to);
      if (all && bj >= 0 && my == r0 + j) g = g0 + 31 - __clz(all);
    }
    g_from = from_next;
    g_to = to_next;
  }
  const bool live = lane < 16 && (lane & 7) < nr && b >= 0;
  const int own = live ? min(max(own_len, 0), cap) : 0;
  const int see = min(max(own - b_rows + my - b_from + 1, 0), own);  // own keys that the row sees
  const int b_before = __shfl_up_sync(0xffffffffu, b, 1), g_before = __shfl_up_sync(0xffffffffu, g, 1);
  const bool first = live && ((lane & 7) == 0 || (lane < 8 ? g != g_before : b != b_before));
  const unsigned int firsts = __ballot_sync(0xffffffffu, first || !live);  // (a row of none ends a run as well)
  const int run = __ffs(firsts >> (lane & 31) >> 1 | 1u << (8 - (lane & 7) - 1));  // rows of the run that begins here
  const int see_last = __shfl_sync(0xffffffffu, see, (lane + run - 1) & 31);
  int keys = 0, cols = 0;  // the lane's keys; its vectors, begin | end << 8, and 1 << 16 for own keys
  const int* tab = a.table;
  if (first && lane >= 8) {
    keys = see_last;
    cols = (lane - 8) * G | (lane - 8 + run) * G << 8 | 1 << 16;
    tab = a.table + (size_t)b * a.max_pages;
  } else if (first && g >= 0) {
    keys = min(max(__ldg(a.plens + g), 0), pcap);
    cols = lane * G | (lane + run) * G << 8;
    tab = a.ptable + (size_t)g * a.pmax_pages;
  }
  const int mine = (keys + WK_KEYS - 1) / WK_KEYS;
  int upto = mine;  // tiles of the lanes up to this one
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  const int tiles = __shfl_sync(0xffffffffu, upto, 15);
  const unsigned int lives = __ballot_sync(0xffffffffu, live);
  const size_t W = (size_t)a.Hkv * DH;
  const size_t plane = ((size_t)a.n_pages << a.page_shift) * W;
  const uint32_t ring = smem_u32(row_ring) + warp * RK_NS * C::STAGE;

  struct Tile {
    int page, row, n, cols, k0;  // page, its first key's row there, keys (0: there is no such tile), vectors, first key
  };
  // The lane whose tiles come next: its first tile and the one behind its last, keys, vectors, table.  (Every warp looks
  // at its tiles in order.)
  int seg_from = 0, seg_to = 0, seg_keys = 0, seg_cols = 0;
  const int* seg_tab = nullptr;
  auto look = [&](int t) {
    Tile x;
    x.page = x.row = x.n = x.cols = x.k0 = 0;
    if (t >= tiles) return x;
    if (t >= seg_to) {
      const int from = __popc(__ballot_sync(0xffffffffu, lane < 16 && upto <= t));
      seg_from = __shfl_sync(0xffffffffu, upto - mine, from);
      seg_to = seg_from + __shfl_sync(0xffffffffu, mine, from);
      seg_keys = __shfl_sync(0xffffffffu, keys, from);
      seg_cols = __shfl_sync(0xffffffffu, cols, from);
      seg_tab = reinterpret_cast<const int*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(tab), from));
    }
    const int k0 = (t - seg_from) * WK_KEYS;
    x.n = min(WK_KEYS, seg_keys - k0);
    x.cols = seg_cols;
    x.k0 = k0;
    x.row = k0 & ((1 << a.page_shift) - 1);
    x.page = __ldg(seg_tab + (k0 >> a.page_shift));
    return x;
  };
  // A tile's rows: lane = 16-byte piece, rows in turn, pieces exchanged so that reading them meets no bank twice.  Rows
  // past the keys are zeros.
  constexpr int STEP = 32 / CPR;
  const int piece = lane % CPR, row_in = lane / CPR;
  const uint32_t put = row_in * C::ROW + ((piece ^ row_in) << 4);
  auto load = [&](const Tile& x, int slot) {
    const bool ok = x.page >= 0 && x.page < a.n_pages;
    if (!ok && lane == 0) set_error(a.err, SP_DEVERR_INDEX);
    const __nv_bfloat16* src = a.kv + ((((size_t)(ok ? x.page : 0)) << a.page_shift) + x.row) * W + kvh * DH + piece * 8;
    const uint32_t dst = ring + slot * C::STAGE;
    if (ok && x.n == WK_KEYS) {
      const __nv_bfloat16 *k = src + row_in * W, *v = k + plane;
#pragma unroll
      for (int i = 0; i < WK_KEYS; i += STEP) {
        const uint32_t to = dst + (put ^ ((i & 7) << 4)) + i * C::ROW;
        cp_async16(to, k, 16);
        cp_async16(to + C::HALF, v, 16);
        k += STEP * W;
        v += STEP * W;
      }
    } else {
      const int n = ok ? x.n : 0;
#pragma unroll 1
      for (int i = 0; i < WK_KEYS; i += STEP) {
        const int r = i + row_in;
        const __nv_bfloat16* from = src + (r < n ? r : 0) * W;
        const uint32_t to = dst + (put ^ ((i & 7) << 4)) + i * C::ROW;
        cp_async16(to, from, r < n ? 16 : 0);
        cp_async16(to + C::HALF, from + plane, r < n ? 16 : 0);
      }
    }
  };

  Tile q[RK_NS];  // the tile at hand, those in flight, and the one to be loaded next
#pragma unroll
  for (int i = 0; i < RK_NS; ++i) q[i] = look(warp + i * warps);
#pragma unroll
  for (int i = 0; i < RK_NS - 1; ++i) {
    if (q[i].n) load(q[i], i);
    cp_async_commit();
  }
  // the query vectors: vector lane / 4
  uint32_t qf[DH / 16][2];
  {
    const int vec = lane >> 2, r = min(vec / G, nr - 1);
    const bool have = vec < nr * G;
    const __nv_bfloat16* qr = a.q + (r0 + r) * a.ld_q + (kvh * G + (have ? vec - r * G : 0)) * DH + (lane & 3) * 2;
#pragma unroll
    for (int kk = 0; kk < DH / 16; ++kk)
#pragma unroll
      for (int x = 0; x < 2; ++x) qf[kk][x] = have ? __ldg(reinterpret_cast<const unsigned int*>(qr + kk * 16 + x * 8)) : 0u;
  }
  float o[DH / 16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};  // of vectors 2 (lane % 4) and the next
#pragma unroll
  for (int n = 0; n < DH / 16; ++n)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[n][c] = 0.f;
  const int whole = nr * G << 8;
  int limit[2];  // own keys of the rows of this lane's vectors
#pragma unroll
  for (int v = 0; v < 2; ++v) limit[v] = __shfl_sync(0xffffffffu, see, min(((lane & 3) * 2 + v) / G, nr - 1));
  // a lane's address for the pieces 0 and 1 of K, of V transposed; pieces 2 i and 2 i + 1 are at it ^ (i << 5)
  const uint32_t get_k = (lane & 15) * C::ROW + (((lane >> 4) ^ (lane & 7)) << 4);
  const uint32_t get_v = ((lane >> 4) * 8 + (lane & 7)) * C::ROW + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
  int slot = 0, slot_put = RK_NS - 1;
  for (int t = warp; t < tiles; t += warps) {
    const Tile now = q[0];
    if (q[RK_NS - 1].n) load(q[RK_NS - 1], slot_put);
    cp_async_commit();
    if (++slot_put == RK_NS) slot_put = 0;
#pragma unroll
    for (int i = 0; i < RK_NS - 1; ++i) q[i] = q[i + 1];
    q[RK_NS - 1] = look(t + RK_NS * warps);
    cp_async_wait<RK_NS - 1>();
    __syncwarp();  // every lane's copies have landed and are visible to the warp
    const uint32_t ks = ring + slot * C::STAGE + get_k, vs = ring + slot * C::STAGE + C::HALF + get_v;
    float s[4] = {0.f, 0.f, 0.f, 0.f};  // keys lane / 4 and 8 on, two vectors each
#pragma unroll
    for (int kk = 0; kk < DH / 16; ++kk) {
      uint32_t k[4];
      ldsm4(ks ^ (kk << 5), k);
      mma16816(s, k, qf[kk][0], qf[kk][1]);
    }
    float corr[2], x[4];
    bool sees[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const int vec = (lane & 3) * 2 + v;
      sees[v] = vec >= (now.cols & 255) && vec < (now.cols >> 8 & 255);
      const int n = !sees[v] ? 0 : now.cols >> 16 ? min(now.n, limit[v] - now.k0) : now.n;
      x[v] = (lane >> 2) < n ? s[v] * a.scale_log2 : -INFINITY;
      x[v + 2] = (lane >> 2) + 8 < n ? s[v + 2] * a.scale_log2 : -INFINITY;
      float mx = fmaxf(x[v], x[v + 2]);
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const float mn = fmaxf(m[v], mx), mz = mn == -INFINITY ? 0.f : mn;
      corr[v] = ex2(m[v] - mz);  // (0 while m is -infinity)
      m[v] = mn;
      x[v] = ex2(x[v] - mz);
      x[v + 2] = ex2(x[v + 2] - mz);
      l[v] = l[v] * corr[v] + (x[v] + x[v + 2]);
    }
    const uint32_t p0 = transpose8(pack_bf16x2(x[0], x[1])), p1 = transpose8(pack_bf16x2(x[2], x[3]));
    if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
      for (int d = 0; d < DH / 16; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[d][c] *= corr[c & 1];
    }
    if ((now.cols & 0xffff) == whole) {
#pragma unroll
      for (int d = 0; d < DH / 16; ++d) {
        uint32_t vt[4];
        ldsm4_t(vs ^ (d << 5), vt);
        mma16816(o[d], vt, p0, p1);
      }
    } else {  // (a zero weight times a NaN of another row's keys is no zero)
#pragma unroll
      for (int d = 0; d < DH / 16; ++d) {
        uint32_t vt[4];
        float y[4] = {0.f, 0.f, 0.f, 0.f};
        ldsm4_t(vs ^ (d << 5), vt);
        mma16816(y, vt, p0, p1);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[d][c] += sees[c & 1] ? y[c] : 0.f;
      }
    }
    __syncwarp();  // the tile is read before a lane's next copies overwrite it
    if (++slot == RK_NS) slot = 0;
  }
  // the join: every warp's (m, l) and, over its tiles, its O
  float* os = reinterpret_cast<float*>(row_ring + (size_t)warp * RK_NS * C::STAGE);
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    l[v] += __shfl_xor_sync(0xffffffffu, l[v], 4);
    l[v] += __shfl_xor_sync(0xffffffffu, l[v], 8);
    l[v] += __shfl_xor_sync(0xffffffffu, l[v], 16);
    const int vec = (lane & 3) * 2 + v;
    if (lane < 4) ml_s[warp][vec] = make_float2(m[v], l[v]);
    if (vec < nr * G) {
#pragma unroll
      for (int d = 0; d < DH / 16; ++d) {
        os[vec * DH + d * 16 + (lane >> 2)] = o[d][v];
        os[vec * DH + d * 16 + 8 + (lane >> 2)] = o[d][v + 2];
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nr * G * (DH / 2); i += blockDim.x) {  // two values of a vector each
    const int vec = i / (DH / 2), d = i % (DH / 2) * 2;
    if (!(lives >> (vec / G) & 1)) continue;  // (a row of no sequence stays as it is)
    float mm = -INFINITY, ll = 0.f, y0 = 0.f, y1 = 0.f;
    for (int w = 0; w < warps; ++w) mm = fmaxf(mm, ml_s[w][vec].x);
    const float mz = mm == -INFINITY ? 0.f : mm;
#pragma unroll 4
    for (int w = 0; w < warps; ++w) {
      const float2 ml = ml_s[w][vec];
      const float c = ex2(ml.x - mz);
      const float2 y = *reinterpret_cast<const float2*>(row_ring + (size_t)w * RK_NS * C::STAGE + (vec * DH + d) * 4);
      ll += ml.y * c;
      y0 += y.x * c;
      y1 += y.y * c;
    }
    const int r = vec / G, h = kvh * G + vec - r * G;
    const float inv = ll == 0.f ? 0.f : 1.f / ll;  // (NaN stays NaN)
    *reinterpret_cast<uint32_t*>(a.out + (r0 + r) * a.ld_out + (long long)h * DH + d) = pack_bf16x2(y0 * inv, y1 * inv);
    if (a.lse && d == 0) a.lse[(size_t)(r0 + r) * a.Hq + h] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.69314718055994531f;
  }
  // lengths outside the tables, of all sequences and groups (last: nothing waits for it)
  if (kvh == 0 && warp == 0)
    for (int i = blockIdx.y * 32 + lane; i < a.B + a.n_groups; i += gridDim.y * 32) {
      const int n = __ldg(i < a.B ? a.lens + i : a.plens + i - a.B);
      if (n < 0 || n > (i < a.B ? cap : pcap)) set_error(a.err, SP_DEVERR_INDEX);
    }
}

}  // namespace

// What a call launches, from what the host knows, and its workspace.
struct PrefixLayout {
  PlanArgs warp, tc;       // the kernel for few vectors per entry, the one for many (workers 0: not launched)
  size_t off_warp, off_tc; // their parts of the workspace
  size_t bytes;
};

// Vectors per entry from which its products can go to prefix_tc_kernel.
constexpr int kTcVectors = 32;
// They stay with prefix_warp_kernel, whose start is shorter, while that has no more than kFewTiles key tiles of 16
// vectors per warp of the GPU, taking every sequence and prefix as long as the tables can hold and the rows as evenly
// spread, and none has more than kFewKeys keys (whose many segments cost the merge more).  Us of a call with that
// kernel and with prefix_tc_kernel, 40 heads of 128 and one kv head: 16 rows and a prefix of 250 keys (0.5 tiles per
// warp) 11.5 and 15.4, of 2,000 (4) 18.8 and 17.9, 64 rows and 250 keys (2) 15.1 and 16.7; 64 heads, 4 kv heads, 64 rows
// in 16 prefixes of 250 keys (3.4) 17.4 and 19.3 (the second each with a prefix table for 2,064 positions); of 1,000 (13;
// 28 heads, once with the limit raised) 30 and 22.
constexpr int kFewTiles = 7, kFewKeys = 2048;

// A plan's arrays in its part of the workspace (base NULL: sizes only); returns its bytes.
static size_t plan_carve(PlanArgs* p, char* base, int T_cap, int B, int n_groups, int G, int Hkv, int dh) {
  const size_t full = ((size_t)T_cap * G) / p->tile_rows;  // row tiles besides each entry's last
  const size_t items = ((p->prefix ? full + n_groups : 0) + (p->own ? full + B : 0)) * Hkv;
  p->max_items = (int)items;
  const size_t rows = (items + p->workers) * p->slot_rows, E = (size_t)n_groups + B + 1;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* at = base + off;
    off = (off + bytes + 255) & ~size_t(255);
    return at;
  };
  p->unit0 = reinterpret_cast<int*>(take(E * 4));
  p->item0 = reinterpret_cast<int*>(take(E * 4));
  p->rows_prefix = reinterpret_cast<int4*>(take(p->prefix ? (size_t)T_cap * 16 : 0));
  p->rows_own = reinterpret_cast<int4*>(take(p->own ? (size_t)T_cap * 16 : 0));
  p->part_ml = reinterpret_cast<float2*>(take(rows * 8));
  p->part_o = reinterpret_cast<float*>(take(rows * dh * 4));
  return off;
}

// keys_prefix, keys_own: what the tables can hold of a prefix, of a sequence.
static PrefixLayout prefix_layout(int T_cap, int B, int n_groups, int Hq, int Hkv, int dh, long long keys_prefix,
                                  long long keys_own) {
  PrefixLayout L = {};
  const int G = Hq / Hkv, sms = device_sm_count();
  const bool fits = G <= 128;
  bool tc_prefix = fits && n_groups > 0 && (long long)T_cap * G >= (long long)kTcVectors * n_groups;
  bool tc_own = fits && (long long)T_cap * G >= (long long)kTcVectors * B;
  auto tiles = [&](int entries, long long keys) {
    return ((long long)T_cap * G / WK_ROWS + entries) * Hkv * ((keys + WK_KEYS - 1) / WK_KEYS);
  };
  if (std::max(tc_prefix ? keys_prefix : 0, tc_own ? keys_own : 0) <= kFewKeys &&
      (tc_prefix ? tiles(n_groups, keys_prefix) : 0) + (tc_own ? tiles(B, keys_own) : 0) <= (long long)kFewTiles * sms * WK_WARPS)
    tc_prefix = tc_own = false;
  L.warp.tile_rows = G <= WK_ROWS ? WK_ROWS / G * G : WK_ROWS;  // (whole rows where they fit)
  L.warp.key_shift = 4;
  L.warp.over = 2;
  L.warp.min_shift = 2;
  L.warp.prefix = n_groups > 0 && !tc_prefix;
  L.warp.own = !tc_own;
  L.warp.workers = L.warp.prefix || L.warp.own ? sms * WK_WARPS : 0;
  L.warp.slot_rows = (int)std::min<size_t>(L.warp.tile_rows, (size_t)T_cap * G);
  L.tc.tile_rows = fits ? 128 / G * G : 128;
  L.tc.key_shift = 7;
  L.tc.over = 4;     // (a segment of one tile takes as long as four more tiles in a row)
  L.tc.min_shift = 2;
  L.tc.prefix = tc_prefix;
  L.tc.own = tc_own;
  L.tc.workers = tc_prefix || tc_own ? sms : 0;
  L.tc.slot_rows = (int)std::min<size_t>(L.tc.tile_rows, (size_t)T_cap * G);
  L.off_warp = 0;
  if (L.warp.workers) L.bytes = plan_carve(&L.warp, nullptr, T_cap, B, n_groups, G, Hkv, dh);
  L.off_tc = L.bytes;
  if (L.tc.workers) L.bytes += plan_carve(&L.tc, nullptr, T_cap, B, n_groups, G, Hkv, dh);
  return L;
}

// Rows and warps of a CTA of prefix_row_kernel where a call goes to it (rows 0: it does not): up to RK_VECS heads per kv
// head, as long as a warp's share of the CTA's tiles, with tables as full as they can be and rows evenly spread, is short
// (kRowTiles), or no prefix is read by two CTAs of a kv head and half the SMs have one (kRowTilesAlone).  Us with it and
// without (the same call with tables for 16,400 positions), single tokens: four rows of 32 heads of 128, one prefix of 240
// and 20 own keys (1.2 tiles a warp) 5.7 and 11.0, of 2,000 keys (9) 14.9 and 18.4; 16 rows of 28 heads, 4 kv heads, 2,000
// keys (9) 14.7 and 18.2; without sharing, 64 rows of 32 heads and 500 keys (33, CTAs of one warp) 93 and 94.  Questions:
// 3 rows of 28 heads and 250 keys 7.5 and 10.6, four of 16 rows and 1,000 keys (11) 15.8 and 19.2, 16 of 48 rows without a
// prefix (6, CTAs of one warp) 21.7 and 30.6, of 32 heads on as many kv heads 24.0 and 46.0.  Beyond the limits (each once
// with the limit raised): 4 rows, 4,000 keys (18) 22.3 and 19.3; 64 rows, one prefix of 2,944 keys (27) 33.0 and 23.3; not
// CTAs of one warp for few rows of a sequence that lie in several: 128 of 4 rows 22.1 and 16.3.
struct RowLayout {
  int rows, warps;
};
constexpr int kRowTiles = 12, kRowTilesAlone = 36;
// Rows of a CTA are doubled, up to the rows of a prefix, while the warps of the GPU would have more tiles than this each:
// below that the SMs are better used by a row each.
constexpr int kRowSpread = 2;
static RowLayout row_layout(const PrefixArgs& a, int dh, int sms) {
  const int G = a.Hq / a.Hkv, T = a.T_cap;
  if (G > RK_VECS) return {0, 0};
  const int per = std::max(1, T / a.B);  // rows of a sequence
  const int share = a.n_groups > 0 ? std::max(1, T / a.n_groups) : per;  // rows of a prefix
  const long long pt = ((long long)a.pmax_pages << a.page_shift) / WK_KEYS, ot = ((long long)a.max_pages << a.page_shift) / WK_KEYS;
  const int most = dh == 128 ? RkCfg<128>::WARPS : RkCfg<64>::WARPS;
  const int warp_smem = RK_NS * (dh == 128 ? RkCfg<128>::STAGE : RkCfg<64>::STAGE);
  const int sm_warps = dh == 128 ? RkCfg<128>::SM_WARPS : RkCfg<64>::SM_WARPS;
  auto places = [&](int R) { return (long long)(T + R - 1) / R * a.Hkv; };
  auto tiles = [&](int R) { return (R + share - 1) / share * pt + (R + per - 1) / per * ot; };
  int R = 1;
  while (2 * R * G <= RK_VECS && R < share && places(R) * tiles(R) > (long long)kRowSpread * sms * sm_warps) R *= 2;
  // as many warps as let all CTAs be there at once (2 KB: a CTA's other shared memory)
  int warps = (int)std::max(1ll, std::min<long long>(most, tiles(R)));
  while (warps > 1 && (227 * 1024) / (warps * warp_smem + 2048) * (long long)sms < places(R)) --warps;
  if (places(R) > 64ll * sms || (warps == 1 && R < per && (long long)T * G < (long long)kTcVectors * a.B)) return {0, 0};
  const bool alone = R % share == 0 && 2 * places(R) >= sms;
  return tiles(R) <= (long long)(alone ? kRowTilesAlone : kRowTiles) * warps ? RowLayout{R, warps} : RowLayout{0, 0};
}

static cudaError_t prefix_attention_launch(const PrefixArgs& a, int dh, void* ws, cudaStream_t st) {
  if (a.T_cap == 0) return cudaSuccess;
  if (const RowLayout x = row_layout(a, dh, device_sm_count()); x.rows) {
    const size_t warp_smem = RK_NS * (dh == 128 ? RkCfg<128>::STAGE : RkCfg<64>::STAGE);
    auto* kern = dh == 128 ? prefix_row_kernel<128> : prefix_row_kernel<64>;
    static std::atomic<unsigned long long> allowed[2];
    cudaError_t r = allow_smem(kern, warp_smem * (dh == 128 ? RkCfg<128>::WARPS : RkCfg<64>::WARPS), allowed[dh == 128]);
    if (r != cudaSuccess) return r;
    prof_begin_launch(st);
    r = launch_pdl(kern, dim3(a.Hkv, (a.T_cap + x.rows - 1) / x.rows), dim3(x.warps * 32), warp_smem * x.warps, st, a,
                   x.rows, a.T_cap);
    prof_end_launch(st, SP_K_ATTN, 0.0, 0.0);
    return r;
  }
  PrefixLayout L = prefix_layout(a.T_cap, a.B, a.n_groups, a.Hq, a.Hkv, dh, (long long)a.pmax_pages << a.page_shift,
                                 (long long)a.max_pages << a.page_shift);
  const int sms = device_sm_count(), G = a.Hq / a.Hkv;
  char* base = static_cast<char*>(ws);
  cudaError_t r;
  if (L.tc.workers) {
    plan_carve(&L.tc, base + L.off_tc, a.T_cap, a.B, a.n_groups, G, a.Hkv, dh);
    prof_begin_launch(st);
    r = prefix_tc_launch(a, L.tc, dh, st);
    prof_end_launch(st, SP_K_ATTN, 0.0, 0.0);
    if (r != cudaSuccess) return r;
  }
  if (L.warp.workers) {
    plan_carve(&L.warp, base + L.off_warp, a.T_cap, a.B, a.n_groups, G, a.Hkv, dh);
    const size_t smem = dh == 128 ? WkCfg<128>::SMEM : WkCfg<64>::SMEM;
    auto* kern = dh == 128 ? prefix_warp_kernel<128> : prefix_warp_kernel<64>;
    static std::atomic<unsigned long long> allowed[2];
    r = allow_smem(kern, smem, allowed[dh == 128]);
    if (r != cudaSuccess) return r;
    prof_begin_launch(st);
    r = launch_pdl(kern, dim3(sms), dim3(WK_NT), smem, st, a, L.warp, L.tc.workers ? 1 : 0);
    prof_end_launch(st, SP_K_ATTN, 0.0, 0.0);
    if (r != cudaSuccess) return r;
  }
  const PlanArgs &pp = L.tc.prefix ? L.tc : L.warp, &po = L.tc.own ? L.tc : L.warp;
  prof_begin_launch(st);
  r = dh == 128 ? launch_merge<128>(a, pp, po, st) : launch_merge<64>(a, pp, po, st);
  prof_end_launch(st, SP_K_ATTN, 0.0, 0.0);
  return r;
}

size_t prefix_attention_bytes(int T_cap, int B, int n_groups, int Hq, int Hkv, int dh) {
  // (for tables of any width)
  return std::max(prefix_layout(T_cap, B, n_groups, Hq, Hkv, dh, 0, 0).bytes,
                  prefix_layout(T_cap, B, n_groups, Hq, Hkv, dh, kFewKeys + 1, kFewKeys + 1).bytes);
}

cudaError_t prefix_attention(const PrefixAttention& x, void* ws, cudaStream_t st) {
  PrefixArgs a;
  a.q = static_cast<const __nv_bfloat16*>(x.q);
  a.ld_q = x.ld_q;
  a.out = static_cast<__nv_bfloat16*>(x.out);
  a.ld_out = x.ld_out;
  a.lse = x.lse;
  a.kv = static_cast<const __nv_bfloat16*>(x.kv);
  a.n_pages = x.n_pages;
  a.page_shift = __builtin_ctz(x.page_size);
  a.table = x.table;
  a.max_pages = x.max_pages;
  a.lens = x.lens;
  a.ptable = x.ptable;
  a.pmax_pages = x.pmax_pages;
  a.plens = x.plens;
  a.group_cu = x.group_cu;
  a.n_groups = x.n_groups;
  a.cu_rows = x.cu_rows;
  a.B = x.B;
  a.T_cap = x.T_cap;
  a.Hq = x.Hq;
  a.Hkv = x.Hkv;
  a.scale_log2 = (x.scale > 0.f ? x.scale : 1.f / sqrtf((float)x.dh)) * 1.4426950408889634f;
  a.err = x.err;
  return prefix_attention_launch(a, x.dh, ws, st);
}

}  // namespace sp
