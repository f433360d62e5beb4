// Attention over shared prefixes, many query vectors per entry: tcgen05 products on row tiles of up to 128
// vectors (whole rows of the kv head's G query heads: 128 / G rows).  prefix_plan.cuh says how the work is
// cut; prefix_merge_kernel (prefix_attn.cu) joins the segments.
//
// One CTA per SM with two independent pipelines, each a worker of the plan with its own tiles: while one
// waits for its softmax the other's products run.  A key tile is 64 keys.
//
//   warps 0 / 3   loads of pipeline 0 / 1 by TMA: the Q tile once per segment, then per key tile the K and V
//                 rows, one box per page (and 64 columns), into two-slot rings.  Rows past the entry's keys
//                 are not to be multiplied: a zero weight times what lies there (NaN, say) is no zero, so the
//                 warp clears those rows of V in shared memory behind the copy.
//   warps 1 / 12  issue the scores S = Q K^T (M 128, N 64) into one of two S / P buffers in tensor memory
//                 (warp 1 also allocates its 512 columns)
//   warps 2 / 13  issue O += P V (P from tensor memory, where the softmax wrote it over its S)
//   warps 4-7     softmax of pipeline 0, warps 8-11 of pipeline 1: a thread per query vector (= lane of tensor
//                 memory); O is rescaled only when the running max moves by more than 2^8 (O and the sum share
//                 the max that was used, so the result is exact); at the segment's end (max, sum) and O go to
//                 the segment's slot.
// Tensor memory: S / P buffer b of pipeline t at columns 128 t + 64 b, O of pipeline t at 256 + DH t.
// Bound by the exponentials and the chain scores -> softmax -> product within a pipeline.
#include <algorithm>

#include "internal.h"
#include "prefix_plan.cuh"

namespace sp {

namespace {

constexpr int TC_KV = 64, TC_NT = 448;
constexpr float kRescaleLog2 = 8.f;

template <int DH>
struct TcCfg {
  static constexpr uint32_t BOX_Q = 128 * 128;             // 128 vectors x 64 elements
  static constexpr uint32_t BOX_KV = TC_KV * 128;
  static constexpr uint32_t Q_BYTES = DH / 64 * BOX_Q;
  static constexpr uint32_t KV_BYTES = DH / 64 * BOX_KV;
  static constexpr uint32_t OFF_Q = 0;                     // [2 pipelines]
  static constexpr uint32_t OFF_K = 2 * Q_BYTES;           // [2 pipelines][2 slots]
  static constexpr uint32_t OFF_V = OFF_K + 4 * KV_BYTES;
  static constexpr uint32_t OFF_BAR = OFF_V + 4 * KV_BYTES;
  static constexpr size_t SMEM_USED = 1024 + OFF_BAR + 512;
  // more than half of the shared memory: a second CTA would only wait for the tensor memory
  static constexpr size_t SMEM = SMEM_USED > 116 * 1024 ? SMEM_USED : 116 * 1024;
  static constexpr uint32_t T_O = 256;
};

// Per pipeline t: Q_FULL, Q_EMPTY, O_FULL, O_EMPTY, V_TAIL (the copies of a tile whose rows are cleared next)
// + t; per slot / buffer b of it: X + 2 t + b.  K_FULL counts the copies (with their bytes) and the end of
// O += P V two tiles before, the last reader of the S / P buffer that the scores will overwrite (the loader
// arrives twice for the first two tiles); P_FULL the four softmax warps and the copies of V.  A K slot is free
// when its scores are done (S_FULL), a V slot when its product is (PV_DONE).
enum TcBar {
  Q_FULL = 0, Q_EMPTY = 2, K_FULL = 4, S_FULL = 8, P_FULL = 12, PV_DONE = 16, O_FULL = 20, O_EMPTY = 22, V_TAIL = 24,
  MMA_DONE = 26, TC_BARS = 30
};

SP_DEVINL float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

SP_DEVINL float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

SP_DEVINL void tma_load_3d(void* smem_dst, const void* tmap, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(smem_u32(smem_dst)), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}

// The segments of one worker, one after the other.
struct SegWalk {
  TileCursor c;
  long long t, t1;
  int n;  // tiles of the present segment: c.j .. c.j + n - 1 of its item
  SP_DEVINL bool begin(const PlanShared& s, const PlanArgs& p, int E, int Hkv, long long N, int w) {
    const int P = plan_workers(N, p.workers, p.min_tiles);
    if (N == 0 || w >= P) return false;
    t = part_begin(N, P, w);
    t1 = part_begin(N, P, w + 1);
    if (t >= t1) return false;
    c.seek(s, p, E, Hkv, t);
    size();
    return true;
  }
  SP_DEVINL void size() { n = (int)(t1 - t < c.kt - c.j ? t1 - t : c.kt - c.j); }
  SP_DEVINL bool next(const PlanShared& s, const PlanArgs& p, int Hkv) {
    t += n;
    if (t >= t1) return false;
    c.j = c.kt - 1;
    c.next(s, p, Hkv);
    size();
    return true;
  }
};

template <int DH>
__global__ void __launch_bounds__(TC_NT, 1)
prefix_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const PrefixArgs a, const PlanArgs p) {
  using C = TcCfg<DH>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ PlanShared plan;
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bar = reinterpret_cast<uint64_t*>(sm + C::OFF_BAR);
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + TC_BARS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int E = a.n_groups + a.B, G = a.Hq / a.Hkv;

  if (threadIdx.x == 0) {
    for (int i = 0; i < TC_BARS; ++i)
      mbar_init(&bar[i], (i >= P_FULL && i < P_FULL + 4)              ? 5
                         : (i == O_EMPTY || i == O_EMPTY + 1)         ? 4
                         : (i >= K_FULL && i < K_FULL + 4)            ? 2
                                                                      : 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(tslot, 512);
    tmem_relinquish();
  }
  // vectors behind a tile's last row are multiplied too (to nothing): let them be zeros, not what was there
  for (uint32_t i = threadIdx.x * 16; i < 2 * C::Q_BYTES; i += TC_NT * 16)
    *reinterpret_cast<uint4*>(sm + C::OFF_Q + i) = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;
  pdl_wait();
  pdl_trigger();
  build_plan<TC_NT>(a, p, plan, blockIdx.x == 0);
  const long long N = plan.tile0[E];

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------ loads of pipeline t
    const int t = warp == 3;
    SegWalk sg;
    bool more = sg.begin(plan, p, E, a.Hkv, N, blockIdx.x + t * gridDim.x);
    uint32_t g = 0, nseg = 0;
    bool ok = true;
    uint8_t* sQ = sm + C::OFF_Q + t * C::Q_BYTES;
    const int brows = min(TC_KV, 1 << a.page_shift);  // rows of a box: a page's, or the tile's
    const int rows_per_tile = 128 / G;
    uint32_t tails = 0;
    while (ok && more) {
      const bool pre = sg.c.e < a.n_groups;
      const int* tb = pre ? a.ptable + (size_t)sg.c.e * a.pmax_pages
                          : a.table + (size_t)(sg.c.e - a.n_groups) * a.max_pages;
      const int keys = plan.keys[sg.c.e];
      // lane i < boxes of a tile: page of its box of tile j
      auto page_of = [&](int j) {
        const int k = j * TC_KV + lane * brows;
        return lane * brows < TC_KV && k < keys ? __ldg(tb + (k >> a.page_shift)) : -1;
      };
      int page = page_of(sg.c.j);
      if (!mbar_wait_warp(&bar[Q_EMPTY + t], (nseg & 1) ^ 1u, a.err)) { ok = false; break; }
      if (lane == 0) {
        mbar_arrive_expect_tx(&bar[Q_FULL + t], DH / 64 * 128u * (uint32_t)(rows_per_tile * G));
#pragma unroll
        for (int bx = 0; bx < DH / 64; ++bx)
          tma_load_3d(sQ + bx * C::BOX_Q, &tmQ, &bar[Q_FULL + t], bx * 64, sg.c.kvh * G,
                      plan.row0[sg.c.e] + sg.c.rt * rows_per_tile);
      }
      ++nseg;
      for (int j = sg.c.j; j < sg.c.j + sg.n; ++j, ++g) {
        const uint32_t st = g & 1, pe = ((g >> 1) & 1) ^ 1u;
        uint8_t* sK = sm + C::OFF_K + (2 * t + st) * C::KV_BYTES;
        uint8_t* sV = sm + C::OFF_V + (2 * t + st) * C::KV_BYTES;
        uint64_t* kfull = &bar[K_FULL + 2 * t + st];
        uint64_t* vfull = &bar[P_FULL + 2 * t + st];
        const int k0 = j * TC_KV, here = min(TC_KV, keys - k0);
        const bool mine = lane * brows < here;  // a box of this lane's is wanted
        const bool good = mine && page >= 0 && page < a.n_pages;
        if (mine && !good) set_error(a.err, SP_DEVERR_INDEX);
        const unsigned int boxes = __ballot_sync(0xffffffffu, good);
        const bool bad = __any_sync(0xffffffffu, mine && !good);
        const int row = (page << a.page_shift) + ((k0 + lane * brows) & ((1 << a.page_shift) - 1));
        const uint32_t bytes = (uint32_t)__popc(boxes) * (uint32_t)brows * (DH * 2);
        page = j + 1 < sg.c.j + sg.n ? page_of(j + 1) : -1;
        // clears rows r0 .. r1 - 1 of a tile of 64 keys
        auto clear = [&](uint8_t* s, int r0, int r1) {
          for (int i = lane; i < (r1 - r0) * 8 * (DH / 64); i += 32) {
            const int bx = i / ((r1 - r0) * 8), k = i - bx * ((r1 - r0) * 8);
            *reinterpret_cast<uint4*>(s + bx * C::BOX_KV + r0 * 128 + k * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        };
        if (g >= 2 && !mbar_wait_warp(&bar[S_FULL + 2 * t + st], pe, a.err)) { ok = false; break; }
        if (bad) {  // a page outside the pool: its keys are zeros
          for (int b = 0; b * brows < here; ++b)
            if (!((boxes >> b) & 1)) clear(sK, b * brows, (b + 1) * brows);
          fence_proxy_async_smem();
          __syncwarp();
        }
        if (lane == 0) {
          mbar_arrive_expect_tx(kfull, bytes);
          if (g < 2) mbar_arrive(kfull);  // (no product two tiles before)
        }
        __syncwarp();
        if (good) {
#pragma unroll
          for (int bx = 0; bx < DH / 64; ++bx)
            tma_load_2d(sK + bx * C::BOX_KV + lane * brows * 128, &tmK, kfull, sg.c.kvh * DH + bx * 64, row);
        }
        if (g >= 2 && !mbar_wait_warp(&bar[PV_DONE + 2 * t + st], pe, a.err)) { ok = false; ++g; break; }
        const bool tail = here < TC_KV || bad;
        uint64_t* vbar = tail ? &bar[V_TAIL + t] : vfull;
        if (lane == 0) mbar_arrive_expect_tx(vbar, bytes);
        __syncwarp();
        if (good) {
#pragma unroll
          for (int bx = 0; bx < DH / 64; ++bx)
            tma_load_2d(sV + bx * C::BOX_KV + lane * brows * 128, &tmV, vbar, sg.c.kvh * DH + bx * 64, row);
        }
        if (tail) {
          if (!mbar_wait_warp(vbar, tails & 1, a.err)) { ok = false; ++g; break; }
          ++tails;
          if (bad)
            for (int b = 0; b * brows < here; ++b)
              if (!((boxes >> b) & 1)) clear(sV, b * brows, (b + 1) * brows);
          if (here < TC_KV) clear(sV, here, TC_KV);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(vfull);
        }
      }
      if (ok) more = sg.next(plan, p, a.Hkv);
    }
    // every copy lands before the CTA may exit (bounded waits; normally the consumers have waited for them)
    if (nseg > 0) mbar_wait_warp(&bar[Q_FULL + t], (nseg - 1) & 1, a.err);
    for (uint32_t gg = g >= 2 ? g - 2 : 0; gg < g; ++gg) {
      mbar_wait_warp(&bar[K_FULL + 2 * t + (gg & 1)], (gg >> 1) & 1, a.err);
      mbar_wait_warp(&bar[P_FULL + 2 * t + (gg & 1)], (gg >> 1) & 1, a.err);
    }
  } else if (warp == 1 || warp == 2 || warp >= 12) {
    // ------------------------------------------------------------ issuers of pipeline t
    if (lane == 0) {
      const int t = warp >= 12 ? 1 : 0;
      const bool pv_issuer = warp == 2 || warp == 13;
      constexpr uint32_t IDESC_S = umma_idesc_bf16_f32(128, TC_KV);
      constexpr uint32_t IDESC_O = umma_idesc_bf16_f32(128, DH) | (1u << 16);  // V: MN-major
      const uint64_t dQ = umma_desc_sw128(smem_u32(sm + C::OFF_Q + t * C::Q_BYTES));
      const uint64_t dK = umma_desc_sw128(smem_u32(sm + C::OFF_K + 2 * t * C::KV_BYTES));
      const uint64_t dV = umma_desc_sw128_mn(smem_u32(sm + C::OFF_V + 2 * t * C::KV_BYTES), C::BOX_KV);
      const uint64_t slot16 = C::KV_BYTES >> 4;
      const uint32_t tS = tmem + t * 128, tO = tmem + C::T_O + t * DH;
      SegWalk sg;
      bool more = sg.begin(plan, p, E, a.Hkv, N, blockIdx.x + t * gridDim.x);
      uint32_t g = 0, nseg = 0;
      bool ok = true;
      while (ok && more) {
        if (!pv_issuer) {
          ok = mbar_wait(&bar[Q_FULL + t], nseg & 1, a.err);
          for (int j = 0; ok && j < sg.n; ++j) {
            const uint32_t gg = g + j, b = gg & 1;
            if (!mbar_wait(&bar[K_FULL + 2 * t + b], (gg >> 1) & 1, a.err)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk)
              umma_bf16(tS + b * TC_KV, dQ + (((kk >> 2) * C::BOX_Q + (kk & 3) * 32) >> 4),
                        dK + b * slot16 + (((kk >> 2) * C::BOX_KV + (kk & 3) * 32) >> 4), IDESC_S, kk ? 1u : 0u);
            umma_commit(&bar[S_FULL + 2 * t + b]);
            if (j + 1 == sg.n) umma_commit(&bar[Q_EMPTY + t]);
          }
        } else {
          for (int j = 0; ok && j < sg.n; ++j) {
            const uint32_t gg = g + j, b = gg & 1;
            if (!mbar_wait(&bar[P_FULL + 2 * t + b], (gg >> 1) & 1, a.err) ||
                (j == 0 && !mbar_wait(&bar[O_EMPTY + t], (nseg & 1) ^ 1u, a.err))) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < TC_KV / 16; ++kk)
              umma_bf16_ta(tO, tS + b * TC_KV + kk * 8, dV + b * slot16 + ((kk * 2048) >> 4), IDESC_O,
                           (j | kk) ? 1u : 0u);
            umma_commit(&bar[PV_DONE + 2 * t + b]);
            umma_commit(&bar[K_FULL + 2 * t + b]);  // (counts toward the K barrier of the tile after the next)
            if (j + 1 == sg.n) umma_commit(&bar[O_FULL + t]);
          }
        }
        g += sg.n;
        ++nseg;
        more = sg.next(plan, p, a.Hkv);
      }
      // tensor memory stays allocated until every product this thread issued is done
      umma_commit(&bar[MMA_DONE + 2 * t + (pv_issuer ? 1 : 0)]);
      mbar_wait(&bar[MMA_DONE + 2 * t + (pv_issuer ? 1 : 0)], 0, a.err);
    }
    __syncwarp();
  } else if (warp >= 4 && warp < 12) {
    // ------------------------------------------------------------ softmax (vector = lane of tensor memory)
    const int t = (warp - 4) >> 2;
    const int quad = warp & 3;
    const int r = quad * 32 + lane;
    const uint32_t trow = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t tS = trow + t * 128, tO = trow + C::T_O + t * DH;
    const int w = blockIdx.x + t * gridDim.x;
    SegWalk sg;
    bool more = sg.begin(plan, p, E, a.Hkv, N, w);
    uint32_t g = 0, nseg = 0;
    bool ok = true;
    while (ok && more) {
      const int M = plan.rows[sg.c.e] * G, keys = plan.keys[sg.c.e];
      const int mv = sg.c.rt * p.tile_rows + r;
      const bool have = r < p.tile_rows && mv < M;
      int row_lim = 0;  // keys [0, row_lim) are visible
      if (have) row_lim = sg.c.e < a.n_groups ? keys : min(max(keys - plan.rows[sg.c.e] + mv / G + 1, 0), keys);
      float m = -INFINITY, l = 0.f;  // m: the max in use, log2 units
      for (int j = sg.c.j; j < sg.c.j + sg.n; ++j, ++g) {
        const uint32_t b = g & 1;
        if (!mbar_wait_warp(&bar[S_FULL + 2 * t + b], (g >> 1) & 1, a.err)) { ok = false; break; }
        tc_fence_after();
        float v[TC_KV];
        tmem_ld_32x32b_x32(tS + b * TC_KV, *reinterpret_cast<float(*)[32]>(v));
        tmem_ld_32x32b_x32(tS + b * TC_KV + 32, *reinterpret_cast<float(*)[32]>(v + 32));
        tmem_ld_wait();
        const int lim = row_lim - j * TC_KV;
        if (lim < TC_KV) {
#pragma unroll
          for (int c = 0; c < TC_KV; ++c) v[c] = c < lim ? v[c] : -INFINITY;
        }
        float mx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = max3(v[e], v[e + 8], v[e + 16]);
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = max3(mx[e], v[e + 24], v[e + 32]);
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = max3(mx[e], v[e + 40], v[e + 48]);
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(mx[e], v[e + 56]);
        const float mb =
            max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * a.scale_log2;
        float corr = 1.f;
        bool moved = false;
        if (mb > m + kRescaleLog2 || (m == -INFINITY && mb > -INFINITY)) {
          corr = m == -INFINITY ? 0.f : ex2(m - mb);
          moved = m != -INFINITY;
          m = mb;
        }
        const float nm = m == -INFINITY ? 0.f : -m;
        float ls[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) ls[e] = 0.f;
        float pk[TC_KV / 2];  // bf16 pairs
#pragma unroll
        for (int e = 0; e < TC_KV / 2; ++e) {
          const float p0 = ex2(fmaf(v[2 * e], a.scale_log2, nm)), p1 = ex2(fmaf(v[2 * e + 1], a.scale_log2, nm));
          ls[(2 * e) & 7] += p0;
          ls[(2 * e + 1) & 7] += p1;
          pk[e] = __uint_as_float(pack_bf16x2(p0, p1));
        }
        l = l * corr + ((ls[0] + ls[1]) + (ls[2] + ls[3])) + ((ls[4] + ls[5]) + (ls[6] + ls[7]));
        if (__any_sync(0xffffffffu, moved)) {
          // the product of the tile before is done with O before it is rescaled
          if (!mbar_wait_warp(&bar[PV_DONE + 2 * t + ((g - 1) & 1)], ((g - 1) >> 1) & 1, a.err)) { ok = false; break; }
          tc_fence_after();
          float o[32];
#pragma unroll 1
          for (int c = 0; c < DH; c += 32) {
            tmem_ld_32x32b_x32(tO + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= corr;
            tmem_st_32x32b_x32(tO + c, o);
          }
        }
        tmem_st_32x32b_x32(tS + b * TC_KV, pk);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[P_FULL + 2 * t + b]);
      }
      if (!ok) break;
      // ---- the segment's (max, sum) and O
      if (!mbar_wait_warp(&bar[O_FULL + t], nseg & 1, a.err)) { ok = false; break; }
      tc_fence_after();
      const size_t at = ((size_t)sg.c.item + w) * p.slot_rows + r;
      if (have) p.part_ml[at] = make_float2(m, l);
      float o[32];
#pragma unroll 1
      for (int c = 0; c < DH; c += 32) {
        tmem_ld_32x32b_x32(tO + c, o);
        tmem_ld_wait();
        if (have) {
          float4* d = reinterpret_cast<float4*>(p.part_o + at * DH + c);
#pragma unroll
          for (int q = 0; q < 8; ++q) d[q] = make_float4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[O_EMPTY + t]);
      ++nseg;
      more = sg.next(plan, p, a.Hkv);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int DH>
cudaError_t launch_tc(const PrefixArgs& a, const PlanArgs& p, cudaStream_t st) {
  using C = TcCfg<DH>;
  const int G = a.Hq / a.Hkv;
  CUtensorMap tq, tk, tv;
  const uint64_t rows = (uint64_t)a.n_pages << a.page_shift, W = (uint64_t)a.Hkv * DH;
  const uint32_t brows = (uint32_t)std::min(TC_KV, 1 << a.page_shift);
  if (!encode_tmap_rows3(&tq, a.q, DH, a.Hq, a.T_cap, (uint64_t)a.ld_q, 64, G, 128 / G) ||
      !encode_tmap_2d(&tk, a.kv, false, rows, W, 64, brows, nullptr) ||
      !encode_tmap_2d(&tv, a.kv + rows * W, false, rows, W, 64, brows, nullptr))
    return cudaErrorInvalidValue;
  const cudaError_t r =
      cudaFuncSetAttribute(prefix_tc_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM);
  if (r != cudaSuccess) return r;
  return launch_pdl(prefix_tc_kernel<DH>, dim3(p.workers / 2), dim3(TC_NT), C::SMEM, st, tq, tk, tv, a, p);
}

}  // namespace

cudaError_t prefix_tc_launch(const PrefixArgs& a, const PlanArgs& p, int dh, cudaStream_t st) {
  return dh == 128 ? launch_tc<128>(a, p, st) : launch_tc<64>(a, p, st);
}

}  // namespace sp
