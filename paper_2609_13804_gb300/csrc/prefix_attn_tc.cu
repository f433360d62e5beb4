// Attention over shared prefixes, many query vectors per entry: tcgen05 products on row tiles of up to 128
// vectors (whole rows of the kv head's G query heads: 128 / G rows).  prefix_plan.cuh says how the work is
// cut; prefix_merge_kernel (prefix_attn.cu) joins the segments.
//
// One CTA per SM is a worker of the plan; a key tile is 128 keys.
//
//   warp 0        Q and K by TMA: the Q tile once per segment, then per key tile its K rows, one box per page
//                 (and 64 columns), into a two-slot ring
//   warp 3        V by TMA into a three-slot ring.  Rows past the entry's keys are not to be multiplied: a zero
//                 weight times what lies there (NaN, say) is no zero, so the warp clears those rows in shared
//                 memory behind the copy.
//   warp 1        issues the scores S = Q K^T (M 128, N 128) into one of three S / P buffers of tensor memory
//                 (and allocates its 512 columns)
//   warp 2        issues O += P V (P from tensor memory, where the softmax wrote it over its S)
//   warps 4-7     softmax of the even tiles (counted over the CTA's whole walk), warps 8-11 of the odd ones: a
//                 thread per query vector (= lane of tensor memory)
// The two softmax streams work on consecutive tiles at once and share one O, so both scale by the same running
// max m.  m moves only when a tile's max exceeds it by more than 2^8 (O and the sums are rescaled then, so the
// result is exact); a tile hands its m to the next through shared memory, and that wait costs a row maximum, not
// a softmax.  Each stream sums with a reference max of its own; at the segment's end both are brought to the last
// m and added, and O, half its columns by each stream, goes through a small stage in shared memory to the
// segment's slot, in whole 64-byte pieces.  The scores run up to two tiles ahead; those of tile j + 3 reuse tile
// j's buffer once its O += P V is done.
// Tensor memory: S / P buffer b at columns 128 b, O at 384.
// Bound by the chain scores -> softmax -> product through the three buffers tensor memory holds: three tiles are in
// flight, and a tile takes 0.89 us of a CTA (by the difference of prefixes of 16,384 and 32,768 keys; 1,024 cycles of the
// tensor pipe).  128 rows of 28 query heads over 16,384 keys, the merge included: 41.7 us (720 TFLOP/s).  (Two pipelines
// of a row tile each with single 128-key buffers took 71 us when this took 51: only tiles in flight hide the chain.)
#include <algorithm>

#include "internal.h"
#include "prefix_plan.cuh"

namespace sp {

namespace {

constexpr int TC_KV = 128, TC_NT = 384, NSB = 3, NKS = 2, NVS = 3;
constexpr float kRescaleLog2 = 8.f;

template <int DH>
struct TcCfg {
  static constexpr uint32_t BOX = 128 * 128;               // 128 rows x 64 elements
  static constexpr uint32_t TILE = DH / 64 * BOX;          // a Q tile or a K / V tile
  static constexpr uint32_t OFF_Q = 0;
  static constexpr uint32_t OFF_K = TILE;                  // [NKS]
  static constexpr uint32_t OFF_V = OFF_K + NKS * TILE;    // [NVS]
  static constexpr uint32_t OFF_M = OFF_V + NVS * TILE;    // running max by tile parity: [2][128] floats
  static constexpr uint32_t OFF_L = OFF_M + 2 * 128 * 4;   // sums: [segment parity][stream][128] floats
  static constexpr uint32_t OFF_STG = OFF_L + 4 * 128 * 4; // output stage: [8 warps][32 rows][64 B]
  static constexpr uint32_t OFF_BAR = OFF_STG + 8 * 2048;
  static constexpr size_t SMEM_USED = 1024 + OFF_BAR + 256;
  // more than half of the shared memory: a second CTA would only wait for the tensor memory
  static constexpr size_t SMEM = SMEM_USED > 116 * 1024 ? SMEM_USED : 116 * 1024;
  static constexpr uint32_t T_O = 384;
  static_assert(SMEM + sizeof(PlanShared) <= 227 * 1024, "a CTA's shared memory");
};

// X + s for S / P buffer s (tile % 3).  K_FULL counts the copies of K (with their bytes) and the end of O += P V three tiles
// before, the last reader of the S / P buffer that the scores will overwrite (the loader arrives twice for the
// first three tiles); P_FULL the stream's four warps and the copies of V.  A K slot is free when its scores are
// done (S_FULL), a V slot when its product is (PV_DONE).  V_TAIL: the copies of a tile whose rows are cleared next;
// M_FULL + (tile & 1): its running max; XL: both streams' sums.
enum TcBar {
  Q_FULL = 0, Q_EMPTY = 1, K_FULL = 2, S_FULL = 5, P_FULL = 8, PV_DONE = 11, O_FULL = 14, O_EMPTY = 15, MMA_DONE = 16,
  M_FULL = 18, XL = 20, V_TAIL = 21, TC_BARS = 22
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

// Two fp32 numbers as one operand of the packed arithmetic: half the instructions of the exponents and sums.
SP_DEVINL unsigned long long pack2(float lo, float hi) {
  unsigned long long r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
SP_DEVINL void unpack2(unsigned long long v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
SP_DEVINL unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
SP_DEVINL unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Orders later uses of registers written by tcgen05.ld behind the tcgen05.wait::ld before this call.
template <int N>
SP_DEVINL void loaded(float (&r)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) asm volatile("" : "+f"(r[e]));
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
  int t1;
  int n;  // tiles of the present segment: c.j .. c.j + n - 1 of its item
  SP_DEVINL bool begin(const PlanShared& s, const PlanArgs& p, int E, int Hkv, int N, int w) {
    if (N == 0) return false;
    const int P = plan_workers(p, N);
    if (w >= P) return false;
    int t0;
    part_of_worker(N, P, w, t0, t1);
    if (!c.seek(s, p, E, Hkv, t0, t1)) return false;
    size();
    return true;
  }
  SP_DEVINL void size() { n = min(t1 - c.u, c.kt - c.j); }
  SP_DEVINL bool next(const PlanShared& s, const PlanArgs& p, int Hkv) {
    c.j += n - 1;
    c.u += n - 1;
    if (!c.next(s, p, Hkv, t1)) return false;
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
    for (int i = 0; i < TC_BARS; ++i) {
      uint32_t n = 1;
      if (i >= K_FULL && i < K_FULL + NSB) n = 2;
      if (i >= P_FULL && i < P_FULL + NSB) n = 5;
      if (i == O_EMPTY || i == XL) n = 8;           // all softmax warps
      if (i == M_FULL || i == M_FULL + 1) n = 4;    // a stream's warps
      mbar_init(&bar[i], n);
    }
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(tslot, 512);
    tmem_relinquish();
  }
  if (threadIdx.x == 96) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  // vectors behind a tile's last row are multiplied too (to nothing): let them be zeros, not what was there
  for (uint32_t i = threadIdx.x * 16; i < C::TILE; i += TC_NT * 16)
    *reinterpret_cast<uint4*>(sm + C::OFF_Q + i) = make_uint4(0u, 0u, 0u, 0u);
  fence_proxy_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tslot;
  // in this order: the kernel behind this one may read its inputs without a wait of its own (prefix_warp_kernel, late)
  pdl_wait();
  pdl_trigger();
  build_plan<TC_NT>(a, p, plan, blockIdx.x == 0);
  const int N = plan.unit0[E], w = blockIdx.x;
  SegWalk sg;
  bool more = sg.begin(plan, p, E, a.Hkv, N, w);
  bool ok = true;
  uint32_t g = 0, nseg = 0;  // tiles and segments so far

  if (warp == 0 || warp == 3) {
    // ------------------------------------------------------------ loads: Q and K (warp 0), V (warp 3)
    const bool is_v = warp == 3;
    const int brows = min(TC_KV, 1 << a.page_shift);  // rows of a box: a page's, or the tile's
    const int rows_per_tile = 128 / G;
    uint32_t tails = 0;
    while (ok && more) {
      const bool pre = sg.c.e < a.n_groups;
      const int* tb = pre ? a.ptable + (size_t)sg.c.e * a.pmax_pages
                          : a.table + (size_t)(sg.c.e - a.n_groups) * a.max_pages;
      const int keys = plan.keys[sg.c.e];
      // page of this lane's box of tile j (lanes beyond its boxes: none)
      auto page_of = [&](int j) {
        const int k = j * TC_KV + lane * brows;
        return lane * brows < TC_KV && k < keys ? __ldg(tb + (k >> a.page_shift)) : -1;
      };
      int page = page_of(sg.c.j);
      if (!is_v) {
        if (!mbar_wait_warp(&bar[Q_EMPTY], (nseg & 1) ^ 1u, a.err)) { ok = false; break; }
        if (lane == 0) {
          mbar_arrive_expect_tx(&bar[Q_FULL], DH / 64 * 128u * (uint32_t)(rows_per_tile * G));
#pragma unroll
          for (int bx = 0; bx < DH / 64; ++bx)
            tma_load_3d(sm + C::OFF_Q + bx * C::BOX, &tmQ, &bar[Q_FULL], bx * 64, sg.c.kvh * G,
                        plan.row0[sg.c.e] + sg.c.rt * rows_per_tile);
        }
      }
      ++nseg;
      for (int j = sg.c.j; j < sg.c.j + sg.n; ++j, ++g) {
        const int k0 = j * TC_KV, here = min(TC_KV, keys - k0);
        const bool mine = lane * brows < here;  // a box of this lane's is wanted
        const bool good = mine && page >= 0 && page < a.n_pages;
        if (mine && !good) set_error(a.err, SP_DEVERR_INDEX);
        const unsigned int boxes = __ballot_sync(0xffffffffu, good);
        const bool bad = __any_sync(0xffffffffu, mine && !good);
        const int row = (page << a.page_shift) + ((k0 + lane * brows) & ((1 << a.page_shift) - 1));
        const uint32_t bytes = (uint32_t)__popc(boxes) * (uint32_t)brows * (DH * 2);
        page = j + 1 < sg.c.j + sg.n ? page_of(j + 1) : -1;
        // clears rows r0 .. r1 - 1 of a tile
        auto clear = [&](uint8_t* s, int r0, int r1) {
          for (int i = lane; i < (r1 - r0) * 8 * (DH / 64); i += 32) {
            const int bx = i / ((r1 - r0) * 8), k = i - bx * ((r1 - r0) * 8);
            *reinterpret_cast<uint4*>(s + bx * C::BOX + r0 * 128 + k * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        };
        auto clear_bad = [&](uint8_t* s) {  // a page outside the pool: its keys and values are zeros
          for (int b = 0; b * brows < here; ++b)
            if (!((boxes >> b) & 1)) clear(s, b * brows, (b + 1) * brows);
        };
        const uint32_t sb = g % NSB;
        if (!is_v) {
          uint8_t* s = sm + C::OFF_K + (g % NKS) * C::TILE;
          uint64_t* full = &bar[K_FULL + sb];
          // the slot last held tile g - 2: free once its scores are done
          if (g >= NKS && !mbar_wait_warp(&bar[S_FULL + (g - NKS) % NSB], ((g - NKS) / NSB) & 1, a.err)) { ok = false; break; }
          if (bad) {
            clear_bad(s);
            fence_proxy_async_smem();
            __syncwarp();
          }
          if (lane == 0) {
            mbar_arrive_expect_tx(full, bytes);
            if (g < NSB) mbar_arrive(full);  // (no product three tiles before)
          }
          __syncwarp();
          if (good) {
#pragma unroll
            for (int bx = 0; bx < DH / 64; ++bx)
              tma_load_2d(s + bx * C::BOX + lane * brows * 128, &tmK, full, sg.c.kvh * DH + bx * 64, row);
          }
        } else {
          uint8_t* s = sm + C::OFF_V + (g % NVS) * C::TILE;
          uint64_t* full = &bar[P_FULL + sb];
          // the slot last held tile g - 3: free once its product is done
          if (g >= NVS && !mbar_wait_warp(&bar[PV_DONE + (g - NVS) % NSB], ((g - NVS) / NSB) & 1, a.err)) { ok = false; break; }
          const bool tail = here < TC_KV || bad;
          uint64_t* land = tail ? &bar[V_TAIL] : full;
          if (lane == 0) mbar_arrive_expect_tx(land, bytes);
          __syncwarp();
          if (good) {
#pragma unroll
            for (int bx = 0; bx < DH / 64; ++bx)
              tma_load_2d(s + bx * C::BOX + lane * brows * 128, &tmV, land, sg.c.kvh * DH + bx * 64, row);
          }
          if (tail) {
            if (!mbar_wait_warp(land, tails & 1, a.err)) { ok = false; break; }
            ++tails;
            if (bad) clear_bad(s);
            if (here < TC_KV) clear(s, here, TC_KV);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(full);
          }
        }
      }
      if (ok) more = sg.next(plan, p, a.Hkv);
    }
    // every copy lands before the CTA may exit (bounded waits; normally the consumers have waited for them)
    if (!is_v && nseg > 0) mbar_wait_warp(&bar[Q_FULL], (nseg - 1) & 1, a.err);
    for (uint32_t gg = g >= NSB ? g - NSB : 0; gg < g; ++gg)
      mbar_wait_warp(&bar[(is_v ? P_FULL : K_FULL) + gg % NSB], (gg / NSB) & 1, a.err);
  } else if (warp == 1 || warp == 2) {
    // ------------------------------------------------------------ issuers: scores (warp 1), products (warp 2)
    if (lane == 0) {
      const bool pv_issuer = warp == 2;
      constexpr uint32_t IDESC_S = umma_idesc_bf16_f32(128, TC_KV);
      constexpr uint32_t IDESC_O = umma_idesc_bf16_f32(128, DH) | (1u << 16);  // V: MN-major
      const uint64_t dQ = umma_desc_sw128(smem_u32(sm + C::OFF_Q));
      const uint64_t dK = umma_desc_sw128(smem_u32(sm + C::OFF_K));
      const uint64_t dV = umma_desc_sw128_mn(smem_u32(sm + C::OFF_V), C::BOX);
      const uint64_t slot16 = C::TILE >> 4;
      while (ok && more) {
        if (!pv_issuer) {
          ok = mbar_wait(&bar[Q_FULL], nseg & 1, a.err);
          for (int j = 0; ok && j < sg.n; ++j) {
            const uint32_t gg = g + j, sb = gg % NSB;
            if (!mbar_wait(&bar[K_FULL + sb], (gg / NSB) & 1, a.err)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk)
              umma_bf16(tmem + sb * TC_KV, dQ + (((kk >> 2) * C::BOX + (kk & 3) * 32) >> 4),
                        dK + (gg % NKS) * slot16 + (((kk >> 2) * C::BOX + (kk & 3) * 32) >> 4), IDESC_S, kk ? 1u : 0u);
            umma_commit(&bar[S_FULL + sb]);
            if (j + 1 == sg.n) umma_commit(&bar[Q_EMPTY]);
          }
        } else {
          for (int j = 0; ok && j < sg.n; ++j) {
            const uint32_t gg = g + j, sb = gg % NSB;
            if (!mbar_wait(&bar[P_FULL + sb], (gg / NSB) & 1, a.err) ||
                (j == 0 && !mbar_wait(&bar[O_EMPTY], (nseg & 1) ^ 1u, a.err))) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint64_t dVs = dV + (gg % NVS) * slot16;
#pragma unroll
            for (int kk = 0; kk < TC_KV / 16; ++kk)
              umma_bf16_ta(tmem + C::T_O, tmem + sb * TC_KV + kk * 8, dVs + ((kk * 2048) >> 4), IDESC_O,
                           (j | kk) ? 1u : 0u);
            umma_commit(&bar[PV_DONE + sb]);
            umma_commit(&bar[K_FULL + sb]);  // (counts toward the K barrier of tile gg + 3)
            if (j + 1 == sg.n) umma_commit(&bar[O_FULL]);
          }
        }
        g += sg.n;
        ++nseg;
        more = sg.next(plan, p, a.Hkv);
      }
      // tensor memory stays allocated until every product this thread issued is done
      umma_commit(&bar[MMA_DONE + (pv_issuer ? 1 : 0)]);
      mbar_wait(&bar[MMA_DONE + (pv_issuer ? 1 : 0)], 0, a.err);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax streams (vector = lane of tensor memory)
    const uint32_t s = (uint32_t)(warp - 4) >> 2;
    const int r0 = (warp & 3) * 32, r = r0 + lane;
    const uint32_t trow = tmem + ((uint32_t)r0 << 16);
    write_rows(a, p, plan, threadIdx.x - 128, TC_NT - 128);
    float* mchain = reinterpret_cast<float*>(sm + C::OFF_M);
    float* lsum = reinterpret_cast<float*>(sm + C::OFF_L);
    while (ok && more) {
      const int M = plan.rows[sg.c.e] * G, keys = plan.keys[sg.c.e], m0 = sg.c.rt * p.tile_rows;
      const int rows = min(p.tile_rows, M - m0);  // vectors of the tile
      // keys [0, row_lim) are visible; a lane without a vector masks nothing (its results go nowhere, and the one
      // masked lane would cost its warp the masking of every tile)
      int row_lim = 0x7fffffff;
      if (r < rows)
        row_lim = sg.c.e < a.n_groups ? keys : min(max(keys - plan.rows[sg.c.e] + (m0 + r) / G + 1, 0), keys);
      float mlast = -INFINITY;             // m of this stream's latest tile
      float ms = -INFINITY, ls = 0.f;      // this stream's sum, relative to 2^ms
      for (int j = (int)((g & 1) != s); j < sg.n; j += 2) {
        const uint32_t gg = g + j, sb = gg % NSB;
        if (!mbar_wait_warp(&bar[S_FULL + sb], (gg / NSB) & 1, a.err)) { ok = false; break; }
        tc_fence_after();
        float v[TC_KV];
#pragma unroll
        for (int c = 0; c < TC_KV / 32; ++c)
          tmem_ld_32x32b_x32(trow + sb * TC_KV + c * 32, *reinterpret_cast<float(*)[32]>(v + c * 32));
        tmem_ld_wait();
        loaded(v);
        const int lim = row_lim - (sg.c.j + j) * TC_KV;
        if (lim < TC_KV) {
#pragma unroll
          for (int c = 0; c < TC_KV; ++c) v[c] = c < lim ? v[c] : -INFINITY;
        }
        float mx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = max3(v[e], v[e + 8], v[e + 16]);
#pragma unroll
        for (int c = 24; c + 16 <= TC_KV; c += 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) mx[e] = max3(mx[e], v[c + e], v[c + 8 + e]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(mx[e], v[TC_KV - 8 + e]);
        const float mh = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
        // m of the segment's tile before (the other stream's), then this tile's
        float mp = -INFINITY;
        if (j > 0) {
          const uint32_t pb = gg - 1;
          if (!mbar_wait_warp(&bar[M_FULL + (pb & 1)], (pb >> 1) & 1, a.err)) { ok = false; break; }
          mp = mchain[(pb & 1) * 128 + r];
        }
        const float mb = mh * a.scale_log2;
        float m = mp, corr = 1.f;
        bool moved = false;
        if (mb > mp + kRescaleLog2 || (mp == -INFINITY && mb > -INFINITY)) {
          corr = mp == -INFINITY ? 0.f : ex2(mp - mb);
          moved = mp != -INFINITY;
          m = mb;
        }
        mchain[(gg & 1) * 128 + r] = m;
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[M_FULL + (gg & 1)]);
        mlast = m;
        if (m != ms) {  // bring this stream's sum to the new reference (from -infinity: zero, or NaN, which stays)
          ls *= ex2(ms == -INFINITY ? 0.f : ms - m);
          ms = m;
        }
        const float nm = m == -INFINITY ? 0.f : -m;
        const unsigned long long sc2 = pack2(a.scale_log2, a.scale_log2), nm2 = pack2(nm, nm);
        unsigned long long rs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) rs[e] = 0ull;
#pragma unroll
        for (int c = 0; c < TC_KV / 32; ++c) {
          float pk[16];  // bf16 pairs
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float x0, x1;
            unpack2(fma2(pack2(v[c * 32 + 2 * e], v[c * 32 + 2 * e + 1]), sc2, nm2), x0, x1);
            const float p0 = ex2(x0), p1 = ex2(x1);
            rs[e & 3] = add2(rs[e & 3], pack2(p0, p1));
            pk[e] = __uint_as_float(pack_bf16x2(p0, p1));
          }
          tmem_st_cols<16>(trow + sb * TC_KV + c * 16, pk);
        }
        float sum0, sum1;
        unpack2(add2(add2(rs[0], rs[1]), add2(rs[2], rs[3])), sum0, sum1);
        ls += sum0 + sum1;
        if (__any_sync(0xffffffffu, moved)) {
          // the product of the tile before is done with O before it is rescaled
          const uint32_t pb = gg - 1;
          if (!mbar_wait_warp(&bar[PV_DONE + pb % NSB], (pb / NSB) & 1, a.err)) { ok = false; break; }
          tc_fence_after();
          float o[32];
#pragma unroll 1
          for (int c = 0; c < DH; c += 32) {
            tmem_ld_32x32b_x32(trow + C::T_O + c, o);
            tmem_ld_wait();
            loaded(o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= corr;
            tmem_st_32x32b_x32(trow + C::T_O + c, o);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar[P_FULL + sb]);
      }
      if (!ok) break;
      // ---- the segment's (max, sum): the two streams' sums at the last tile's m
      const uint32_t last = g + sg.n - 1;
      if ((last & 1) != s) {
        if (!mbar_wait_warp(&bar[M_FULL + (last & 1)], (last >> 1) & 1, a.err)) { ok = false; break; }
        mlast = mchain[(last & 1) * 128 + r];
      }
      // (scores that are all NaN leave m at -infinity: their sum is passed on)
      const float lsc = (ms == -INFINITY || mlast == -INFINITY) ? ls : ls * ex2(ms - mlast);
      float* xl = lsum + (nseg & 1) * 256;
      xl[s * 128 + r] = lsc;
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[XL]);
      if (!mbar_wait_warp(&bar[XL], nseg & 1, a.err)) { ok = false; break; }
      const size_t at = ((size_t)sg.c.item + w) * p.slot_rows;
      if (s == 0 && r < rows) p.part_ml[at + r] = make_float2(mlast, xl[r] + xl[128 + r]);
      // ---- and O, this stream's half of its columns
      if (!mbar_wait_warp(&bar[O_FULL], nseg & 1, a.err)) { ok = false; break; }
      tc_fence_after();
      constexpr int HD = DH / 2;
      float o[HD];
#pragma unroll
      for (int c = 0; c < HD; c += 32)
        tmem_ld_32x32b_x32(trow + C::T_O + s * HD + c, *reinterpret_cast<float(*)[32]>(o + c));
      tmem_ld_wait();
      loaded(o);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bar[O_EMPTY]);  // O may be overwritten from here
      // stage: row `lane` of this warp, 16 columns (64 bytes) at a time; 16-byte granule q of a row sits at
      // q ^ ((row >> 1) & 3) (no bank conflicts)
      uint8_t* stg = sm + C::OFF_STG + (warp - 4) * 2048;
      float* dst = p.part_o + (at + r0) * DH + s * HD;
#pragma unroll
      for (int c = 0; c < HD; c += 16) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<float4*>(stg + lane * 64 + ((q ^ ((lane >> 1) & 3)) * 16)) =
              make_float4(o[c + 4 * q], o[c + 4 * q + 1], o[c + 4 * q + 2], o[c + 4 * q + 3]);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int row = k * 8 + (lane >> 2), q = lane & 3;
          const float4 x = *reinterpret_cast<const float4*>(stg + row * 64 + ((q ^ ((row >> 1) & 3)) * 16));
          if (r0 + row < rows) *reinterpret_cast<float4*>(dst + (size_t)row * DH + c + q * 4) = x;
        }
        __syncwarp();
      }
      g += sg.n;
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
  static std::atomic<unsigned long long> allowed;
  const cudaError_t r = allow_smem(prefix_tc_kernel<DH>, C::SMEM, allowed);
  if (r != cudaSuccess) return r;
  return launch_pdl(prefix_tc_kernel<DH>, dim3(p.workers), dim3(TC_NT), C::SMEM, st, tq, tk, tv, a, p);
}

}  // namespace

cudaError_t prefix_tc_launch(const PrefixArgs& a, const PlanArgs& p, int dh, cudaStream_t st) {
  return dh == 128 ? launch_tc<128>(a, p, st) : launch_tc<64>(a, p, st);
}

}  // namespace sp
