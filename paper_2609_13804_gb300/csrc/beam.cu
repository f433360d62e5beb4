// Beam search over the sequences of an element: the best continuations of its beams, and the beams' cache
// put into their order.
//
// Selection.  The score of token v after beam w is cum_w + log softmax(x_w)_v = cum_w + x_v - m - log sum exp(x - m).
// Within a beam the order is that of the logits, so one pass over a row finds its m, its sum and its n_out
// largest logits together; which beams they came from matters only for the n_out best of each row, whose
// scores are formed and compared in 64 bits (two beams' scores can be nearer than fp32 tells apart).  Equal
// ones: the lower beam, then the lower token.  Equal rows have equal scores, to the bit: their logits are added in the same
// order, by pieces of 16 bytes.  Where the rows of a call begin at different places within 16 bytes these are pieces of
// the row, each put together from two aligned loads, else the aligned pieces.
#include <algorithm>

#include "common.cuh"
#include "internal.h"
#include "logits.cuh"

namespace sp {

namespace {

constexpr int BS_NT = 256, BS_WARPS = BS_NT / 32, BS_MAX_OUT = 2 * SP_MAX_BEAMS;
constexpr int BS_LOADS = 4;                 // 16-byte loads per thread and tile
constexpr int BS_RING = 3;                  // tiles in flight
constexpr int BS_BLOCK = 16;                // tiles of a block
constexpr int BS_CAP = 128;                 // candidates a warp keeps at most
constexpr int BS_LIST = 256;                // slices x n_out of a row, at most (shared memory of the join)

// A logit and its token as one key that sorts by (logit, lower token first); 0: none.
SP_DEVINL unsigned long long cand_key(float x, int v) {
  const uint32_t u = __float_as_uint(x + 0.f);  // (-0 is 0)
  const uint32_t s = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return ((unsigned long long)s << 32) | (uint32_t)~v;
}
SP_DEVINL float key_logit(unsigned long long k) {
  const uint32_t s = (uint32_t)(k >> 32);
  return __uint_as_float((s & 0x80000000u) ? (s & 0x7fffffffu) : ~s);
}
SP_DEVINL int key_token(unsigned long long k) { return (int)~(uint32_t)k; }

// 16 bytes that begin WORD words and `bits` bits into a, and go on in b
template <bool F32, int WORD>
SP_DEVINL uint4 piece_at(const uint4& a, const uint4& b, uint32_t bits) {
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (F32) return make_uint4(w[WORD], w[WORD + 1], w[WORD + 2], w[WORD + 3]);
  return make_uint4(__funnelshift_r(w[WORD], w[WORD + 1], bits), __funnelshift_r(w[WORD + 1], w[WORD + 2], bits),
                    __funnelshift_r(w[WORD + 2], w[WORD + 3], bits), __funnelshift_r(w[WORD + 3], w[WORD + 4], bits));
}

// The n_out largest of a warp's list of n (at most BS_CAP) to its front, in order, by counting the larger ones
// of each; returns how many there are.  (A function of its own: its registers are not the scan's.)
__device__ __noinline__ int cut_list(unsigned long long* list, int n, int n_out) {
  const int lane = threadIdx.x & 31;
  unsigned long long mine[BS_CAP / 32];
  int rank[BS_CAP / 32];
#pragma unroll
  for (int q = 0; q < BS_CAP / 32; ++q) {
    const int i = q * 32 + lane;
    mine[q] = i < n ? list[i] : 0ull;
    rank[q] = 0;
  }
  for (int i = 0; i < n; ++i) {
    const unsigned long long u = list[i];
#pragma unroll
    for (int q = 0; q < BS_CAP / 32; ++q)
      if (q * 32 < n) rank[q] += u > mine[q];
  }
  __syncwarp();
#pragma unroll
  for (int q = 0; q < BS_CAP / 32; ++q)
    if (mine[q] != 0 && rank[q] < n_out) list[rank[q]] = mine[q];
  __syncwarp();
  return min(n, n_out);
}

// One CTA: a slice of one row.  The slice goes by in blocks of tiles (a tile: 4 loads of every thread).  First a
// block's share of (m, sum), every thread noting the maximum of each of its tiles; nothing is selected on the way,
// which would cost more than the sums.  Then a bound T below which n_out of the slice are known not to lie: the
// least, over the warps, of the ceil(n_out / warps)-th largest thread maximum of the block (n_out threads hold
// something at or above it, and only about 2.7 n_out logits of the block lie there).  Then the few threads whose
// tiles reach T load those again (from L2) and put what lies above T into their warp's list.  A list that could
// overflow is cut down to its n_out largest and T raised to the last of them, so any order of logits, and any
// number of equal ones (keys tell them apart by token), is taken exactly.  At the end the lists' n_out largest,
// in order, and (m, sum) go to part.
// Bound by issue (some 6 instructions a logit with the exponential's) and by what a slice costs besides, about 3 us:
// 256 rows of 152,064 bf16 logits, a fifth of them finished, 62 MB, 18 us (3.4 TB/s); 4 rows of 32,000 fp32 3.5 us.
// SHIFT: the rows begin at different places within 16 bytes.  The aligned pieces go through the ring as they lie; a
// lane puts each of its pieces from its own and the next lane's (the warp's last from a piece loaded beside).  Both
// kernels, 64 x 4 rows of 152,063 bf16 logits 27.5 us (23.1 by aligned pieces, which tie by where a row lies), 16 x 4 of
// 50,257 fp32 13.7 (12.2): some 30 instructions more for the 32 or 16 logits of a thread and tile.
template <bool F32, bool SHIFT>
__global__ void __launch_bounds__(BS_NT, SHIFT ? 2 : 3)
beam_scan_kernel(const void* __restrict__ logits, long long ld, int V, const float* __restrict__ cum,
                 const unsigned char* __restrict__ done, int n_out, int slice, float2* __restrict__ part_ms,
                 unsigned long long* __restrict__ part_key) {
  using K = Chunk<F32>;
  __shared__ unsigned long long list_s[BS_WARPS][BS_CAP];
  __shared__ unsigned long long list_all[BS_WARPS * 32];
  extern __shared__ uint4 ring[];  // [BS_RING][BS_LOADS][BS_NT]: a thread's own loads (SHIFT: read by the lane before too)
  uint4* beside = ring + BS_RING * BS_LOADS * BS_NT;  // SHIFT: [BS_RING][BS_WARPS][BS_LOADS] behind each warp's loads
  __shared__ float2 ms_s[BS_WARPS];
  __shared__ float tile_max[BS_BLOCK][BS_NT];
  __shared__ uint32_t bound_s[2][BS_WARPS];
  __shared__ int events[BS_WARPS][64];
  __shared__ int n_s[BS_WARPS];
  pdl_wait();
  const int row = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float cw = __ldg(cum + row);
  const bool over = done && __ldg(done + row);
  constexpr int esz = F32 ? 4 : 2, PER = BS_LOADS * K::N;  // logits per thread and tile: one to a lane at most
  static_assert(PER <= 32, "");
  const char* base = static_cast<const char*>(logits) + row * ld * esz;
  const int v0 = min(blockIdx.x * slice, V), v1 = min(v0 + slice, V);
  // whole 16-byte chunks of the slice; what is before and behind them goes one by one
  const uint32_t off = reinterpret_cast<uintptr_t>(base + (size_t)v0 * esz) & 15;  // (the same for all slices of a row)
  const int head = SHIFT ? 0 : min((int)((16 - off) & 15) / esz, v1 - v0);
  const int c0 = v0 + head, chunks = (v1 - c0) / K::N, c1 = c0 + chunks * K::N;
  unsigned long long* list = list_s[warp];
  int n = 0;
  MaxSum ms{-INFINITY, 0.f};
  if (warp == 0) {
    const bool in = lane < head + (v1 - c1);  // (fewer than 16)
    const int v = lane < head ? v0 + lane : c1 + lane - head;
    const float x = in ? K::one(base, v) : -INFINITY;
    const bool some = x > -INFINITY;  // (NaN and -infinity are no candidates and have no weight)
    const unsigned int all = __ballot_sync(0xffffffffu, some);
    if (some) {
      ms.m = x;
      ms.s = 1.f;
      list[__popc(all & ((1u << lane) - 1u))] = cand_key(x, v);
    }
    n = __popc(all);
  }
  const uint4* src = reinterpret_cast<const uint4*>(base + (size_t)c0 * esz - (SHIFT ? off : 0));
  unsigned long long T = 0;  // keys above T are candidates
  const int tile_chunks = BS_NT * BS_LOADS, tiles = (chunks + tile_chunks - 1) / tile_chunks;
  auto copy16 = [&](uint4* to, int c) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(src + c) : "memory");
  };
  // SHIFT: aligned piece c, as far as it holds the slice's chunks (0 .. chunks - 1 begin in it, the last ends in the next).
  // What lies before the first row may be no one's: its first piece is put there by elements.
  const bool first = SHIFT && row == 0 && v0 == 0 && off != 0;
  auto part = [&](uint4* to, int c) {
    if (first && c == 0 && chunks > 0) {
      for (int k = off / esz; k < K::N; ++k) {
        if (F32) reinterpret_cast<float*>(to)[k] = reinterpret_cast<const float*>(base)[k - off / esz];
        else reinterpret_cast<__nv_bfloat16*>(to)[k] = reinterpret_cast<const __nv_bfloat16*>(base)[k - off / esz];
      }
    } else if (c < chunks) {
      copy16(to, c);
    } else if (c == chunks && c > 0 && off != 0) {
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(src + c), "r"(off) : "memory");
    }
  };
  auto load = [&](int t) {  // (what lies past the slice is not loaded, and read as -infinity)
    uint4* to = ring + (t % BS_RING) * (BS_LOADS * BS_NT) + tid;
    const int c = t * tile_chunks + tid;
    if (!SHIFT) {
#pragma unroll
      for (int q = 0; q < BS_LOADS; ++q)
        if (c + q * BS_NT < chunks) copy16(to + q * BS_NT, c + q * BS_NT);
    } else if (t < tiles) {
      uint4* last = beside + ((t % BS_RING) * BS_WARPS + warp) * BS_LOADS + lane;
      const int c_last = t * tile_chunks + lane * BS_NT + (warp + 1) * 32;
      if ((t + 1) * tile_chunks < chunks && !(first && t == 0)) {  // (whole pieces, the one behind the tile too)
#pragma unroll
        for (int q = 0; q < BS_LOADS; ++q) copy16(to + q * BS_NT, c + q * BS_NT);
        if (off != 0 && lane < BS_LOADS) copy16(last, c_last);
      } else {
#pragma unroll 1
        for (int q = 0; q < BS_LOADS; ++q) part(to + q * BS_NT, c + q * BS_NT);
        if (off != 0 && lane < BS_LOADS) part(last, c_last);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float bm = -INFINITY;  // the thread's maximum of the block
  auto take = [&](const uint4 (&u)[BS_LOADS], int place) {
    float lm = -INFINITY;
#pragma unroll
    for (int q = 0; q < BS_LOADS; ++q) lm = fmaxf(lm, K::top(u[q]));
    tile_max[place][tid] = lm;
    bm = fmaxf(bm, lm);
    if (lm == -INFINITY) return;
    if (lm > ms.m) {
      ms.s = ms.m == -INFINITY ? 0.f : ms.s * ex2((ms.m - lm) * kLog2e);
      ms.m = lm;
    }
    // (x - m first, exactly where it matters, then log2 e: m log2 e rounded would shift the whole sum)
    const unsigned long long nm = pack2(-ms.m, -ms.m), l2 = pack2(kLog2e, kLog2e);
    unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
    for (int q = 0; q < BS_LOADS; ++q)
#pragma unroll
      for (int k = 0; k < K::N; k += 2) {
        float a, b;
        unpack2(mul2(add2(pack2(K::at(u[q], k), K::at(u[q], k + 1)), nm), l2), a, b);
        sum[(k >> 1) & 1] = add2(sum[(k >> 1) & 1], pack2(ex2(a), ex2(b)));
      }
    float sa, sb;
    unpack2(add2(sum[0], sum[1]), sa, sb);
    float ts = sa + sb;
    if (ts != ts) {  // a NaN, or infinity less infinity, among them
      ts = 0.f;
      for (int i = 0; i < PER; ++i) {
        float x = 0.f;
#pragma unroll
        for (int q = 0; q < BS_LOADS; ++q)
#pragma unroll
          for (int k = 0; k < K::N; ++k)
            if (i == q * K::N + k) x = K::at(u[q], k);
        if (x == ms.m) ts += 1.f;
        else if (x < ms.m) ts += ex2((x - ms.m) * kLog2e);
      }
    }
    ms.s += ts;
  };
#pragma unroll
  for (int t = 0; t < BS_RING - 1; ++t) load(t);
  // (The join reads nothing of such a beam's row.  Told before the first loads, it would cost the others the wait for
  // done and cum: four rows of 32,000 fp32 logits 7.9 us instead of 7.7.)
  if (over || !(cw > -INFINITY)) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  for (int tb = 0, block = 0; tb < tiles; tb += BS_BLOCK, ++block) {
    const int te = min(tb + BS_BLOCK, tiles);
    bm = -INFINITY;
    for (int t = tb; t < te; ++t) {
      if (SHIFT) __syncwarp();  // the tile that is overwritten has been read by the lanes before
      load(t + BS_RING - 1);
      asm volatile("cp.async.wait_group %0;" ::"n"(BS_RING - 1) : "memory");
      const uint4* from = ring + (t % BS_RING) * (BS_LOADS * BS_NT) + tid;
      uint4 u[BS_LOADS];
#pragma unroll
      for (int q = 0; q < BS_LOADS; ++q) u[q] = from[q * BS_NT];
      if (SHIFT && off != 0) {
        __syncwarp();  // the next lane's loads have landed
        const uint4* next = lane < 31 ? from + 1 : beside + ((t % BS_RING) * BS_WARPS + warp) * BS_LOADS;
        const int step = lane < 31 ? BS_NT : 1;
        const uint32_t bits = (off & 2) * 8;
        uint4 b[BS_LOADS];
#pragma unroll
        for (int q = 0; q < BS_LOADS; ++q) b[q] = next[q * step];
#pragma unroll
        for (int q = 0; q < BS_LOADS; ++q) {
          if (off < 4) u[q] = piece_at<F32, 0>(u[q], b[q], bits);  // (off is the CTA's)
          else if (off < 8) u[q] = piece_at<F32, 1>(u[q], b[q], bits);
          else if (off < 12) u[q] = piece_at<F32, 2>(u[q], b[q], bits);
          else u[q] = piece_at<F32, 3>(u[q], b[q], bits);
        }
      }
      if (t == tiles - 1) {
#pragma unroll
        for (int q = 0; q < BS_LOADS; ++q)
          if (t * tile_chunks + q * BS_NT + tid >= chunks) u[q] = make_uint4(K::kNone, K::kNone, K::kNone, K::kNone);
      }
      take(u, t - tb);
    }
    // the block's bound
    uint32_t rest = bm > -INFINITY ? (uint32_t)(cand_key(bm, 0) >> 32) : 0u, hi = 0;
    for (int r = 0; r < n_out; r += BS_WARPS) {
      hi = __reduce_max_sync(0xffffffffu, rest);
      if (lane == __ffs(__ballot_sync(0xffffffffu, rest == hi)) - 1) rest = 0;
    }
    if (lane == 0) bound_s[block & 1][warp] = hi;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < BS_WARPS; ++w) hi = min(hi, bound_s[block & 1][w]);
    if (hi != 0 && ((unsigned long long)hi << 32) - 1 > T) T = ((unsigned long long)hi << 32) - 1;
    float Tf = T == 0 ? -INFINITY : key_logit(T);  // (a little below T: keys decide)
    unsigned int who = __ballot_sync(0xffffffffu, bm >= Tf && bm > -INFINITY);
    int* ev = events[warp];
    while (who) {
      // tiles of threads of the warp that reach T, 64 at most at a time
      int ne = 0;
      for (; who && ne <= 64 - BS_BLOCK; who &= who - 1) {
        const int other = __ffs(who) - 1;
        const bool reach = lane < te - tb && tile_max[lane & (BS_BLOCK - 1)][(warp << 5) + other] >= Tf;
        const unsigned int all = __ballot_sync(0xffffffffu, reach);
        if (reach) ev[ne + __popc(all & ((1u << lane) - 1u))] = (lane << 5) + other;
        ne += __popc(all);
      }
      __syncwarp();
      for (int e0 = 0; e0 < ne; e0 += 4) {  // each tile's logits, one to a lane; four tiles' loads at once
        float x[4];
        int v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int code = ev[min(e0 + i, ne - 1)];
          const int q = lane / K::N, c = (tb + (code >> 5)) * tile_chunks + q * BS_NT + (warp << 5) + (code & 31);
          v[i] = c0 + c * K::N + lane % K::N;
          x[i] = e0 + i < ne && q < BS_LOADS && c < chunks ? K::one(base, v[i]) : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned long long key = cand_key(x[i], v[i]);
          const bool in = x[i] > -INFINITY && key > T;
          const unsigned int all = __ballot_sync(0xffffffffu, in);
          if (in) list[n + __popc(all & ((1u << lane) - 1u))] = key;
          n += __popc(all);
          __syncwarp();
          if (n > BS_CAP - 32) {
            n = cut_list(list, n, n_out);
            if (list[n_out - 1] - 1 > T) T = list[n_out - 1] - 1;
            Tf = key_logit(T);
          }
        }
      }
      __syncwarp();
    }
  }
  pdl_trigger();  // (not before: CTAs of the join would sit on the SMs that slices still need)
  const float mw = warp_max(ms.m);
  const float sw = warp_sum(ms.m == mw ? ms.s : ms.m > -INFINITY ? ms.s * ex2((ms.m - mw) * kLog2e) : 0.f);
  if (n > 32) n = cut_list(list, n, n_out);
  if (lane == 0) {
    ms_s[warp] = make_float2(mw, sw);
    n_s[warp] = n;
  }
  __syncthreads();
  // the warps' candidates side by side, then every one's place: how many are larger
  const size_t at = (size_t)row * gridDim.x + blockIdx.x;
  int total = 0, before = 0;
#pragma unroll
  for (int w = 0; w < BS_WARPS; ++w) {
    const int nw = n_s[w];
    before += w < warp ? nw : 0;
    total += nw;
  }
  unsigned long long* all = &list_all[0];
  if (lane < n) all[before + lane] = list[lane];
  __syncthreads();
  if (tid < total) {
    const unsigned long long k = all[tid];
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < total; ++i) rank += all[i] > k;
    if (rank < n_out) part_key[at * n_out + rank] = k;
  }
  if (tid < n_out && tid >= total) part_key[at * n_out + tid] = 0ull;
  if (tid == 0) {
    ms = MaxSum{ms_s[0].x, ms_s[0].y};
    for (int w = 1; w < BS_WARPS; ++w) ms.add(ms_s[w].x, ms_s[w].y);
    part_ms[at] = make_float2(ms.m, ms.s);
  }
}

// Up to this many scores of an element are all compared with one another; of more, those that can be among the best
// (16 beams of 32 answers each: 15.6 us of both kernels instead of 29.4; 8 of 16: 12.0 instead of 12.4; for fewer the
// two barriers cost what they save).
constexpr int BJ_ALL = 64;

// The bits of a double so that they sort as it does.
SP_DEVINL unsigned long long order_bits(double v) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(v + 0.0);
  return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

// The largest of the lanes' values.
SP_DEVINL unsigned long long warp_max64(unsigned long long v) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return ((unsigned long long)hi << 32) | lo;
}

// One CTA per element, a warp per beam: the n_out best of the beam's lists, their scores in 64 bits, then the n_out
// best over the beams.  Comparisons are of integers (the 64-bit floating-point pipe is slow here).  log(sum) is e log 2 + log f with
// sum = 2^e f: exact in e, and log f, below 0.7, is good to 2^-24 in fp32, as are the sums that go into it.
__global__ void __launch_bounds__(32 * SP_MAX_BEAMS)
beam_join_kernel(int W, int S, const float* __restrict__ cum, const unsigned char* __restrict__ done, int eos, int n_out,
                 const float2* __restrict__ part_ms, const unsigned long long* __restrict__ part_key,
                 float* __restrict__ score, int* __restrict__ parent, int* __restrict__ token) {
  extern __shared__ unsigned long long rows_s[];  // [W][S n_out] the beams' lists
  __shared__ unsigned long long sc_s[SP_MAX_BEAMS * BS_MAX_OUT];  // order_bits of the score, 0: none
  __shared__ float val_s[SP_MAX_BEAMS * BS_MAX_OUT];
  __shared__ int tk_s[SP_MAX_BEAMS * BS_MAX_OUT];
  __shared__ unsigned long long left_s[SP_MAX_BEAMS * BS_MAX_OUT];
  __shared__ int from_s[SP_MAX_BEAMS * BS_MAX_OUT];
  __shared__ int in_s[SP_MAX_BEAMS];
  pdl_wait();
  pdl_trigger();
  const int e = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = e * W + warp, n = S * n_out;
  // (a beam that was not scanned has nothing there: what is loaded for it is not used)
  unsigned long long* keys = rows_s + (size_t)warp * n;
  const float cw = __ldg(cum + row);
  const bool over = done && __ldg(done + row);
  const float2 ms = lane < S ? __ldcg(part_ms + (size_t)row * S + lane) : make_float2(-INFINITY, 0.f);
  for (int i = lane; i < n; i += 32) keys[i] = __ldcg(part_key + (size_t)row * n + i);
  __syncwarp();
  unsigned long long sc = 0;
  float val = 0.f;
  int tk = 0;
  unsigned long long* best = sc_s + warp * n_out;  // (its scores' place: the keys are read before)
  if (lane < n_out) best[lane] = 0;
  if (!(cw > -INFINITY)) {
  } else if (over) {
    if (lane == 0) {
      sc = order_bits((double)cw);
      val = cw;
      tk = eos;
    }
  } else {
    const float m = warp_max(ms.x);
    const float sum = warp_sum(ms.x == m ? ms.y : ms.x > -INFINITY ? ms.y * ex2((ms.x - m) * kLog2e) : 0.f);
    unsigned long long mine = 0;  // lane r: the r-th best
    if (n <= 64) {  // by counting the larger ones of each: two keys per lane
      const unsigned long long k0 = lane < n ? keys[lane] : 0ull, k1 = lane + 32 < n ? keys[lane + 32] : 0ull;
      int r0 = 0, r1 = 0;
#pragma unroll 8
      for (int i = 0; i < n; ++i) {
        const unsigned long long u = keys[i];
        r0 += u > k0;
        r1 += u > k1;
      }
      __syncwarp();
      if (k0 != 0 && r0 < n_out) best[r0] = k0;
      if (k1 != 0 && r1 < n_out) best[r1] = k1;
      __syncwarp();
      if (lane < n_out) mine = best[lane];
    } else {  // a lane holds a list's next key: the largest, n_out times
      unsigned long long next = lane < S ? keys[lane * n_out] : 0ull;
      int at = 0;
      for (int r = 0; r < n_out; ++r) {
        const unsigned long long most = warp_max64(next);
        if (most == 0) break;
        if (lane == r) mine = most;
        if (next == most) next = ++at < n_out ? keys[lane * n_out + at] : 0ull;  // (no two keys are equal)
      }
    }
    int ex = 0;
    const float f = frexpf(sum, &ex) * 2.f;  // sum = f 2^(ex - 1), f in [1, 2)
    if (mine != 0) {
      const double lsum = (double)(ex - 1) * 0.69314718055994530942 + (double)logf(f);
      const float x = key_logit(mine);
      const double d = x == m ? 0.0 : (double)x - (double)m;  // (m = +infinity: its tokens alone have weight)
      const double v = (double)cw + (d - lsum);
      if (v > -INFINITY) {
        sc = order_bits(v);
        val = (float)v;
        tk = key_token(mine);
      }
    }
  }
  if (lane < n_out) {
    sc_s[warp * n_out + lane] = sc;
    val_s[warp * n_out + lane] = val;
    tk_s[warp * n_out + lane] = tk;
  }
  const int have = __syncthreads_count(sc != 0);
  // over the beams: how many are better; (beam, rank) breaks ties
  const int t = threadIdx.x;
  int total = W * n_out, at = t;  // the scores that are compared, and this thread's
  const unsigned long long* list = sc_s;
  if (total > BJ_ALL) {
    // Not the ones that n_out lie above for certain: n_out scores reach the least of the beams' ceil(n_out / W)-th
    // best, and n_out reach any beam's last.
    const int last = lane < W ? lane : 0;
    const unsigned long long each = ~warp_max64(~sc_s[last * n_out + (n_out - 1) / W]);
    const unsigned long long most = warp_max64(sc_s[last * n_out + n_out - 1]);
    const unsigned long long bound = max(max(each, most), 1ull);
    const unsigned int in = __ballot_sync(0xffffffffu, sc >= bound);
    if (lane == 0) in_s[warp] = __popc(in);
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < W; ++w) {
      before += w < warp ? in_s[w] : 0;
      total += in_s[w];
    }
    if (sc >= bound) {
      const int to = before + __popc(in & ((1u << lane) - 1u));
      left_s[to] = sc;
      from_s[to] = warp * n_out + lane;
    }
    __syncthreads();
    list = left_s;
    at = t < total ? from_s[t] : 0;
  }
  const size_t o = (size_t)e * n_out;
  if (t < total) {
    const unsigned long long s = list[t];
    int rank = 0;
#pragma unroll 8
    for (int i = 0; i < total; ++i) {
      const unsigned long long u = list[i];
      rank += u > s || (u == s && i < t);
    }
    if (s != 0 && rank < n_out) {
      score[o + rank] = val_s[at];
      parent[o + rank] = at / n_out;
      token[o + rank] = tk_s[at];
    }
  }
  if (t < n_out && t >= have) {
    score[o + t] = -INFINITY;
    parent[o + t] = -1;
    token[o + t] = -1;
  }
}

// --------------------------------------------------------------- reordering
// Beam w of an element continues beam p(w).  Full pages are never written again, so beams share them: w's
// table takes p(w)'s entries.  The partly filled page is copied: every beam has a page of its own for each
// place of its table (own_table), the only ones it ever writes, so the rows of own[p(w)] go to own[w], in
// place for all beams at once: a thread reads its 16 bytes of every parent before it writes any.
// blockIdx.y: a plane (layer, K or V), or behind the last the tables.  Bound by the copied rows' bytes (66 MB of 16 x 4
// beams, 28 layers, in 14.2 us, 4.7 TB/s read and written), for few of them by the chain length -> pages -> rows.
constexpr int BR_NT = 256;

template <int WMAX>
__global__ void __launch_bounds__(BR_NT)
beam_reorder_kernel(uint4* __restrict__ kv, int planes, int n_pages, int page_shift, int row16, int* __restrict__ table,
                    const int* __restrict__ own, int max_pages, const int* __restrict__ lens,
                    const int* __restrict__ parent, int ld_parent, int W, int* err) {
  pdl_wait();
  pdl_trigger();
  // every warp looks up the element by itself (lane w: beam w), which takes no barrier
  const int e = blockIdx.z, tid = threadIdx.x, lane = tid & 31, w0 = min(lane, W - 1);
  const int len = __ldg(lens + e * W), mine = __ldg(lens + e * W + w0);
  int par = __ldg(parent + (size_t)e * ld_parent + w0);
  if (par < -1 || par >= W) {
    if (tid == lane) set_error(err, SP_DEVERR_INDEX);
    par = -1;
  }
  if (par < 0) par = w0;
  // all beams of an element are equally long, and within their tables
  if (__any_sync(0xffffffffu, mine != len || len < 0 || len > (max_pages << page_shift))) {
    if (tid == 0) set_error(err, SP_DEVERR_INDEX);
    return;
  }
  const int full = len >> page_shift, rows = len & ((1 << page_shift) - 1);
  if (blockIdx.y == planes) {  // the tables: a column per thread
    for (int c0 = blockIdx.x * BR_NT; c0 < max_pages; c0 += gridDim.x * BR_NT) {
      const int c = c0 + tid;
      int v[WMAX];
#pragma unroll
      for (int w = 0; w < WMAX; ++w) {
        const int q = __shfl_sync(0xffffffffu, par, w);
        if (w < W && c < max_pages)
          v[w] = c < full ? table[(size_t)(e * W + q) * max_pages + c] : __ldg(own + (size_t)(e * W + w) * max_pages + c);
      }
#pragma unroll
      for (int w = 0; w < WMAX; ++w)
        if (w < W && c < max_pages) table[(size_t)(e * W + w) * max_pages + c] = v[w];
    }
    return;
  }
  if (rows == 0) return;
  const int s = __ldg(own + (size_t)(e * W + par) * max_pages + full);
  const int d = __ldg(own + (size_t)(e * W + w0) * max_pages + full);
  const bool ok = s >= 0 && s < n_pages && d >= 0 && d < n_pages;
  if (!ok && tid == lane) set_error(err, SP_DEVERR_INDEX);
  const unsigned int move = __ballot_sync(0xffffffffu, lane < W && ok && s != d);
  uint4* pl = kv + (((size_t)blockIdx.y * n_pages) << page_shift) * row16;
  const uint4* from[WMAX];
  uint4* to[WMAX];
#pragma unroll
  for (int w = 0; w < WMAX; ++w) {
    from[w] = pl + ((size_t)(unsigned)__shfl_sync(0xffffffffu, s, w) << page_shift) * row16;
    to[w] = pl + ((size_t)(unsigned)__shfl_sync(0xffffffffu, d, w) << page_shift) * row16;
  }
  const int n = rows * row16;
  for (int i = blockIdx.x * BR_NT + tid; i < n; i += gridDim.x * BR_NT) {
    uint4 v[WMAX];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (move >> w & 1) v[w] = from[w][i];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (move >> w & 1) to[w][i] = v[w];
  }
}

}  // namespace

// Slices of a row: about two CTAs per SM (what a CTA does besides reading, some 3 us, is not hidden by more: four
// took 25.4 us instead of 23.1 for 256 rows of 152,064 bf16 logits), of at least 4,096 logits each, and no more lists than lanes to join them
// (and keys than BS_LIST).
static int beam_slices(int rows, int V, int n_out) {
  const int want = (device_sm_count() * 2 + rows / 2) / rows;
  return std::max(1, std::min(std::min(want, std::min(32, BS_LIST / n_out)), (V + 4095) / 4096));
}

size_t beam_select_bytes(int rows, int V, int n_out) {
  const size_t n = (size_t)rows * beam_slices(rows, V, n_out);
  return ((n * 8 + 255) & ~size_t(255)) + n * n_out * 8;
}

cudaError_t beam_select_launch(const void* logits, bool f32, long long ld, int B, int W, int V, const float* cum,
                               const unsigned char* done, int eos, int n_out, void* ws, float* score, int* parent,
                               int* token, cudaStream_t st) {
  const int rows = B * W, S = beam_slices(rows, V, n_out);
  const int slice = (((V + S - 1) / S) + 7) & ~7;
  auto* ms = static_cast<float2*>(ws);
  auto* key = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + (((size_t)rows * S * 8 + 255) & ~size_t(255)));
  prof_begin_launch(st);
  // (beams of one element whose rows begin at different places within 16 bytes)
  const bool shift = W > 1 && ld * (f32 ? 4 : 2) % 16 != 0;
  auto* scan = f32 ? (shift ? beam_scan_kernel<true, true> : beam_scan_kernel<true, false>)
                   : (shift ? beam_scan_kernel<false, true> : beam_scan_kernel<false, false>);
  const int ring = (BS_RING * BS_LOADS * BS_NT + (shift ? BS_RING * BS_WARPS * BS_LOADS : 0)) * 16;
  static std::atomic<unsigned long long> allowed[2][2];
  cudaError_t r = allow_smem(scan, ring, allowed[f32][shift]);
  if (r == cudaSuccess)
    r = launch_pdl(scan, dim3(S, rows), dim3(BS_NT), (size_t)ring, st, logits, ld, V, cum, done, n_out, slice, ms, key);
  prof_end_launch(st, SP_K_MISC, 0.0, (double)rows * V * (f32 ? 4 : 2));
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  r = launch_pdl(beam_join_kernel, dim3(B), dim3(W * 32), (size_t)W * S * n_out * 8, st, W, S, cum, done, eos,
                 n_out, (const float2*)ms, (const unsigned long long*)key, score, parent, token);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

cudaError_t beam_reorder_launch(void* kv, int n_layers, int n_pages, int page_shift, int row_bytes, int* table,
                                const int* own, int max_pages, const int* lens, const int* parent, int ld_parent,
                                int B, int W, int* err, cudaStream_t st) {
  const int planes = 2 * n_layers, row16 = row_bytes / 16;
  const int most = ((1 << page_shift) - 1) * row16;  // chunks of a plane's partly filled page, at most
  // (four 16-byte pieces of every beam per thread of a full page: one took 15.6 us instead of 14.2 for 16 x 4 beams of
  // 28 layers)
  const int gx = std::max(1, std::min((most + BR_NT * 4 - 1) / (BR_NT * 4), 16));
  const dim3 grid(gx, planes + 1, B);
  auto* k = W <= 4 ? beam_reorder_kernel<4> : W <= 8 ? beam_reorder_kernel<8> : beam_reorder_kernel<16>;
  prof_begin_launch(st);
  const cudaError_t r = launch_pdl(k, grid, dim3(BR_NT), 0, st, static_cast<uint4*>(kv), planes, n_pages, page_shift,
                                   row16, table, own, max_pages, lens, parent, ld_parent, W, err);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
