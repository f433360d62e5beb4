// Beam search over the sequences of an element: the best continuations of its beams, and the beams' cache
// put into their order.
//
// Selection.  The score of token v after beam w is cum_w + log softmax(x_w)_v = cum_w + x_v - m - log sum exp(x - m).
// Within a beam the order is that of the logits, so one pass over a row finds its m, its sum and its n_out
// largest logits together; which beams they came from matters only for the n_out best of each row, whose
// scores are formed and compared in 64 bits (two beams' scores can be nearer than fp32 tells apart).  Equal
// ones: the lower beam, then the lower token.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sp {

namespace {

constexpr int BS_NT = 256, BS_WARPS = BS_NT / 32, BS_MAX_OUT = 32;
constexpr float kLog2e = 1.44269504088896341f;

SP_DEVINL float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A logit and its token as one key that sorts by (logit, lower token first); 0: none.
SP_DEVINL unsigned long long cand_key(float x, int v) {
  const uint32_t u = __float_as_uint(x);
  const uint32_t s = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
  return ((unsigned long long)s << 32) | (uint32_t)~v;
}
SP_DEVINL float key_logit(unsigned long long k) {
  const uint32_t s = (uint32_t)(k >> 32);
  return __uint_as_float((s & 0x80000000u) ? (s & 0x7fffffffu) : ~s);
}
SP_DEVINL int key_token(unsigned long long k) { return (int)~(uint32_t)k; }

// Running max and sum of exponentials; +infinity counts its occurrences (the limit of the softmax).
struct MaxSum {
  float m, s;
  SP_DEVINL void add(float m2, float s2) {
    const float mn = fmaxf(m, m2);
    if (mn == -INFINITY) return;
    s = (m == mn ? s : s * ex2((m - mn) * kLog2e)) + (m2 == mn ? s2 : s2 * ex2((m2 - mn) * kLog2e));
    m = mn;
  }
};

// The n largest keys seen by a warp, one per lane in descending order.
struct WarpTop {
  unsigned long long key;  // lane i: the i-th largest (0: none)
  unsigned long long least;  // the n-th largest: what a new key has to exceed
  SP_DEVINL void offer(unsigned long long k, int n, int lane) {
    unsigned int some = __ballot_sync(0xffffffffu, k > least);
    while (some) {
      const int src = __ffs(some) - 1;
      some &= some - 1;
      const unsigned long long c = __shfl_sync(0xffffffffu, k, src);
      if (c <= least) continue;
      const int at = __popc(__ballot_sync(0xffffffffu, key > c));
      const unsigned long long up = __shfl_up_sync(0xffffffffu, key, 1);
      if (lane == at) key = c;
      else if (lane > at) key = up;
      if (lane >= n) key = 0;
      least = __shfl_sync(0xffffffffu, key, n - 1);
    }
  }
};

template <bool F32>
struct Chunk;  // 16 bytes of logits
template <>
struct Chunk<true> {
  static constexpr int N = 4;
  SP_DEVINL static void unpack(const uint4& u, float (&x)[4]) {
    x[0] = __uint_as_float(u.x);
    x[1] = __uint_as_float(u.y);
    x[2] = __uint_as_float(u.z);
    x[3] = __uint_as_float(u.w);
  }
  SP_DEVINL static float one(const void* row, int v) { return __ldg(static_cast<const float*>(row) + v); }
};
template <>
struct Chunk<false> {
  static constexpr int N = 8;
  SP_DEVINL static void unpack(const uint4& u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  SP_DEVINL static float one(const void* row, int v) {
    return __bfloat162float(static_cast<const __nv_bfloat16*>(row)[v]);
  }
};

// One CTA: a slice of one row.  Its (m, sum) and n_out largest keys to part.
template <bool F32>
__global__ void __launch_bounds__(BS_NT)
beam_scan_kernel(const void* __restrict__ logits, long long ld, int V, const float* __restrict__ cum,
                 const unsigned char* __restrict__ done, int n_out, int slice, float2* __restrict__ part_ms,
                 unsigned long long* __restrict__ part_key) {
  using K = Chunk<F32>;
  __shared__ unsigned long long top_s[BS_WARPS * BS_MAX_OUT];
  __shared__ float2 ms_s[BS_WARPS];
  pdl_wait();
  pdl_trigger();
  const int row = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if ((done && done[row]) || !(cum[row] > -INFINITY)) return;  // (the join reads nothing of such a beam's row)
  const char* base = static_cast<const char*>(logits) + row * ld * (F32 ? 4 : 2);
  const int v0 = min(blockIdx.x * slice, V), v1 = min(v0 + slice, V);
  // whole 16-byte chunks of the slice; what is before and behind them goes one by one
  const int esz = F32 ? 4 : 2;
  const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(base + (size_t)v0 * esz) & 15)) & 15) / esz, v1 - v0);
  const int c0 = v0 + head, chunks = (v1 - c0) / K::N, c1 = c0 + chunks * K::N;
  MaxSum ms{-INFINITY, 0.f};
  WarpTop top{0ull, 0ull};
  auto single = [&](float x, int v, bool in) {
    in = in && x > -INFINITY;  // (NaN and -infinity are no candidates and have no weight)
    if (in) ms.add(x, 1.f);
    top.offer(in ? cand_key(x, v) : 0ull, n_out, lane);
  };
  if (warp == 0 && head > 0) {
    const bool in = lane < head;
    single(in ? K::one(base, v0 + lane) : 0.f, v0 + lane, in);
  }
  if (warp == 1 && c1 < v1) {
    const bool in = lane < v1 - c1;
    single(in ? K::one(base, c1 + lane) : 0.f, c1 + lane, in);
  }
  const uint4* src = reinterpret_cast<const uint4*>(base + (size_t)c0 * esz);
  const int steps = (chunks + BS_NT - 1) / BS_NT;
  for (int i = 0; i < steps; ++i) {
    const int c = i * BS_NT + threadIdx.x;
    const bool in = c < chunks;
    float x[K::N];
    if (in) {
      K::unpack(__ldg(src + c), x);
    } else {
#pragma unroll
      for (int k = 0; k < K::N; ++k) x[k] = -INFINITY;
    }
    float cm = -INFINITY;
#pragma unroll
    for (int k = 0; k < K::N; ++k) cm = fmaxf(cm, x[k]);  // (fmaxf passes over NaN)
    if (cm > -INFINITY) {
      if (cm > ms.m) {
        ms.s = ms.m == -INFINITY ? 0.f : ms.s * ex2((ms.m - cm) * kLog2e);
        ms.m = cm;
      }
      if (ms.m == INFINITY) {
#pragma unroll
        for (int k = 0; k < K::N; ++k) ms.s += x[k] == INFINITY ? 1.f : 0.f;
      } else {
#pragma unroll
        for (int k = 0; k < K::N; ++k) {
          const float d = x[k] == x[k] ? x[k] : -INFINITY;
          ms.s += ex2((d - ms.m) * kLog2e);
        }
      }
    }
    if (__any_sync(0xffffffffu, cm > -INFINITY && cand_key(cm, 0) > top.least)) {
#pragma unroll
      for (int k = 0; k < K::N; ++k)
        top.offer(x[k] > -INFINITY ? cand_key(x[k], c0 + c * K::N + k) : 0ull, n_out, lane);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float m2 = __shfl_xor_sync(0xffffffffu, ms.m, o), s2 = __shfl_xor_sync(0xffffffffu, ms.s, o);
    ms.add(m2, s2);
  }
  if (lane < n_out) top_s[warp * n_out + lane] = top.key;
  if (lane == 0) ms_s[warp] = make_float2(ms.m, ms.s);
  __syncthreads();
  const size_t at = (size_t)row * gridDim.x + blockIdx.x;
  const int n = BS_WARPS * n_out;
  if (threadIdx.x < n) {  // rank of every warp's keys among all (no two are equal, but for the empty ones)
    const unsigned long long k = top_s[threadIdx.x];
    int rank = 0;
    for (int i = 0; i < n; ++i) {
      const unsigned long long u = top_s[i];
      rank += u > k || (u == k && i < threadIdx.x);
    }
    if (rank < n_out) part_key[at * n_out + rank] = k;
  }
  if (threadIdx.x == 0) {
    for (int w = 1; w < BS_WARPS; ++w) ms.add(ms_s[w].x, ms_s[w].y);
    part_ms[at] = make_float2(ms.m, ms.s);
  }
}

SP_DEVINL double shfl_xor_d(double v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }

// One CTA per element, a warp per beam: the slices' lists joined into the beam's n_out best, their scores in
// 64 bits, then one warp takes the n_out best over the beams.
__global__ void __launch_bounds__(512)
beam_join_kernel(int W, int V, int S, const float* __restrict__ cum, const unsigned char* __restrict__ done, int eos,
                 int n_out, const float2* __restrict__ part_ms, const unsigned long long* __restrict__ part_key,
                 float* __restrict__ score, int* __restrict__ parent, int* __restrict__ token) {
  __shared__ double sc_s[16 * BS_MAX_OUT];
  __shared__ int tk_s[16 * BS_MAX_OUT];
  pdl_wait();
  pdl_trigger();
  const int e = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp < W) {
    const int row = e * W + warp;
    const float cw = cum[row];
    double sc = -INFINITY;
    int tk = -1;
    if (!(cw > -INFINITY)) {
    } else if (done && done[row]) {
      if (lane == 0) {
        sc = cw;
        tk = eos;
      }
    } else {
      float m = -INFINITY;
      for (int s = lane; s < S; s += 32) m = fmaxf(m, __ldcg(part_ms + (size_t)row * S + s).x);
      m = warp_max(m);
      double sum = 0.0;
      for (int s = lane; s < S; s += 32) {
        const float2 u = __ldcg(part_ms + (size_t)row * S + s);
        if (u.x == m) sum += u.y;
        else if (u.x > -INFINITY) sum += (double)u.y * exp((double)u.x - (double)m);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += shfl_xor_d(sum, o);
      const double lsum = log(sum);
      // S sorted lists: a lane holds the heads of lists lane, lane + 32, ... one after the other
      const unsigned long long* keys = part_key + (size_t)row * S * n_out;
      unsigned long long mine = 0, best = 0;
      for (int l0 = 0; l0 < S; l0 += 32) {  // 32 lists at a time into the running n_out best
        int head = 0;
        const int l = l0 + lane;
        unsigned long long h = l < S ? __ldcg(keys + (size_t)l * n_out) : 0ull;
        unsigned long long old = mine;  // the best so far, in lane order: a 33rd list
        int taken = 0;                  // of them
        mine = 0;
        for (int r = 0; r < n_out; ++r) {
          const unsigned long long o33 = __shfl_sync(0xffffffffu, old, taken);
          best = h;
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) {
            const unsigned long long u = __shfl_xor_sync(0xffffffffu, best, o);
            if (u > best) best = u;
          }
          if (o33 >= best) {
            best = o33;
            ++taken;
          } else if (h == best) {
            ++head;
            h = head < n_out ? __ldcg(keys + (size_t)l * n_out + head) : 0ull;
          }
          if (lane == r) mine = best;
        }
      }
      if (mine != 0 && lane < n_out) {
        const float x = key_logit(mine);
        const double d = x == m ? 0.0 : (double)x - (double)m;  // (m = +infinity: its tokens alone have weight)
        sc = (double)cw + (d - lsum);
        tk = key_token(mine);
      }
    }
    if (lane < n_out) {
      sc_s[warp * n_out + lane] = sc;
      tk_s[warp * n_out + lane] = tk;
    }
  }
  __syncthreads();
  if (warp != 0) return;
  int head = 0;  // lane w: the head of beam w's list
  for (int r = 0; r < n_out; ++r) {
    double s = -INFINITY;
    int t = -1;
    if (lane < W && head < n_out) {
      s = sc_s[lane * n_out + head];
      t = tk_s[lane * n_out + head];
    }
    int from = lane;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const double s2 = shfl_xor_d(s, o);
      const int t2 = __shfl_xor_sync(0xffffffffu, t, o), f2 = __shfl_xor_sync(0xffffffffu, from, o);
      if (t2 >= 0 && (t < 0 || s2 > s || (s2 == s && f2 < from))) {
        s = s2;
        t = t2;
        from = f2;
      }
    }
    if (t >= 0 && from == lane) ++head;
    if (lane == 0) {
      score[(size_t)e * n_out + r] = t >= 0 ? (float)s : -INFINITY;
      parent[(size_t)e * n_out + r] = t >= 0 ? from : -1;
      token[(size_t)e * n_out + r] = t;
    }
  }
}

// --------------------------------------------------------------- reordering
// Beam w of an element continues beam p(w).  Full pages are never written again, so beams share them: w's
// table takes p(w)'s entries.  The partly filled page is copied: every beam has a page of its own for each
// place of its table (own_table), the only ones it ever writes, so the rows of own[p(w)] go to own[w], in
// place for all beams at once: a thread reads its 16 bytes of every parent before it writes any.
// blockIdx.y: a plane (layer, K or V), or behind the last the tables; bound by the copied rows' bytes.
constexpr int BR_NT = 256;

template <int WMAX>
__global__ void __launch_bounds__(BR_NT)
beam_reorder_kernel(uint4* __restrict__ kv, int planes, int n_pages, int page_shift, int row16, int* __restrict__ table,
                    const int* __restrict__ own, int max_pages, const int* __restrict__ lens,
                    const int* __restrict__ parent, int ld_parent, int W, int* err) {
  __shared__ int par[WMAX];
  __shared__ int src_page[WMAX], dst_page[WMAX];
  __shared__ int ok_s;
  pdl_wait();
  pdl_trigger();
  const int e = blockIdx.z, tid = threadIdx.x;
  const int len = __ldg(lens + e * W);
  if (tid == 0) ok_s = 1;
  __syncthreads();
  const int full = len >> page_shift;  // (of a negative length: negative)
  if (tid < W) {
    int q = __ldg(parent + (size_t)e * ld_parent + tid);
    if (q < -1 || q >= W) {
      set_error(err, SP_DEVERR_INDEX);
      q = -1;
    }
    par[tid] = q < 0 ? tid : q;
    // all beams of an element are equally long, and within their tables
    if (__ldg(lens + e * W + tid) != len || len < 0 || len > (max_pages << page_shift)) {
      set_error(err, SP_DEVERR_INDEX);
      ok_s = 0;
    }
  }
  __syncthreads();
  if (!ok_s) return;
  if (blockIdx.y == planes) {  // the tables: a column per thread
    for (int c = blockIdx.x * BR_NT + tid; c < max_pages; c += gridDim.x * BR_NT) {
      int v[WMAX];
#pragma unroll
      for (int w = 0; w < WMAX; ++w)
        if (w < W) v[w] = c < full ? table[(size_t)(e * W + par[w]) * max_pages + c] : __ldg(own + (size_t)(e * W + w) * max_pages + c);
#pragma unroll
      for (int w = 0; w < WMAX; ++w)
        if (w < W) table[(size_t)(e * W + w) * max_pages + c] = v[w];
    }
    return;
  }
  const int rows = len & ((1 << page_shift) - 1);
  if (rows == 0) return;
  if (tid < W) {
    const int s = __ldg(own + (size_t)(e * W + par[tid]) * max_pages + full);
    const int d = __ldg(own + (size_t)(e * W + tid) * max_pages + full);
    const bool ok = s >= 0 && s < n_pages && d >= 0 && d < n_pages;
    if (!ok) set_error(err, SP_DEVERR_INDEX);
    src_page[tid] = ok && s != d ? s : -1;
    dst_page[tid] = d;
  }
  __syncthreads();
  uint4* pl = kv + (((size_t)blockIdx.y * n_pages) << page_shift) * row16;
  const int n = rows * row16;
  for (int i = blockIdx.x * BR_NT + tid; i < n; i += gridDim.x * BR_NT) {
    uint4 v[WMAX];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < W && src_page[w] >= 0) v[w] = pl[((size_t)src_page[w] << page_shift) * row16 + i];
#pragma unroll
    for (int w = 0; w < WMAX; ++w)
      if (w < W && src_page[w] >= 0) pl[((size_t)dst_page[w] << page_shift) * row16 + i] = v[w];
  }
}

}  // namespace

int beam_slices(int rows, int V) {
  // slices of a row: enough CTAs for four per SM, of at least 2,048 logits each
  const int want = (device_sm_count() * 4 + rows - 1) / rows;
  return std::max(1, std::min(want, (V + 2047) / 2048));
}

size_t beam_select_bytes(int rows, int V, int n_out) {
  const size_t n = (size_t)rows * beam_slices(rows, V);
  return ((n * 8 + 255) & ~size_t(255)) + n * n_out * 8;
}

cudaError_t beam_select_launch(const void* logits, bool f32, long long ld, int B, int W, int V, const float* cum,
                               const unsigned char* done, int eos, int n_out, void* ws, float* score, int* parent,
                               int* token, cudaStream_t st) {
  const int rows = B * W, S = beam_slices(rows, V);
  const int slice = (((V + S - 1) / S) + 7) & ~7;
  auto* ms = static_cast<float2*>(ws);
  auto* key = reinterpret_cast<unsigned long long*>(static_cast<char*>(ws) + (((size_t)rows * S * 8 + 255) & ~size_t(255)));
  prof_begin_launch(st);
  cudaError_t r = f32 ? launch_pdl(beam_scan_kernel<true>, dim3(S, rows), dim3(BS_NT), 0, st, logits, ld, V, cum, done,
                                   n_out, slice, ms, key)
                      : launch_pdl(beam_scan_kernel<false>, dim3(S, rows), dim3(BS_NT), 0, st, logits, ld, V, cum, done,
                                   n_out, slice, ms, key);
  prof_end_launch(st, SP_K_MISC, 0.0, (double)rows * V * (f32 ? 4 : 2));
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  r = launch_pdl(beam_join_kernel, dim3(B), dim3(W * 32), 0, st, W, V, S, cum, done, eos, n_out,
                 (const float2*)ms, (const unsigned long long*)key, score, parent, token);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

cudaError_t beam_reorder_launch(void* kv, int n_layers, int n_pages, int page_shift, int row_bytes, int* table,
                                const int* own, int max_pages, const int* lens, const int* parent, int ld_parent,
                                int B, int W, int* err, cudaStream_t st) {
  const int planes = 2 * n_layers, row16 = row_bytes / 16;
  const int most = ((1 << page_shift) - 1) * row16;  // chunks of a plane's partly filled page, at most
  const int gx = std::max(1, std::min((most + BR_NT - 1) / BR_NT, 8));
  const dim3 grid(gx, planes + 1, B);
  auto* k = W <= 4 ? beam_reorder_kernel<4> : W <= 8 ? beam_reorder_kernel<8> : beam_reorder_kernel<16>;
  prof_begin_launch(st);
  const cudaError_t r = launch_pdl(k, grid, dim3(BR_NT), 0, st, static_cast<uint4*>(kv), planes, n_pages, page_shift,
                                   row16, table, own, max_pages, lens, parent, ld_parent, W, err);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
