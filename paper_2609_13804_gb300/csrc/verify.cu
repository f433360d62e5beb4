// Verification of drafted tokens.  With p_j = softmax(x_j / t) of the target's logits in a sequence's row j and
// q_j = softmax(y_j / t) of the draft's, the drafted token d_j stays iff u_j q_j(d_j) < p_j(d_j); at the first row that
// rejects its draft (or the last, which has none) the next token is drawn from what is left,
//   r = max(p_a - q_a, 0), or p_a behind the last draft,
// by an exponential race: argmax r(v) / E(v) with E(v) ~ Exp(1) falls on v with probability r(v) / sum r.  Nothing but
// a maximum is taken over the race, so it needs no sum of r, and its answer moves only if two of V scores are nearer
// than fp32 tells apart.
//
// Two kernels: the sums of every row, then per sequence the decision and the race over the one row where it ends.
#include <algorithm>
#include <cfloat>

#include "common.cuh"
#include "internal.h"
#include "logits.cuh"

namespace sp {

namespace {

constexpr int VF_NT = 256, VF_WARPS = VF_NT / 32;
constexpr int VF_LOADS = 4;    // 16-byte loads of a thread at once
constexpr int VF_SLICES = 32;  // of a row, at most: a lane joins each
constexpr int VF_CLUSTER = 8;  // CTAs of a sequence's race, at most

// A slice's maximum, its sum of exp((x - m) / t) and the first token that holds the maximum (greedy sequences).
struct __align__(16) RowPart {
  float m, s;
  int at, unused;
};

struct Seq {
  int row0, n;    // its rows (0: none)
  bool greedy;
  float t;        // temperature, 1 where greedy
  float c;        // log2 e / t, kept within the finite numbers so that 0 c is 0
};

SP_DEVINL Seq sequence(const VerifyArgs& a, int b) {
  Seq q;
  q.row0 = a.cu_rows ? __ldg(a.cu_rows + b) : b;
  const long long n = a.cu_rows ? (long long)__ldg(a.cu_rows + b + 1) - q.row0 : 1;
  q.n = q.row0 >= 0 && n >= 0 && n <= a.max_rows && q.row0 + n <= a.T_cap ? (int)n : -1;
  const float t = a.temperature ? __ldg(a.temperature + b) : 1.f;
  q.greedy = !a.noise || !(t > 0.f);
  q.t = q.greedy ? 1.f : t;
  q.c = fmaxf(fminf(kLog2e / q.t, FLT_MAX), FLT_MIN);
  return q;
}

// exp((x - m) / t) of a row with maximum m: 1 at the maximum (the tokens at +infinity have all the weight between
// them), 0 for NaN and -infinity.
SP_DEVINL float weight(float x, float m, float c) { return x == m ? 1.f : x < m ? ex2((x - m) * c) : 0.f; }

// Sums of every row, a slice to a CTA: blockIdx.x = which * slices + slice (which: 0 the target's, 1 the draft's).
template <bool F32>
__global__ void __launch_bounds__(VF_NT, 4) verify_sums_kernel(const VerifyArgs a, int slices, int slice, RowPart* part) {
  using K = Chunk<F32>;
  __shared__ float2 ms_s[VF_WARPS];
  __shared__ int at_s[VF_WARPS];
  pdl_wait();
  const int which = blockIdx.x / slices, sl = blockIdx.x % slices, j = blockIdx.z;
  const Seq q = sequence(a, blockIdx.y);
  if (j >= q.n || (which == 1 && (q.greedy || j == q.n - 1))) return;
  const int row = q.row0 + j, tid = threadIdx.x;
  constexpr int esz = F32 ? 4 : 2;
  const char* base = static_cast<const char*>(which ? a.draft_logits : a.logits) + row * (which ? a.ld_draft : a.ld) * esz;
  const int v0 = min(sl * slice, a.V), v1 = min(v0 + slice, a.V);
  // whole 16-byte pieces of the slice; what is before and behind them goes one by one
  const int off = reinterpret_cast<uintptr_t>(base + (size_t)v0 * esz) & 15;
  const int c0 = v0 + min(((16 - off) & 15) / esz, v1 - v0), chunks = (v1 - c0) / K::N, c1 = c0 + chunks * K::N;
  const uint4* src = reinterpret_cast<const uint4*>(base + (size_t)c0 * esz);
  float m = -INFINITY, s = 0.f;
  int first = -1;  // the first batch of loads that holds m
  const int beside = tid < c0 - v0 ? v0 + tid : c1 + tid - (c0 - v0);
  const float mine = beside < (tid < c0 - v0 ? c0 : v1) ? K::one(base, beside) : -INFINITY;
  for (int c = tid; c < chunks; c += VF_NT * VF_LOADS) {
    uint4 u[VF_LOADS];
#pragma unroll
    for (int k = 0; k < VF_LOADS; ++k)
      u[k] = c + k * VF_NT < chunks ? __ldcs(src + c + k * VF_NT) : make_uint4(K::kNone, K::kNone, K::kNone, K::kNone);
    float lm = -INFINITY;
#pragma unroll
    for (int k = 0; k < VF_LOADS; ++k) lm = fmaxf(lm, K::top(u[k]));
    if (lm == -INFINITY) continue;
    if (lm > m) {
      s = m == -INFINITY ? 0.f : s * ex2((m - lm) * q.c);
      m = lm;
      first = c;
    }
    // (x - m first, exactly where it matters: m log2 e rounded would shift the whole sum)
    const unsigned long long nm = pack2(-m, -m), cc = pack2(q.c, q.c);
    unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
    for (int k = 0; k < VF_LOADS; ++k)
#pragma unroll
      for (int i = 0; i < K::N; i += 2) {
        float x, y;
        unpack2(mul2(add2(pack2(K::at(u[k], i), K::at(u[k], i + 1)), nm), cc), x, y);
        sum[(i >> 1) & 1] = add2(sum[(i >> 1) & 1], pack2(ex2(x), ex2(y)));
      }
    float sa, sb;
    unpack2(add2(sum[0], sum[1]), sa, sb);
    float ts = sa + sb;
    if (ts != ts) {  // a NaN, or infinity less infinity, among them
      ts = 0.f;
#pragma unroll
      for (int k = 0; k < VF_LOADS; ++k)
#pragma unroll
        for (int i = 0; i < K::N; ++i) ts += weight(K::at(u[k], i), m, q.c);
    }
    s += ts;
  }
  if (mine > -INFINITY) {
    const float mn = fmaxf(m, mine);
    s = (m > -INFINITY ? s * weight(m, mn, q.c) : 0.f) + weight(mine, mn, q.c);
    if (mine > m) first = -1;
    m = mn;
  }
  pdl_trigger();
  const int warp = tid >> 5, lane = tid & 31;
  const float mw = warp_max(m);
  const float sw = warp_sum(m > -INFINITY ? (m == mw ? s : s * ex2((m - mw) * q.c)) : 0.f);
  if (lane == 0) ms_s[warp] = make_float2(mw, sw);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < VF_WARPS; ++w) top = fmaxf(top, ms_s[w].x);
  int at = 0x7fffffff;
  if (q.greedy && m == top && m > -INFINITY) {  // the first of this thread's tokens with the maximum
    if (mine == top) at = beside;
    if (first >= 0) {
#pragma unroll 1
      for (int i = 0; i < VF_LOADS * K::N; ++i) {
        const int c = first + i / K::N * VF_NT, v = c0 + c * K::N + i % K::N;
        if (c < chunks && K::one(base, v) == top) {
          at = min(at, v);
          break;
        }
      }
    }
  }
  if (q.greedy) {
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) at_s[warp] = at;
    __syncthreads();
  }
  if (tid == 0) {
    float sum = 0.f;
    for (int w = 0; w < VF_WARPS; ++w) {
      if (ms_s[w].x > -INFINITY) sum += ms_s[w].x == top ? ms_s[w].y : ms_s[w].y * ex2((ms_s[w].x - top) * q.c);
      if (q.greedy) at = min(at, at_s[w]);
    }
    part[((size_t)row * 2 + which) * slices + sl] = RowPart{top, sum, at, 0};
  }
}

// A row's maximum, sum and (greedy) first token with the maximum, joined by a warp from its slices; every lane has them.
SP_DEVINL RowPart join_row(const RowPart* part, int slices, float c) {
  const int lane = threadIdx.x & 31;
  RowPart r{-INFINITY, 0.f, 0x7fffffff, 0};
  if (lane < slices) {
    const int4 v = __ldcg(reinterpret_cast<const int4*>(part) + lane);
    r = RowPart{__int_as_float(v.x), __int_as_float(v.y), v.z, 0};
  }
  const float m = warp_max(r.m);
  const float s = warp_sum(r.m > -INFINITY ? (r.m == m ? r.s : r.s * ex2((r.m - m) * c)) : 0.f);
  const int at = __reduce_min_sync(0xffffffffu, r.m == m ? r.at : 0x7fffffff);
  return RowPart{m, s, at, 0};
}

// p(x) and log p(x) of a logit in a row, from its maximum and sum, in 64 bits.
SP_DEVINL double prob(float x, const RowPart& r, float t) {
  if (!(x > -INFINITY) || !(x <= r.m)) return 0.0;
  return (x == r.m ? 1.0 : exp(((double)x - (double)r.m) / (double)t)) / (double)r.s;
}
SP_DEVINL float log_prob(float x, const RowPart& r, float t) {
  if (!(x > -INFINITY) || !(x <= r.m)) return -INFINITY;
  return (float)((x == r.m ? 0.0 : ((double)x - (double)r.m) / (double)t) - log((double)r.s));
}

// A race's score and token as one key that sorts by (score, lower token first); scores are above 0, 0: none.
SP_DEVINL unsigned long long race_key(float score, int v) {
  return ((unsigned long long)__float_as_uint(score) << 32) | (uint32_t)~v;
}

// The row where a sequence ends, as its race needs it.
template <bool F32>
struct Race {
  const void *p, *q;  // q NULL: nothing is taken off
  const float* e;
  float mp, ip, mq, iq, c;  // maxima and inverse sums
  int out;                  // a token whose probability is taken off whole (a draft without a distribution), -1: none

  SP_DEVINL void take(float x, float y, float noise, int v, float& best, int& at) const {
    float r = weight(x, mp, c) * ip;
    if (q) r = fmaxf(r - weight(y, mq, c) * iq, 0.f);
    if (v == out) r = 0.f;
    const float score = __fdividef(r, noise);  // (noise 0: infinity, or NaN for r = 0, which is no candidate)
    if (score > best) {
      best = score;
      at = v;
    }
  }
  // The best of tokens v0 .. v1 - 1 for this thread of the CTA.
  SP_DEVINL unsigned long long run(int v0, int v1) const {
    using K = Chunk<F32>;
    constexpr int esz = F32 ? 4 : 2;
    float best = 0.f;
    int at = 0;
    const char* pb = static_cast<const char*>(p) + (size_t)v0 * esz;
    const char* qb = static_cast<const char*>(q) + (size_t)v0 * esz;
    const int off = reinterpret_cast<uintptr_t>(pb) & 15, head = min(((16 - off) & 15) / esz, v1 - v0);
    const int c0 = v0 + head;
    const bool together = (!q || (reinterpret_cast<uintptr_t>(qb) & 15) == off) &&
                          (reinterpret_cast<uintptr_t>(e + c0) & 15) == 0;
    if (!together) {
#pragma unroll 4
      for (int v = v0 + threadIdx.x; v < v1; v += VF_NT)
        take(K::one(p, v), q ? K::one(q, v) : 0.f, __ldg(e + v), v, best, at);
      return best > 0.f ? race_key(best, at) : 0ull;
    }
    const int chunks = (v1 - c0) / K::N, c1 = c0 + chunks * K::N;
    unsigned long long key = 0;
    if (threadIdx.x < head + v1 - c1) {
      const int v = threadIdx.x < head ? v0 + threadIdx.x : c1 + threadIdx.x - head;
      take(K::one(p, v), q ? K::one(q, v) : 0.f, __ldg(e + v), v, best, at);
      if (best > 0.f) key = race_key(best, at);
      best = 0.f;
    }
    const uint4* ps = reinterpret_cast<const uint4*>(static_cast<const char*>(p) + (size_t)c0 * esz);
    const uint4* qs = reinterpret_cast<const uint4*>(static_cast<const char*>(q) + (size_t)c0 * esz);
    const float4* es = reinterpret_cast<const float4*>(e + c0);
#pragma unroll 2
    for (int c = threadIdx.x; c < chunks; c += VF_NT) {
      const uint4 x = __ldg(ps + c), y = q ? __ldg(qs + c) : make_uint4(0, 0, 0, 0);
      float4 n[K::N / 4];
#pragma unroll
      for (int k = 0; k < K::N / 4; ++k) n[k] = __ldcs(es + c * (K::N / 4) + k);
#pragma unroll
      for (int i = 0; i < K::N; ++i) {
        const float4& f = n[i / 4];
        take(K::at(x, i), K::at(y, i), i % 4 == 0 ? f.x : i % 4 == 1 ? f.y : i % 4 == 2 ? f.z : f.w, c0 + c * K::N + i,
             best, at);
      }
    }
    return best > 0.f ? max(key, race_key(best, at)) : key;
  }
};

// The largest of the CTA's keys, in every thread of warp 0.
SP_DEVINL unsigned long long cta_max(unsigned long long k, unsigned long long* s) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = ((unsigned long long)hi << 32) | lo;
  __syncthreads();
  k = 0;
#pragma unroll
  for (int w = 0; w < VF_WARPS; ++w) k = max(k, s[w]);
  return k;
}

// A cluster per sequence: every CTA finds the row where it ends, each races over its slice of it.
template <bool F32>
__global__ void __launch_bounds__(VF_NT) verify_end_kernel(const VerifyArgs a, int slices, const RowPart* part) {
  using K = Chunk<F32>;
  __shared__ RowPart p_s[VF_WARPS], q_s[VF_WARPS];
  __shared__ int accept_s[VF_WARPS];
  __shared__ unsigned long long key_s[VF_WARPS], cluster_s[VF_CLUSTER];
  pdl_wait();
  pdl_trigger();
  const int C = gridDim.x, rank = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Seq q = sequence(a, b);
  int* token = a.token + (size_t)b * a.max_rows;
  float* logp = a.logp ? a.logp + (size_t)b * a.max_rows : nullptr;
  if (rank == 0)
    for (int j = max(q.n, 0) + tid; j < a.max_rows; j += VF_NT) {
      token[j] = -1;
      if (logp) logp[j] = 0.f;
    }
  if (q.n <= 0) {  // (no row, or rows that are not there)
    if (rank == 0 && tid == 0) {
      if (q.n < 0) set_error(a.err, SP_DEVERR_INDEX);
      a.n_accept[b] = -1;
    }
    return;
  }
  constexpr int esz = F32 ? 4 : 2;
  auto logits = [&](int j) { return static_cast<const char*>(a.logits) + (q.row0 + j) * a.ld * esz; };
  auto draft_logits = [&](int j) { return static_cast<const char*>(a.draft_logits) + (q.row0 + j) * a.ld_draft * esz; };
  int end = -1;
  for (int j0 = 0; end < 0; j0 += VF_WARPS) {  // a warp to a row
    const int j = j0 + warp;
    bool stays = true;
    if (j < q.n) {
      const int row = q.row0 + j;
      const int d = j < q.n - 1 ? __ldg(a.draft + row) : -1;
      const bool there = d >= 0 && d < a.V;
      const RowPart p = join_row(part + ((size_t)row * 2) * slices, slices, q.c);
      const bool with_q = a.draft_logits && !q.greedy && j < q.n - 1;
      RowPart r{0.f, 0.f, 0, 0};
      if (with_q) r = join_row(part + ((size_t)row * 2 + 1) * slices, slices, q.c);
      if (lane == 0) {
        stays = false;
        if (j < q.n - 1) {
          if (!there) {
            if (rank == 0) set_error(a.err, SP_DEVERR_INDEX);
          } else if (q.greedy) {
            stays = d == p.at;
          } else {
            const double pd = prob(K::one(logits(j), d), p, q.t);
            const double qd = with_q ? prob(K::one(draft_logits(j), d), r, q.t) : 1.0;
            stays = (double)__ldg(a.u + row) * qd < pd;
          }
        }
        p_s[warp] = p;
        q_s[warp] = r;
      }
    }
    if (lane == 0) accept_s[warp] = stays;
    __syncthreads();
    int w = 0;
    while (w < VF_WARPS && accept_s[w]) ++w;
    if (w < VF_WARPS) end = j0 + w;
    if (rank == 0 && lane == 0 && j < q.n && warp < w) {
      const int d = __ldg(a.draft + q.row0 + j);
      token[j] = d;
      if (logp) logp[j] = log_prob(K::one(logits(j), d), p_s[warp], q.t);
    }
    if (end < 0) __syncthreads();
  }
  const RowPart p = p_s[end % VF_WARPS], r = q_s[end % VF_WARPS];
  const bool drafted = end < q.n - 1;
  if (rank == 0)
    for (int j = end + 1 + tid; j < q.n; j += VF_NT) {
      token[j] = -1;
      if (logp) logp[j] = 0.f;
    }
  // (sequences whose offsets overlap can find another's sums: never a token that is not there)
  int next = p.m > -INFINITY && p.at >= 0 && p.at < a.V ? p.at : -1;
  if (!q.greedy) {
    if (C > 1) cluster_sync_all();  // every CTA of the cluster runs
    Race<F32> race;
    race.p = logits(end);
    race.q = drafted && a.draft_logits ? draft_logits(end) : nullptr;
    race.e = a.noise + (size_t)b * a.ld_noise;
    race.mp = p.m;
    race.ip = p.s > 0.f ? 1.f / p.s : 0.f;
    race.mq = r.m;
    race.iq = r.s > 0.f ? 1.f / r.s : 0.f;
    race.c = q.c;
    race.out = drafted && !a.draft_logits ? __ldg(a.draft + q.row0 + end) : -1;
    const int per = (((a.V + C - 1) / C) + 7) & ~7;
    const int v0 = min(rank * per, a.V), v1 = min(v0 + per, a.V);
    unsigned long long key = cta_max(race.run(v0, v1), key_s);
    if (C > 1) {
      if (tid == 0) {
        const uint32_t to = mapa_shared(smem_u32(&cluster_s[rank]), 0);
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(key) : "memory");
      }
      cluster_sync_all();
      if (rank != 0) return;
      for (int i = 0; i < C; ++i) key = max(key, cluster_s[i]);
    }
    if (key == 0 && drafted) {  // p and q are the same (or p is all at the draft): from p
      race.q = nullptr;
      race.out = -1;
      key = cta_max(race.run(0, a.V), key_s);
    }
    next = key != 0 ? (int)~(uint32_t)key : -1;
  }
  if (rank == 0 && tid == 0) {
    a.n_accept[b] = end;
    token[end] = next;
    if (logp) logp[end] = next >= 0 ? log_prob(K::one(logits(end), next), p, q.t) : -INFINITY;
  }
}

}  // namespace

static int verify_slices(int rows, int V) {
  rows = std::max(rows, 1);
  const int want = (device_sm_count() * 4 + rows / 2) / rows;
  return std::max(1, std::min(std::min(std::max(want, (V + 32767) / 32768), VF_SLICES), (V + 4095) / 4096));
}

size_t verify_bytes(int T_cap, int V) { return (size_t)T_cap * 2 * verify_slices(T_cap, V) * sizeof(RowPart); }

cudaError_t verify_launch(const VerifyArgs& a, void* ws, cudaStream_t st) {
  auto* part = static_cast<RowPart*>(ws);
  const int slices = verify_slices(a.T_cap, a.V), slice = (((a.V + slices - 1) / slices) + 7) & ~7;
  cudaError_t r = cudaSuccess;
  if (a.T_cap > 0) {
    prof_begin_launch(st);
    r = launch_pdl(a.logits_f32 ? verify_sums_kernel<true> : verify_sums_kernel<false>,
                   dim3(slices * (a.draft_logits ? 2 : 1), a.B, a.max_rows), dim3(VF_NT), 0, st, a, slices, slice, part);
    prof_end_launch(st, SP_K_MISC, 0.0, (double)a.T_cap * a.V * (a.logits_f32 ? 4 : 2) * (a.draft_logits ? 2 : 1));
    if (r != cudaSuccess) return r;
  }
  const int C = a.noise ? std::max(1, std::min(VF_CLUSTER, (a.V + 2047) / 2048)) : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C, a.B);
  cfg.blockDim = dim3(VF_NT);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  prof_begin_launch(st);
  r = cudaLaunchKernelEx(&cfg, a.logits_f32 ? verify_end_kernel<true> : verify_end_kernel<false>, a, slices,
                         (const RowPart*)part);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
