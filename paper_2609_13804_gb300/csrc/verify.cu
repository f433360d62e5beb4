// Verification of drafted tokens.  With p_j = softmax(x_j / t) of the target's logits in a sequence's row j and
// q_j = softmax(y_j / t) of the draft's, the drafted token d_j stays iff u_j q_j(d_j) < p_j(d_j); at the first row that
// rejects its draft (or the last, which has none) the next token is drawn from what is left,
//   r = max(p_a - q_a, 0), or p_a behind the last draft,
// by an exponential race: argmax r(v) / E(v) with E(v) ~ Exp(1) falls on v with probability r(v) / sum r.  Nothing but
// a maximum is taken over the race, so it needs no sum of r, and its answer moves only if two of V scores are nearer
// than fp32 tells apart.
//
// Two kernels: the sums of every row (a maximum and a sum of exponentials, one pass), then per sequence the decision and the
// race over the one row where it ends.  Bound by reading: every row that is looked at once, the last one twice and the noise.
// Without drafts one kernel does both in one pass.  Weights, sums and scores are fp32 and no operand is narrowed; exponentials,
// the noise's reciprocals and a log-probability's quotient are the hardware's approximations, good to 2^-22.  Decisions
// multiply sums out.
#include <algorithm>
#include <cfloat>

#include "common.cuh"
#include "internal.h"
#include "logits.cuh"
#include "verify_cut.h"

namespace sp {

namespace {

constexpr int VF_NT = 256, VF_WARPS = VF_NT / 32;
constexpr int VF_LOADS = 4;    // 16-byte loads of a thread at once
constexpr int VF_RING = 3;     // batches of loads in shared memory
constexpr int VF_RING_BYTES = VF_RING * VF_LOADS * VF_NT * 16;
static_assert(kRowSlices <= 32, "a lane joins each");
constexpr int VF_CLUSTER = 8;  // CTAs of a sequence's race, at most

// A slice's maximum, its sum of exp((x - m) / t) and the first token that holds the maximum (greedy sequences).
struct __align__(16) RowPart {
  float m, s;
  int at;
  float xd;  // slice 0: the row's logit of the draft, -infinity where there is none
};

struct Seq {
  int row0, n;    // its rows (0: none)
  bool greedy;
  float t;        // temperature, 1 where greedy
  float c;        // log2 e / t, kept so that 0 c is 0 and -infinity c is -infinity
};

SP_DEVINL Seq sequence(const VerifyArgs& a, int b) {
  Seq q;
  q.row0 = a.cu_rows ? __ldg(a.cu_rows + b) : b;
  const long long n = a.cu_rows ? (long long)__ldg(a.cu_rows + b + 1) - q.row0 : 1;
  q.n = q.row0 >= 0 && n >= 0 && n <= a.max_rows && q.row0 + n <= a.T_cap ? (int)n : -1;
  const float t = a.temperature ? __ldg(a.temperature + b) : 1.f;
  q.greedy = !a.noise || !(t > 0.f);
  q.t = q.greedy ? 1.f : t;
  q.c = fmaxf(fminf(kLog2e / q.t, 0x1p64f), FLT_MIN);
  return q;
}

// exp((x - m) / t) of a row with maximum m: 1 at the maximum (the tokens at +infinity have all the weight between
// them), 0 for NaN and -infinity.
SP_DEVINL float weight(float x, float m, float c) { return x == m ? 1.f : x < m ? ex2((x - m) * c) : 0.f; }

// Where a row's exponents m c are of ordinary size, weights are exp2(x c - z) with the whole number z next to m c: one fused
// multiply-add, rounded once (m c itself, rounded, would shift all of them), and powers of two between threads whose
// maxima differ.  Else (maxima at infinity or at a type's lowest value, temperatures near 0) they are weight()'s.
SP_DEVINL bool ordinary(float mc) { return fabsf(mc) < 4194304.f; }

// A thread's share of a slice: its maximum, its sum and the first batch of loads that holds the maximum; with noise the
// best of its race too, the logit and noise of which are kept: scores of threads with different maxima are formed again.
struct Share {
  float m, z, s;  // (s in units of exp2(z) where m c is ordinary, else of exp(m / t))
  int first;
  float x, e;  // the race's best so far
  int at;      // -1: none
  bool usual;  // m c is ordinary
  bool infinite;  // the race has had an infinite score (noise of 0): others were not kept, which count if its weight ends as 0
};

// Tokens v0 .. v1 - 1 of a row, 16 bytes at a time where they lie whole in the slice.
template <bool F32>
struct Slice {
  using K = Chunk<F32>;
  static constexpr int esz = F32 ? 4 : 2;
  const char* base;
  int v0, v1, c0, c1, chunks;
  SP_DEVINL Slice(const void* row, int from, int to) : base(static_cast<const char*>(row)), v0(from), v1(to) {
    const int off = reinterpret_cast<uintptr_t>(base + (size_t)v0 * esz) & 15;
    c0 = v0 + min(((16 - off) & 15) / esz, v1 - v0);
    chunks = (v1 - c0) / K::N;
    c1 = c0 + chunks * K::N;
  }
  SP_DEVINL const uint4* src() const { return reinterpret_cast<const uint4*>(base + (size_t)c0 * esz); }
  // the token beside the whole pieces that this thread takes (fewer than 16), -1: none
  SP_DEVINL int beside() const {
    const int i = threadIdx.x, head = c0 - v0;
    return i < head ? v0 + i : c1 + i - head < v1 ? c1 + i - head : -1;
  }
  // the first token of this thread that holds the maximum `top`
  SP_DEVINL int first_of(float top, int first) const {
    int at = 0x7fffffff;
    if (beside() >= 0 && K::one(base, beside()) == top) at = beside();
    if (first >= 0) {
#pragma unroll 1
      for (int i = 0; i < VF_LOADS * K::N; ++i) {
        const int c = first + i / K::N * VF_NT, v = c0 + c * K::N + i % K::N;
        if (c < chunks && K::one(base, v) == top) return min(at, v);
      }
    }
    return at;
  }
};

// Raises a share's maximum to m; what it had counts `the result` as much.
SP_DEVINL float raise_to(float m, float c, Share& r) {
  const float mc = m * c, z = rintf(mc);
  const bool usual = ordinary(mc);
  float f;
  if (usual && r.usual) {
    f = ex2(r.z - z);  // (0 at first, when both are -infinity)
  } else {
    f = r.m == -INFINITY ? 0.f : ex2((r.m - m) * c);
    if (r.usual && r.m > -INFINITY) f *= ex2(__fmaf_rn(-r.m, c, r.z));
    if (usual) f *= ex2(__fmaf_rn(m, c, -z));
  }
  r.s *= f;
  r.m = m;
  r.z = z;
  r.usual = usual;
  return f;
}

// A logit's weight in a share's units.
SP_DEVINL float share_weight(float x, float c, const Share& r) {
  if (!r.usual) return weight(x, r.m, c);
  return x > -INFINITY ? ex2(__fmaf_rn(x, c, -r.z)) : 0.f;
}

// A share's sum in units of exp(m / t).
SP_DEVINL float share_sum(float c, const Share& r) {
  return r.usual && r.m > -INFINITY ? r.s * ex2(__fmaf_rn(-r.m, c, r.z)) : r.s;
}

// The largest logit of a batch.
template <bool F32>
SP_DEVINL float batch_top(const uint4 (&u)[VF_LOADS]) {
  float lm = -INFINITY;
#pragma unroll
  for (int k = 0; k < VF_LOADS; ++k) lm = fmaxf(lm, Chunk<F32>::top(u[k]));
  return lm;
}

// A batch of loads (its first at c); again(k) is its k-th once more.
template <bool F32, typename Again>
SP_DEVINL void add_batch(const uint4 (&u)[VF_LOADS], int c, float cc, Share& r, Again again) {
  using K = Chunk<F32>;
  const float lm = batch_top<F32>(u);
  if (lm > r.m) {
    raise_to(lm, cc, r);
    r.first = c;
  }
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < VF_LOADS; ++k)
#pragma unroll
    for (int i = 0; i < K::N; ++i) sum[i & 1] += ex2(__fmaf_rn(K::at(u[k], i), cc, -r.z));
  float ts = sum[0] + sum[1];
  if (!(ts < INFINITY) || !r.usual) {  // a NaN among them, or no ordinary maximum
    ts = 0.f;
#pragma unroll 1
    for (int k = 0; k < VF_LOADS && lm > -INFINITY; ++k) {
      const uint4 v = again(k);
#pragma unroll
      for (int i = 0; i < K::N; ++i) ts += share_weight(K::at(v, i), cc, r);
    }
  }
  r.s += ts;
}

// One logit that lies beside the batches; what the share had counts `the result` as much, -1: it has no weight.
SP_DEVINL float add_one(float x, float c, Share& r) {
  if (!(x > -INFINITY)) return -1.f;
  float f = 1.f;
  if (x > r.m) {
    f = raise_to(x, c, r);
    r.first = -1;
  }
  r.s += share_weight(x, c, r);
  return f;
}

// A thread's share of a slice.  Its loads go through shared memory of its own (VF_RING batches of VF_LOADS), so no thread
// waits for another; `meanwhile` runs while the first are on their way.  Batches that lie whole in the slice are loaded and
// read without a check of every piece.
template <bool F32, typename Meanwhile>
SP_DEVINL Share sum_slice(const Slice<F32>& sl, float cc, uint4* ring, Meanwhile meanwhile) {
  using K = Chunk<F32>;
  constexpr int STEP = VF_NT * VF_LOADS;
  Share r{-INFINITY, -INFINITY, 0.f, -1, 0.f, 1.f, -1, true, false};
  const uint4* src = sl.src() + threadIdx.x;
  uint4* own = ring + threadIdx.x;
  const int left = sl.chunks - threadIdx.x;  // pieces from this thread's first on
  auto copy = [&](uint4* to, const uint4* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
  };
  auto load = [&](int c0, int place) {  // (c0: the batch's first piece, the same for all threads)
    const uint4* from = src + c0;
    uint4* to = own + place * STEP;
    if (c0 + STEP <= sl.chunks) {
#pragma unroll
      for (int k = 0; k < VF_LOADS; ++k) copy(to + k * VF_NT, from + k * VF_NT);
    } else {
#pragma unroll
      for (int k = 0; k < VF_LOADS; ++k)
        if (c0 + k * VF_NT < left) copy(to + k * VF_NT, from + k * VF_NT);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < VF_RING - 1; ++i) load(i * STEP, i);
  const int beside = sl.beside();
  const float mine = beside >= 0 ? K::one(sl.base, beside) : -INFINITY;
  meanwhile();
  for (int c0 = 0, place = 0; c0 < sl.chunks; c0 += STEP) {
    load(c0 + (VF_RING - 1) * STEP, place == 0 ? VF_RING - 1 : place - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(VF_RING - 1) : "memory");
    const uint4* at = own + place * STEP;
    const bool whole = c0 + STEP <= sl.chunks;
    auto piece = [&](int k) {
      return whole || c0 + k * VF_NT < left ? at[k * VF_NT] : make_uint4(K::kNone, K::kNone, K::kNone, K::kNone);
    };
    uint4 u[VF_LOADS];
    if (whole) {
#pragma unroll
      for (int k = 0; k < VF_LOADS; ++k) u[k] = at[k * VF_NT];
    } else {
#pragma unroll
      for (int k = 0; k < VF_LOADS; ++k) u[k] = piece(k);
    }
    add_batch<F32>(u, c0 + threadIdx.x, cc, r, piece);
    if (++place == VF_RING) place = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  add_one(mine, cc, r);
  return r;
}

// The same with the race, four tokens and their noise at a time: batches of vr_loads() fours, vr_ring() of them (48 KB).
template <bool F32>
constexpr int vr_loads() { return F32 ? 2 : 4; }
template <bool F32>
constexpr int vr_ring() { return F32 ? 3 : 2; }
template <bool F32>
constexpr int vr_bytes() { return vr_ring<F32>() * vr_loads<F32>() * VF_NT * (16 + Four<F32>::kBytes); }

template <bool F32>
SP_DEVINL Share scan_race(const Slice<F32>& sl, float cc, uint4* ring, const float* noise) {
  using K = Chunk<F32>;
  using Q = Four<F32>;
  using T = typename Q::T;
  constexpr int LOADS = vr_loads<F32>(), RING = vr_ring<F32>(), STEP = VF_NT * LOADS;
  Share r{-INFINITY, -INFINITY, 0.f, -1, 0.f, 1.f, -1, true, false};
  float best = 0.f;  // (in r's units)
  const int tid = threadIdx.x, left = sl.chunks * (K::N / 4) - tid;  // fours from this thread's first on
  const T* src = reinterpret_cast<const T*>(sl.src()) + tid;
  const float* e = noise + sl.c0 + tid * 4;
  const bool e16 = (reinterpret_cast<uintptr_t>(e) & 15) == 0;
  uint4* own_n = ring + tid;
  T* own_x = reinterpret_cast<T*>(ring + RING * STEP) + tid;
  auto load = [&](int c0, int place) {
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int c = c0 + k * VF_NT, to = place * STEP + k * VF_NT;
      if (c >= left) continue;
      asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(own_x + to)), "l"(src + c), "n"(Q::kBytes) : "memory");
      const float* from = e + (size_t)c * 4;
      const uint32_t at = smem_u32(own_n + to);
      if (e16) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 4 * i), "l"(from + i) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < RING - 1; ++i) load(i * STEP, i);
  const int beside = sl.beside();
  const float mine = beside >= 0 ? K::one(sl.base, beside) : -INFINITY;
  for (int c0 = 0, place = 0; c0 < sl.chunks * (K::N / 4); c0 += STEP) {
    load(c0 + (RING - 1) * STEP, place == 0 ? RING - 1 : place - 1);
    asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory");
    T x[LOADS];
    uint4 n[LOADS];
    float lm = -INFINITY;
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      x[k] = c0 + k * VF_NT < left ? own_x[place * STEP + k * VF_NT] : Q::none();
      n[k] = own_n[place * STEP + k * VF_NT];  // (of fours that are not there too: they have no weight)
      lm = fmaxf(lm, Q::top(x[k]));
    }
    if (lm > r.m) best *= raise_to(lm, cc, r);
    float sum = 0.f;
    auto weigh = [&](auto weight_of) {
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        float score[4], top = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = weight_of(Q::at(x[k], i));
          sum += w;
          // (noise 0: infinity, or NaN for w = 0, which is no candidate)
          score[i] = w * rcp(__uint_as_float(i == 0 ? n[k].x : i == 1 ? n[k].y : i == 2 ? n[k].z : n[k].w));
          top = fmaxf(top, score[i]);  // (passes over NaN)
        }
        if (top > best) {
          r.infinite |= top == INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (score[i] > best) {
              best = score[i];
              r.at = sl.c0 + (c0 + k * VF_NT + tid) * 4 + i;
            }
        }
      }
    };
    if (r.usual) weigh([&](float v) { return ex2(__fmaf_rn(v, cc, -r.z)); });
    if (!r.usual) weigh([&](float v) { return share_weight(v, cc, r); });
    if (!(sum < INFINITY)) {  // a NaN among them, or no weight yet
      sum = 0.f;
#pragma unroll 1
      for (int k = 0; k < LOADS && lm > -INFINITY; ++k) {
        const T v = c0 + k * VF_NT < left ? own_x[place * STEP + k * VF_NT] : Q::none();
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += share_weight(Q::at(v, i), cc, r);
      }
    }
    r.s += sum;
    if (++place == RING) place = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  const float f = add_one(mine, cc, r);
  if (f >= 0.f) {
    best *= f;
    const float score = share_weight(mine, cc, r) * rcp(__ldg(noise + beside));
    r.infinite |= score == INFINITY;
    if (score > best || (score == best && beside < r.at)) r.at = beside;
  }
  if (r.at >= 0) {
    r.x = K::one(sl.base, r.at);
    r.e = __ldg(noise + r.at);
  }
  return r;
}

// Joins the CTA's shares: the slice's maximum in every thread, its sum (and a greedy sequence's first token with the
// maximum, of `first` of every thread) in thread 0.
template <typename First>
SP_DEVINL RowPart join_cta(float m, float s, float c, bool greedy, First first) {
  __shared__ float2 ms_s[VF_WARPS];
  __shared__ int at_s[VF_WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float mw = warp_max(m);
  const float sw = warp_sum(m > -INFINITY ? (m == mw ? s : s * ex2((m - mw) * c)) : 0.f);
  if (lane == 0) ms_s[warp] = make_float2(mw, sw);
  __syncthreads();
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int w = 0; w < VF_WARPS; ++w) top = fmaxf(top, ms_s[w].x);
  int at = 0x7fffffff;
  if (greedy) {
    if (m == top && m > -INFINITY) at = first(top);
    at = __reduce_min_sync(0xffffffffu, at);
    if (lane == 0) at_s[warp] = at;
    __syncthreads();
  }
  if (threadIdx.x == 0)
    for (int w = 0; w < VF_WARPS; ++w) {
      if (ms_s[w].x > -INFINITY) sum += ms_s[w].x == top ? ms_s[w].y : ms_s[w].y * ex2((ms_s[w].x - top) * c);
      if (greedy) at = min(at, at_s[w]);
    }
  return RowPart{top, sum, at, 0.f};
}

// A row as its decision and its race need it.
struct __align__(16) Row {
  float mp, sp, mq, sq;  // maxima and sums of the target's and the draft's logits
  float xd;              // the target's logit of the draft
  int at;                // greedy: the first token with the maximum
  int stays;             // the draft does
  int unused;
};

// What a call leaves in its workspace between kernels.
struct VerifyWork {
  RowPart* part;  // [T_cap][2][slices]
  Row* rows;      // [T_cap], ordered calls only
  int* count;     // [T_cap] slices of a row that are done, from kUnset on (ordered calls)
  int* end;       // [B] the first row of a sequence known to reject its draft, kUnset: none (ordered calls)
};
constexpr int kUnset = 0x7f7f7f7f;

// A row's slices, joined by a warp; whether its draft stays.  Every lane has the result.  In steps of 2^-24: the weight of a token
// 2^-z times as likely as the likeliest is off by less than 2.5 z + 4 (c by 1.5, x - m and its product by 1 each, times z ln 2;
// the exponential by 4), a sum by 2^-17.5 = 91 (its terms' mean z is below log2 V; adding up 2^-19), so what is compared by less
// than 200 + 5 z.
SP_DEVINL Row decide(const VerifyArgs& a, const Seq& q, int j, const RowPart* part, int slices) {
  const int lane = threadIdx.x & 31, row = q.row0 + j;
  const bool last = j == q.n - 1, with_q = a.draft_logits && !q.greedy && !last;
  const RowPart none{-INFINITY, 0.f, 0x7fffffff, -INFINITY};
  RowPart p = none, r = none;
  if (lane < slices) {
    const int4* from = reinterpret_cast<const int4*>(part + (size_t)row * 2 * slices) + lane;
    const int4 v = __ldcg(from);
    p = RowPart{__int_as_float(v.x), __int_as_float(v.y), v.z, __int_as_float(v.w)};
    if (with_q) {
      const int4 w = __ldcg(from + slices);
      r = RowPart{__int_as_float(w.x), __int_as_float(w.y), w.z, __int_as_float(w.w)};
    }
  }
  const int d = last ? -1 : __ldg(a.draft + row);
  const float u = last || q.greedy ? 0.f : __ldg(a.u + row);
  Row o;
  o.mp = warp_max(p.m);
  o.mq = warp_max(r.m);
  o.sp = warp_sum(p.m > -INFINITY ? (p.m == o.mp ? p.s : p.s * ex2((p.m - o.mp) * q.c)) : 0.f);
  o.sq = warp_sum(r.m > -INFINITY ? (r.m == o.mq ? r.s : r.s * ex2((r.m - o.mq) * q.c)) : 0.f);
  o.at = __reduce_min_sync(0xffffffffu, p.m == o.mp ? p.at : 0x7fffffff);
  o.xd = __shfl_sync(0xffffffffu, p.xd, 0);
  const float yd = __shfl_sync(0xffffffffu, r.xd, 0);
  o.unused = 0;
  if (last) o.stays = 0;
  else if (q.greedy) o.stays = d == o.at && d >= 0 && d < a.V;  // (at: no token in a row without weight)
  else {  // u q(d) < p(d), the sums multiplied out; without weight anywhere p is 0
    const float pd = o.sp > 0.f ? weight(o.xd, o.mp, q.c) : 0.f;
    const float qd = !with_q ? 1.f : o.sq > 0.f ? weight(yd, o.mq, q.c) : 0.f;
    o.stays = pd > 0.f && u * qd * o.sp < pd * (with_q && o.sq > 0.f ? o.sq : 1.f);
  }
  return o;
}

// Sums of every row, a slice to a CTA: blockIdx.x = which * slices + slice (which: 0 the target's, 1 the draft's),
// blockIdx.z the row of the sequence.  ORDERED: the CTA that ends a row decides about its draft, and rows behind one that
// rejects are passed over.  CTAs start in the order of their numbers, so in a call of many waves most of those rows
// are never read; nothing waits, and what is read needlessly has no effect.
// 256 sequences of 5 drafts (2.1 stay), 152,064 bf16 logits: 470 of 856 MB read in 92 us, 5.1 TB/s; all of them, where every
// draft stays, in 141, 6.1 TB/s.  A CTA of a row that is passed over costs the call 1.7 ns, a slice's beginning and end some 5 us
// that three other CTAs of the SM fill; issue 57%, about 9 instructions a logit.  (CTAs that stay, fetch slices from a
// counter and keep bulk copies in flight: 137 to 200.)
template <bool F32, bool ORDERED>
__global__ void __launch_bounds__(VF_NT, 4) verify_sums_kernel(const VerifyArgs a, int slices, int slice, VerifyWork work) {
  extern __shared__ uint4 ring[];
  __shared__ int last_s;
  pdl_wait();
  const int which = blockIdx.x / slices, sl = blockIdx.x % slices, b = blockIdx.y, j = blockIdx.z;
  if (a.clear_err && a.err && blockIdx.x + b + j == 0 && threadIdx.x == 0) *a.err = 0;
  const int ended = ORDERED ? ld_relaxed_gpu(work.end + b) : kUnset;
  const Seq q = sequence(a, b);
  const bool last = j == q.n - 1;
  if (j >= q.n || (which == 1 && (q.greedy || last))) return;
  if (ORDERED && __syncthreads_or(ended < j)) return;  // (the end moves while threads look at it: the CTA goes on, or ends, as one)
  const int row = q.row0 + j;
  const char* base = static_cast<const char*>(which ? a.draft_logits : a.logits) +
                     row * (which ? a.ld_draft : a.ld) * (F32 ? 4 : 2);
  float xd = -INFINITY;
  const int v0 = min(sl * slice, a.V), v1 = min(v0 + slice, a.V);
  const Slice<F32> s(base, v0, v1);
  const Share t = sum_slice<F32>(s, q.c, ring, [&]() {
    if (sl == 0 && threadIdx.x == 0 && !last) {
      const int d = __ldg(a.draft + row);
      if (d >= 0 && d < a.V) xd = Chunk<F32>::one(base, d);
    }
  });
  pdl_trigger();
  RowPart r = join_cta(t.m, share_sum(q.c, t), q.c, q.greedy, [&](float top) { return s.first_of(top, t.first); });
  r.xd = xd;
  if (threadIdx.x == 0) work.part[((size_t)row * 2 + which) * slices + sl] = r;
  if (ORDERED) {
    if (threadIdx.x == 0) {
      __threadfence();
      const int all = slices * (a.draft_logits && !q.greedy && !last ? 2 : 1);
      const bool done = atomicAdd(work.count + row, 1) == kUnset + all - 1;
      if (done) __threadfence();  // (by the thread that counted; the barrier hands the other slices' parts on to its warp)
      last_s = done;
    }
    __syncthreads();
    if (last_s && threadIdx.x < 32) {
      const Row o = decide(a, q, j, work.part, slices);
      if (threadIdx.x == 0) {
        work.rows[row] = o;
        __threadfence();
        if (!o.stays) atomicMin(work.end + b, j);
      }
    }
  }
}

SP_DEVINL float log_prob(float x, float m, float s, float t) {
  if (!(x > -INFINITY) || !(x <= m)) return -INFINITY;
  return (x == m ? 0.f : __fdividef(x - m, t)) - logf(s);  // (both at most 0: nothing cancels)
}

// A race's score and token as one key that sorts by (score, lower token first); scores are above 0, 0: none.
SP_DEVINL unsigned long long race_key(float score, int v) {
  return ((unsigned long long)__float_as_uint(score) << 32) | (uint32_t)~v;
}

// The row where a sequence ends, as its race needs it.
template <bool F32>
struct Race {
  using K = Chunk<F32>;
  static constexpr int E4 = K::N / 4;
  const void *p, *q;  // q NULL: nothing is taken off
  const float* e;
  float mp, sp, mq, sq, c;  // maxima and sums
  int out;                  // a token whose probability is taken off whole (a draft without a distribution), -1: none

  // Scores are in units of the target's (a race does not ask for them): of exp2(z), z next to m c, or of exp(m / t).  q is
  // brought to the same by k.
  bool usual;
  float zp, zq, k;
  SP_DEVINL void prepare() {
    if (q && !(sq > 0.f)) q = nullptr;  // a draft without weight takes nothing off
    usual = ordinary(mp * c) && (!q || ordinary(mq * c));
    zp = rintf(mp * c);
    zq = rintf(mq * c);
    k = !q ? 0.f : usual ? -(sp * ex2(__fmaf_rn(mp, c, -zp))) / (sq * ex2(__fmaf_rn(mq, c, -zq))) : -sp / sq;
  }
  // The best of tokens v0 .. v1 - 1, one at a time, for this thread of the CTA.
  SP_DEVINL unsigned long long slowly(int v0, int v1, int step) const {
    float best = 0.f;
    int at = 0;
#pragma unroll 4
    for (int v = v0; v < v1; v += step) {
      const float x = K::one(p, v);
      float r = usual ? ex2(__fmaf_rn(x, c, -zp)) : weight(x, mp, c);
      if (q) {
        const float y = K::one(q, v);
        r = fmaxf(__fmaf_rn(k, usual ? ex2(__fmaf_rn(fmaxf(y, -INFINITY), c, -zq)) : weight(y, mq, c), r), 0.f);
      }
      const float score = r * rcp(__ldg(e + v));  // (noise 0: infinity, or NaN for r = 0, which is no candidate)
      if (score > best && v != out) {
        best = score;
        at = v;
      }
    }
    return best > 0.f ? race_key(best, at) : 0ull;
  }
  struct Piece {
    uint4 x, y;
    float4 n[E4];
  };
  template <bool DRAFTED>
  SP_DEVINL void pieces(const Slice<F32>& s, float& best, int& at) const {
    const uint4* ps = s.src();
    const uint4* qs = reinterpret_cast<const uint4*>(static_cast<const char*>(q) + (size_t)s.c0 * Slice<F32>::esz);
    const float* es = e + s.c0;
    const bool e16 = (reinterpret_cast<uintptr_t>(es) & 15) == 0;
    const float c_ = c;
    auto load = [&](Piece& g, int c) {
      g.x = __ldg(ps + c);
      if (DRAFTED) g.y = __ldg(qs + c);
#pragma unroll
      for (int k = 0; k < E4; ++k) {
        const float* f = es + (c * E4 + k) * 4;
        g.n[k] = e16 ? __ldcs(reinterpret_cast<const float4*>(f)) : make_float4(__ldg(f), __ldg(f + 1), __ldg(f + 2), __ldg(f + 3));
      }
    };
    auto take = [&](const Piece& g, int c) {
      float score[K::N], top = 0.f;
      const uint4 y = DRAFTED ? without_nan<F32>(g.y) : g.x;  // (a NaN of the target's makes no score)
#pragma unroll
      for (int i = 0; i < K::N; ++i) {
        float r = ex2(__fmaf_rn(K::at(g.x, i), c_, -zp));
        if (DRAFTED) r = fmaxf(__fmaf_rn(k, ex2(__fmaf_rn(K::at(y, i), c_, -zq)), r), 0.f);
        const float4& f = g.n[i / 4];
        score[i] = r * rcp(i % 4 == 0 ? f.x : i % 4 == 1 ? f.y : i % 4 == 2 ? f.z : f.w);
        top = fmaxf(top, score[i]);  // (passes over NaN)
      }
      if (top > best) {
        const int v = s.c0 + c * K::N;
#pragma unroll
        for (int i = 0; i < K::N; ++i)
          if (score[i] > best && v + i != out) {
            best = score[i];
            at = v + i;
          }
      }
    };
    for (int c = threadIdx.x; c < s.chunks; c += 2 * VF_NT) {
      Piece g, h;
      load(g, c);
      const bool two = c + VF_NT < s.chunks;
      if (two) load(h, c + VF_NT);
      take(g, c);
      if (two) take(h, c + VF_NT);
    }
  }
  // The best of tokens v0 .. v1 - 1 for this thread of the CTA.
  SP_DEVINL unsigned long long run(int v0, int v1) const {
    const Slice<F32> s(p, v0, v1);
    if (!(sp > 0.f)) return 0ull;
    // rows that have no 16-byte pieces in common, maxima that are not ordinary: token by token
    if (!usual || (q && ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) != 0))
      return slowly(v0 + threadIdx.x, v1, VF_NT);
    unsigned long long key = s.beside() >= 0 ? slowly(s.beside(), s.beside() + 1, 1) : 0ull;
    float best = 0.f;
    int at = 0;
    if (q) pieces<true>(s, best, at);
    else pieces<false>(s, best, at);
    return best > 0.f ? max(key, race_key(best, at)) : key;
  }
};

// The largest of the CTA's keys, in every thread (callers branch on it around barriers).
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

// A cluster barrier in two halves: that every CTA runs is known long before anything is written to another's memory.
SP_DEVINL void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
SP_DEVINL void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// What a sequence is left with: a row that is not there.
SP_DEVINL void no_rows(const VerifyArgs& a, int b, bool wrong) {
  for (int j = threadIdx.x; j < a.max_rows; j += VF_NT) {
    a.token[(size_t)b * a.max_rows + j] = -1;
    if (a.logp) a.logp[(size_t)b * a.max_rows + j] = 0.f;
  }
  if (threadIdx.x == 0) {
    if (wrong) set_error(a.err, SP_DEVERR_INDEX);
    a.n_accept[b] = -1;
  }
}

// A cluster per sequence: every CTA finds the row where it ends (ORDERED: is told), each races over its slice of it.
// Bound by reading p, q and the noise, and by the chain sums -> decision -> race -> two exchanges (3 to 4 us of a small call's
// 6): 256 sequences of 152,064 bf16 logits, 295 MB, about 60 us behind the sums.  (Reading only the noise, and logits where a
// segment's maximum and the least noise of 8 tokens let one win: 88, a dependent load for every fourth warp.)
template <bool F32, bool ORDERED>
__global__ void __launch_bounds__(VF_NT) verify_end_kernel(const VerifyArgs a, int slices, VerifyWork work) {
  using K = Chunk<F32>;
  __shared__ Row row_s[VF_WARPS];
  __shared__ unsigned long long key_s[VF_WARPS], cluster_s[VF_CLUSTER];
  // Before the wait: what no kernel of this call writes.  (The sums wait for whatever ran before them ahead of their
  // trigger, so it is over.)
  const int C = gridDim.x, rank = blockIdx.x, b = gridDim.y - 1 - blockIdx.y,  // (the rows read last lie in L2)
            tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const Seq q = sequence(a, b);
  const int per = (((a.V + C - 1) / C) + 7) & ~7, v0 = min(rank * per, a.V), v1 = min(v0 + per, a.V);
  if (q.n > 0 && !q.greedy)
    for (int v = v0 + tid * 32; v < v1; v += VF_NT * 32)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(a.noise + (size_t)b * a.ld_noise + v));
  if (C > 1) cluster_arrive();
  pdl_wait();
  pdl_trigger();
  if (q.n <= 0) {
    if (rank == 0) no_rows(a, b, q.n < 0);
    if (C > 1) cluster_wait();
    return;
  }
  int* token = a.token + (size_t)b * a.max_rows;
  float* logp = a.logp ? a.logp + (size_t)b * a.max_rows : nullptr;
  auto logits = [&](int j) { return static_cast<const char*>(a.logits) + (q.row0 + j) * a.ld * (F32 ? 4 : 2); };
  auto stays = [&](int j, const Row& r) {  // a draft that stays, written by a warp's first lane
    const int d = __ldg(a.draft + q.row0 + j);
    if (d < 0 || d >= a.V) set_error(a.err, SP_DEVERR_INDEX);
    token[j] = d;
    if (logp) logp[j] = log_prob(r.xd, r.mp, r.sp, q.t);
  };
  int end = -1;
  Row r;
  if (ORDERED) {
    end = __ldcg(work.end + b);
    if (end >= q.n) {  // (sequences whose offsets overlap)
      if (rank == 0) no_rows(a, b, true);
      if (C > 1) cluster_wait();
      return;
    }
    auto load = [&](int j) {
      const int4* from = reinterpret_cast<const int4*>(work.rows + q.row0 + j);
      const int4 x = __ldcg(from), y = __ldcg(from + 1);
      return Row{__int_as_float(x.x), __int_as_float(x.y), __int_as_float(x.z), __int_as_float(x.w), __int_as_float(y.x),
                 y.y, y.z, 0};
    };
    r = load(end);
    if (rank == C - 1)
      for (int j = tid; j < end; j += VF_NT) stays(j, load(j));
  } else {
    for (int j0 = 0; end < 0; j0 += VF_WARPS) {  // a warp to a row
      const int j = j0 + warp;
      Row mine;
      mine.stays = 1;
      if (j < q.n) mine = decide(a, q, j, work.part, slices);
      if (lane == 0) row_s[warp] = mine;
      __syncthreads();
      const unsigned int out = __ballot_sync(0xffffffffu, lane < VF_WARPS && !row_s[lane % VF_WARPS].stays);
      const int w = out ? __ffs(out) - 1 : VF_WARPS;
      if (out) {
        end = j0 + w;
        r = row_s[w];
      }
      if (rank == C - 1 && lane == 0 && j < q.n && warp < w) stays(j, mine);
      if (end < 0) __syncthreads();
    }
  }
  const bool drafted = end < q.n - 1;
  int d = -1;
  if (drafted) {
    d = __ldg(a.draft + q.row0 + end);
    if (rank == 0 && tid == 0 && (d < 0 || d >= a.V)) set_error(a.err, SP_DEVERR_INDEX);
  }
  if (rank == C - 1)
    for (int j = end + 1 + tid; j < a.max_rows; j += VF_NT) {
      token[j] = -1;
      if (logp) logp[j] = 0.f;
    }
  // (sequences whose offsets overlap can find another's sums: never a token that is not there)
  int next = r.mp > -INFINITY && r.at >= 0 && r.at < a.V ? r.at : -1;
  if (C > 1) cluster_wait();  // every CTA of the cluster runs
  if (!q.greedy) {
    Race<F32> race;
    race.p = logits(end);
    race.q = drafted && a.draft_logits
                 ? static_cast<const char*>(a.draft_logits) + (q.row0 + end) * a.ld_draft * (F32 ? 4 : 2)
                 : nullptr;
    race.e = a.noise + (size_t)b * a.ld_noise;
    race.mp = r.mp;
    race.sp = r.sp;
    race.mq = r.mq;
    race.sq = r.sq;
    race.c = q.c;
    race.out = a.draft_logits ? -1 : d;
    race.prepare();
    unsigned long long key = cta_max(race.run(v0, v1), key_s);
    if (C > 1) {
      if (tid == 0) {
        const uint32_t to = mapa_shared(smem_u32(&cluster_s[rank]), 0);
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(to), "l"(key) : "memory");
      }
      cluster_arrive();
      cluster_wait();
      if (rank != 0) return;
      for (int i = 0; i < C; ++i) key = max(key, cluster_s[i]);
    }
    if (key == 0 && drafted) {  // p and q are the same (or p is all at the draft): from p
      race.q = nullptr;
      race.out = -1;
      race.prepare();
      key = cta_max(race.run(0, a.V), key_s);
    }
    next = key != 0 ? (int)~(uint32_t)key : -1;
  }
  if (rank == 0 && tid == 0) {
    a.n_accept[b] = end;
    token[end] = next;
    if (logp) logp[end] = next >= 0 ? log_prob(K::one(logits(end), next), r.mp, r.sp, q.t) : -INFINITY;
  }
}

// Without drafts: a cluster per sequence, the sums and the race in one pass over its row.  A thread keeps the best of its
// scores next to its own maximum.  What has no weight next to the row's is dropped when shares are joined; where that may have
// been an infinite score, or nothing is left, the first CTA races over the row again, next to its maximum.  64 rows of 32,000
// fp32 logits, 16 MB: 8 us, a chain of temperature -> loads -> join -> exchange; 256 of 152,064 bf16, 233 MB: 44 us (5.3 TB/s; 59
// with 16 bytes of logits and twice 16 of noise to a thread, which split every line of the noise between two loads).
template <bool F32>
__global__ void __launch_bounds__(VF_NT) verify_sample_kernel(const VerifyArgs a) {
  using K = Chunk<F32>;
  struct __align__(16) Best {
    float m, s, x, e;
    int at, greedy_at, infinite, unused;
  };
  extern __shared__ uint4 ring[];
  __shared__ Best best_s[VF_CLUSTER], mine_s;
  __shared__ unsigned long long key_s[VF_WARPS];
  const int C = gridDim.x, rank = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31;
  if (C > 1) cluster_arrive();
  pdl_wait();
  pdl_trigger();
  const Seq q = sequence(a, b);
  if (a.clear_err && a.err && rank + b == 0 && tid == 0 && !a.cu_rows) *a.err = 0;
  if (q.n <= 0) {
    if (rank == 0) no_rows(a, b, q.n < 0);
    if (C > 1) cluster_wait();
    return;
  }
  const char* base = static_cast<const char*>(a.logits) + q.row0 * a.ld * (F32 ? 4 : 2);
  const float* noise = q.greedy ? nullptr : a.noise + (size_t)b * a.ld_noise;
  const int per = (((a.V + C - 1) / C) + 7) & ~7;
  const Slice<F32> s(base, min(rank * per, a.V), min((rank + 1) * per, a.V));
  const Share t = q.greedy ? sum_slice<F32>(s, q.c, ring, []() {}) : scan_race<F32>(s, q.c, ring, noise);
  const RowPart r = join_cta(t.m, share_sum(q.c, t), q.c, q.greedy, [&](float top) { return s.first_of(top, t.first); });
  const float score = t.at >= 0 ? weight(t.x, r.m, q.c) * rcp(t.e) : 0.f;
  const unsigned long long own = score > 0.f ? race_key(score, t.at) : 0ull, key = cta_max(own, key_s);
  if (tid == 0) mine_s = Best{r.m, r.s, 0.f, 1.f, -1, r.at, 0, 0};
  __syncthreads();
  if (own != 0 && own == key) {
    mine_s.x = t.x;
    mine_s.e = t.e;
    mine_s.at = t.at;
  }
  if (t.infinite) mine_s.infinite = 1;
  __syncthreads();
  if (C > 1) {
    cluster_wait();  // every CTA of the cluster runs
    if (tid < 8) {
      const uint32_t to = mapa_shared(smem_u32(reinterpret_cast<uint32_t*>(&best_s[rank]) + tid), 0);
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(reinterpret_cast<uint32_t*>(&mine_s)[tid]) : "memory");
    }
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;
  } else {
    if (tid == 0) best_s[0] = mine_s;
    __syncthreads();
  }
  // a lane to a CTA's best, the same in every warp
  const bool in = lane < C;
  const Best o = best_s[in ? lane : 0];
  const float m = warp_max(in ? o.m : -INFINITY);
  const bool some = in && o.m > -INFINITY;
  const float sum = warp_sum(!some ? 0.f : o.m == m ? o.s : o.s * ex2((o.m - m) * q.c));
  unsigned long long k = 0;
  if (q.greedy) {
    if (some && o.m == m) k = race_key(1.f, o.greedy_at);
  } else if (some && o.at >= 0) {
    const float sc = weight(o.x, m, q.c) * rcp(o.e);
    if (sc > 0.f) k = race_key(sc, o.at);
  }
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  const unsigned int won = __ballot_sync(0xffffffffu, k != 0 && k == (((unsigned long long)hi << 32) | lo));
  int next = won ? (int)~lo : -1;
  float x = __shfl_sync(0xffffffffu, q.greedy ? m : o.x, won ? __ffs(won) - 1 : 0);
  if (!q.greedy && m > -INFINITY && (!won || __any_sync(0xffffffffu, in && o.infinite))) {
    Race<F32> race;
    race.p = base;
    race.q = nullptr;
    race.e = noise;
    race.mp = m;
    race.sp = sum;
    race.mq = race.sq = 0.f;
    race.c = q.c;
    race.out = -1;
    race.prepare();
    const unsigned long long best = cta_max(race.run(0, a.V), key_s);
    next = best != 0 ? (int)~(uint32_t)best : -1;
    if (next >= 0) x = K::one(base, next);
  }
  if (tid == 0) {
    a.n_accept[b] = 0;
    a.token[b] = next;
    if (a.logp) a.logp[b] = next >= 0 ? log_prob(x, m, sum, q.t) : -INFINITY;
  }
}

}  // namespace

// Logits of a slice: whole batches, where it has some (slices that each end in a part of a batch, of three 7 instead of
// 6.2, cost their sums a tenth).
static int slice_of(int V, int slices, bool f32) {
  const int batch = VF_NT * VF_LOADS * (f32 ? 4 : 8), least = (V + slices - 1) / slices;
  return least > batch / 2 ? (least + batch - 1) / batch * batch : (least + 7) & ~7;
}

static size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

static int verify_slots() { return device_sm_count() * 4; }

size_t verify_bytes(int T_cap, int B, int V) {
  const size_t T = (size_t)T_cap;
  return align256(2 * verify_parts(T_cap, V, verify_slots()) * sizeof(RowPart)) + align256(T * sizeof(Row)) + align256((T + B) * 4);
}

template <typename Kernel, typename... Args>
static cudaError_t launch_clusters(Kernel* k, int C, int B, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C, B);
  cfg.blockDim = dim3(VF_NT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = C;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

cudaError_t verify_launch(const VerifyArgs& a, void* ws, cudaStream_t st) {
  const int sms = device_sm_count();
  const double bytes = (double)a.T_cap * a.V * (a.logits_f32 ? 4 : 2);
  const int most = std::min(VF_CLUSTER, (a.V + 4095) / 4096);  // CTAs of a sequence: 4,096 logits for each at least
  cudaError_t r;
  if (a.max_rows == 1) {
    if (a.cu_rows && a.clear_err && a.err) {
      r = cudaMemsetAsync(a.err, 0, 4, st);
      if (r != cudaSuccess) return r;
    }
    prof_begin_launch(st);
    // two CTAs per SM (128 sequences of 152,064 bf16 logits by two CTAs 27 us, by four 29; 256 by one 44, by two 50)
    const int C = std::max(1, std::min(most, sms * 2 / a.B));
    static std::atomic<unsigned long long> allowed[2];
    auto* k = a.logits_f32 ? verify_sample_kernel<true> : verify_sample_kernel<false>;
    const int ring = std::max(VF_RING_BYTES, a.logits_f32 ? vr_bytes<true>() : vr_bytes<false>());
    r = allow_smem(k, ring, allowed[a.logits_f32]);
    if (r == cudaSuccess) r = launch_clusters(k, C, a.B, ring, st, a);
    prof_end_launch(st, SP_K_MISC, 0.0, bytes + (a.noise ? 4.0 * a.B * a.V : 0.0));
    return r;
  }
  const int sets = a.draft_logits ? 2 : 1;
  const Cut cut = verify_cut(a.T_cap, a.B, a.V, a.max_rows, sets == 2, a.logits_f32, verify_slots());
  const int slices = cut.slices, slice = slice_of(a.V, slices, a.logits_f32);
  const bool ordered = cut.ordered;
  char* base = static_cast<char*>(ws);
  VerifyWork w;
  w.part = reinterpret_cast<RowPart*>(base);
  base += align256((size_t)a.T_cap * 2 * slices * sizeof(RowPart));
  w.rows = reinterpret_cast<Row*>(base);
  base += align256((size_t)a.T_cap * sizeof(Row));
  w.count = reinterpret_cast<int*>(base);
  w.end = w.count + a.T_cap;
  if (ordered) {
    r = cudaMemsetAsync(w.count, 0x7f, ((size_t)a.T_cap + a.B) * 4, st);
    if (r != cudaSuccess) return r;
  }
  auto* sums = ordered ? (a.logits_f32 ? verify_sums_kernel<true, true> : verify_sums_kernel<false, true>)
                       : (a.logits_f32 ? verify_sums_kernel<true, false> : verify_sums_kernel<false, false>);
  static std::atomic<unsigned long long> allowed[2][2];
  r = allow_smem(sums, VF_RING_BYTES, allowed[ordered][a.logits_f32]);
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  r = launch_pdl(sums, dim3(slices * sets, a.B, a.max_rows), dim3(VF_NT), VF_RING_BYTES, st, a, slices, slice, w);
  prof_end_launch(st, SP_K_MISC, 0.0, bytes * sets);
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  auto* end = ordered ? (a.logits_f32 ? verify_end_kernel<true, true> : verify_end_kernel<false, true>)
                      : (a.logits_f32 ? verify_end_kernel<true, false> : verify_end_kernel<false, false>);
  // four CTAs per SM, and no more than 25,000 logits for one (256 sequences of 152,064 by six 152 us, by two 157, by
  // eight 158; of 20,000 fp32 by two 31, by six 38)
  const int C = std::max(1, std::min(most, std::max(sms * 4 / a.B, a.V / 25000)));
  r = launch_clusters(end, a.noise ? C : 1, a.B, 0, st, a, slices, w);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
