// The pages of a cache: which of them a sequence's table names, and how many table entries name each page.
// refs[p] is the number of entries that name page p; a page with 0 is free.  Sequences that share positions name the
// same pages; a page that two entries name is not written to, but copied first.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sp {

namespace {

// ------------------------------------------------------------------------- trim

constexpr int PT_NT = 256;

// Entries behind the page of a row's last position go back.  A thread per entry; atomics on counts commute.
__global__ void __launch_bounds__(PT_NT) pages_trim_kernel(const PagesArgs a) {
  pdl_wait();
  pdl_trigger();
  const int s = blockIdx.y, c = blockIdx.x * PT_NT + threadIdx.x;
  const int len = __ldg(a.lens + s);
  if (len < 0 || len > ((long long)a.max_pages << a.page_shift)) {
    if (c == 0) set_error(a.err, SP_DEVERR_INDEX);
    return;
  }
  if (c >= a.max_pages || c < (len + (1 << a.page_shift) - 1) >> a.page_shift) return;
  int* e = a.table + (size_t)s * a.max_pages + c;
  const int page = *e;
  if (page < 0) return;
  if (page < a.n_pages) atomicSub(a.refs + page, 1);
  else set_error(a.err, SP_DEVERR_INDEX);
  *e = -1;
}

// ------------------------------------------------------------------------- fork

constexpr int PF_NT = 512, PF_CTAS = 8;
constexpr int PF_COLS = 8;  // table columns at once

// A row's new entries are its parent's of the same columns, so a CTA needs the old entries of all rows in its columns and
// no others.  One cluster: the lengths change when all of its CTAs have read them.
__global__ void __launch_bounds__(PF_NT) pages_fork_kernel(const PagesArgs a, const int* __restrict__ parent) {
  extern __shared__ int fork_s[];  // [S] old lengths, [S][PF_COLS] old entries
  int* len_s = fork_s;
  int* old_s = fork_s + a.S;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, n = a.S * PF_COLS;
  for (int s = tid; s < a.S; s += PF_NT) len_s[s] = a.lens[s];
  __syncthreads();
  const long long most = (long long)a.max_pages << a.page_shift;
  // the row that row s continues, itself where it stays
  auto from = [&](int s) {
    const int p = __ldg(parent + s);
    if (p == -1) return s;
    if (p < 0 || p >= a.S || len_s[p] < 0 || len_s[p] > most) {
      set_error(a.err, SP_DEVERR_INDEX);
      return s;
    }
    return p;
  };
  for (int c0 = blockIdx.x * PF_COLS; c0 < a.max_pages; c0 += gridDim.x * PF_COLS) {
    for (int i = tid; i < n; i += PF_NT) {
      const int c = c0 + i % PF_COLS;
      old_s[i] = c < a.max_pages ? a.table[(size_t)(i / PF_COLS) * a.max_pages + c] : -1;
    }
    __syncthreads();
    for (int i = tid; i < n; i += PF_NT) {
      const int s = i / PF_COLS, c = c0 + i % PF_COLS;
      if (c >= a.max_pages) continue;
      const int p = from(s);
      if (p == s) continue;
      const int old = old_s[i];
      int now = c < (len_s[p] + (1 << a.page_shift) - 1) >> a.page_shift ? old_s[p * PF_COLS + i % PF_COLS] : -1;
      if (now >= a.n_pages || old >= a.n_pages) set_error(a.err, SP_DEVERR_INDEX);
      if (now >= a.n_pages || now < 0) now = -1;
      if (now == old) continue;
      if (now >= 0) atomicAdd(a.refs + now, 1);
      if (old >= 0 && old < a.n_pages) atomicSub(a.refs + old, 1);
      a.table[(size_t)s * a.max_pages + c] = now;
    }
    __syncthreads();
  }
  cluster_sync_all();
  if (blockIdx.x == 0)
    for (int s = tid; s < a.S; s += PF_NT) {
      const int p = from(s);
      if (p != s) a.lens[s] = len_s[p];
    }
}

// ------------------------------------------------------------------------- reserve, compact

constexpr int PP_NT = 1024, PP_WARPS = PP_NT / 32;

// What the plan leaves for the copies: the positions that move, row by row, and where they were.
struct PageMoves {
  int* start;    // [S + 1] moved positions before each row's
  int* old_len;  // [S]
  int* old;      // [S, max_pages] the entries that rows had: compact all of them; reserve those that are replaced (-1: none
                 // was there, -2: the entry stays)
  int* free;     // [S, max_pages] the free pages that the call takes, in order
};

// Exclusive prefix sums of v over the CTA's threads; total in every thread.
SP_DEVINL int cta_prefix(int v, int* warp_s, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();  // (warp_s has been read)
  if (lane == 31) warp_s[warp] = x;
  __syncthreads();
  int w = lane < PP_WARPS ? warp_s[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  total = __shfl_sync(0xffffffffu, w, PP_WARPS - 1);
  const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
  return x - v + (warp > 0 ? before : 0);
}

// Which free pages the rows take, in order of rows and places, and the tables and counts after it.  One CTA.
template <bool COMPACT>
__global__ void __launch_bounds__(PP_NT)
pages_plan_kernel(const PagesArgs a, const int* __restrict__ add, const int* __restrict__ keep, long long ld_keep, int keep_cap,
                  PageMoves mv) {
  extern __shared__ int plan_s[];  // [S] pages that a row needs, [S] pages before it, [S] positions that move
  __shared__ int warp_s[PP_WARPS];
  int *need_s = plan_s, *before_s = plan_s + a.S, *move_s = plan_s + 2 * a.S;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, S = a.S, shift = a.page_shift, page = 1 << shift;
  const long long most = (long long)a.max_pages << shift;
  // The places [lo, hi) of a row that may get pages, and the positions that it will have in them before any is added.
  auto places = [&](int s, int& lo, int& hi) {
    const int len = a.lens[s], n = __ldg(add + s);
    lo = hi = 0;
    if (COMPACT) {
      if (n == -1) return false;
      if (n < 0 || n > keep_cap || n > most || len < 0 || len > most) return false;
    } else {
      if (len < 0 || n < 0 || (long long)len + n > most) return false;
      if (n > 0) {
        lo = len >> shift;
        hi = (int)(((long long)len + n + page - 1) >> shift);
      }
    }
    return true;
  };
  for (int s = warp; s < S; s += PP_WARPS) {
    int lo, hi, need = 0, move = 0;
    const bool ok = places(s, lo, hi);
    const int* row = a.table + (size_t)s * a.max_pages;
    if (!ok) {
      if (lane == 0 && !(COMPACT && __ldg(add + s) == -1)) set_error(a.err, SP_DEVERR_INDEX);
    } else if (COMPACT) {
      const int n = __ldg(add + s);
      int first = n;  // the first position that moves
      for (int i0 = 0; i0 < n; i0 += 32) {
        const unsigned int other = __ballot_sync(0xffffffffu, i0 + lane < n && __ldg(keep + s * ld_keep + i0 + lane) != i0 + lane);
        if (other) {
          first = i0 + __ffs(other) - 1;
          break;
        }
      }
      const int pages = (n + page - 1) >> shift, stay = first == n ? pages : first >> shift;
      need = pages - stay;
      move = first == n ? 0 : n - (stay << shift);
    } else {
      for (int c = lo + lane; c < hi; c += 32) {
        const int e = row[c];
        const bool there = e >= 0 && e < a.n_pages;
        if (e >= a.n_pages) set_error(a.err, SP_DEVERR_INDEX);
        const bool shared = there && a.refs[e] > 1;
        need += !there || shared;
        mv.old[(size_t)s * a.max_pages + c] = shared ? e : there ? -2 : -1;
        if (c == lo && shared) move = a.lens[s] & (page - 1);
      }
      need = __reduce_add_sync(0xffffffffu, need);
      move = __reduce_add_sync(0xffffffffu, move);
    }
    if (lane == 0) {
      need_s[s] = need;
      move_s[s] = move;
    }
  }
  __syncthreads();
  int total = 0;
  for (int s0 = 0; s0 < S; s0 += PP_NT) {
    const int s = s0 + tid;
    int sum;
    const int before = total + cta_prefix(s < S ? need_s[s] : 0, warp_s, sum);
    if (s < S) before_s[s] = before;
    total += sum;
  }
  // the first `total` free pages, in order
  int found = 0;
  const int n4 = (a.n_pages + 3) >> 2;
  for (int i0 = 0; i0 < n4 && found < total; i0 += PP_NT) {
    const int p = (i0 + tid) * 4;
    unsigned int free = 0;
    if (p + 3 < a.n_pages) {
      const int4 r = __ldcg(reinterpret_cast<const int4*>(a.refs) + i0 + tid);
      free = (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
    } else {
      for (int k = 0; k < 4; ++k)
        if (p + k < a.n_pages) free |= (unsigned)(a.refs[p + k] == 0) << k;
    }
    int sum;
    int at = found + cta_prefix(__popc(free), warp_s, sum);
    for (; free && at < total; free &= free - 1) mv.free[at++] = p + __ffs(free) - 1;
    found += sum;
  }
  __syncthreads();  // (the list is written)
  // the tables and the counts
  for (int s = warp; s < S; s += PP_WARPS) {
    int lo, hi;
    const bool ok = places(s, lo, hi);
    // rows are served in order until one does not fit
    if (!ok || before_s[s] + need_s[s] > found) {
      if (lane == 0) {
        if (ok) set_error(a.err, SP_DEVERR_PAGES);
        move_s[s] = 0;
      }
      continue;
    }
    int* row = a.table + (size_t)s * a.max_pages;
    int at = before_s[s];
    if (COMPACT) {
      const int n = __ldg(add + s), pages = (n + page - 1) >> shift;
      const int stay = move_s[s] ? (n - move_s[s]) >> shift : pages;
      if (lane == 0) mv.old_len[s] = a.lens[s];
      for (int c = lane; c < a.max_pages; c += 32) {
        const int e = row[c];
        mv.old[(size_t)s * a.max_pages + c] = e;
        if (c < stay) continue;
        const int now = c < pages ? mv.free[at + c - stay] : -1;
        if (e >= 0 && e < a.n_pages) atomicSub(a.refs + e, 1);
        else if (e >= a.n_pages) set_error(a.err, SP_DEVERR_INDEX);
        if (now >= 0) a.refs[now] = 1;
        row[c] = now;
      }
      __syncwarp();
      if (lane == 0) a.lens[s] = n;
    } else {
      for (int c0 = lo; c0 < hi; c0 += 32) {
        const int c = c0 + lane, e = c < hi ? mv.old[(size_t)s * a.max_pages + c] : -2;  // (this lane wrote it)
        const unsigned int all = __ballot_sync(0xffffffffu, e != -2);
        if (e != -2) {
          const int now = mv.free[at + __popc(all & ((1u << lane) - 1u))];
          if (e >= 0) atomicSub(a.refs + e, 1);
          a.refs[now] = 1;
          row[c] = now;
        }
        at += __popc(all);
      }
    }
  }
  __syncthreads();
  int moved = 0;
  for (int s0 = 0; s0 < S; s0 += PP_NT) {
    const int s = s0 + tid;
    int sum;
    const int before = cta_prefix(s < S ? move_s[s] : 0, warp_s, sum) + moved;
    if (s < S) mv.start[s] = before;
    moved += sum;
  }
  if (tid == 0) mv.start[S] = moved;
}

constexpr int PM_NT = 256, PM_POS = 8;  // positions of a warp's share

// The rows of the positions that move, all planes (a layer's keys or values).  A warp takes PM_POS positions of one plane.
template <bool COMPACT>
__global__ void __launch_bounds__(PM_NT)
pages_copy_kernel(const PagesArgs a, const int* __restrict__ keep, long long ld_keep, PageMoves mv) {
  extern __shared__ int start_s[];  // [S + 1]
  pdl_wait();
  pdl_trigger();
  const int S = a.S, lane = threadIdx.x & 31, shift = a.page_shift, mask = (1 << shift) - 1;
  if (__ldcg(mv.start + S) == 0) return;
  for (int i = threadIdx.x; i <= S; i += PM_NT) start_s[i] = __ldcg(mv.start + i);
  __syncthreads();
  const int total = start_s[S];
  const int shares = (total + PM_POS - 1) / PM_POS;
  const long long units = (long long)shares * a.planes;
  for (long long u = blockIdx.x * (long long)(PM_NT / 32) + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * (PM_NT / 32)) {
    const int plane = (int)(u / shares), pos = (int)(u % shares) * PM_POS + lane;
    long long src = -1, dst = 0;  // rows of the plane
    if (lane < PM_POS && pos < total) {
      int x = 0, y = S - 1;  // the row it belongs to: the last that begins at or before it
      while (x < y) {
        const int mid = (x + y + 1) >> 1;
        if (start_s[mid] <= pos) x = mid; else y = mid - 1;
      }
      const int at = pos - start_s[x], len = __ldcg(a.lens + x);
      const int* table = a.table + (size_t)x * a.max_pages;
      const int* old = mv.old + (size_t)x * a.max_pages;
      if (COMPACT) {
        const int to = len - (start_s[x + 1] - start_s[x]) + at, from = __ldg(keep + x * ld_keep + to);
        int e = -1;
        if (from >= 0 && from < __ldcg(mv.old_len + x)) e = __ldcg(old + (from >> shift));
        if (e >= 0 && e < a.n_pages) src = ((long long)e << shift) + (from & mask);
        else if (plane == 0) set_error(a.err, SP_DEVERR_INDEX);
        dst = ((long long)__ldcg(table + (to >> shift)) << shift) + (to & mask);
      } else {
        src = ((long long)__ldcg(old + (len >> shift)) << shift) + at;
        dst = ((long long)__ldcg(table + (len >> shift)) << shift) + at;
      }
    }
    uint4* pl = a.kv + ((size_t)plane * a.n_pages << shift) * a.row16;
    for (int i = lane; i - lane < PM_POS * a.row16; i += 32 * 8) {
      uint4 v[8];
      uint4* to[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int w = i + 32 * k, r = min(w / a.row16, PM_POS - 1), at = w - r * a.row16;
        const long long from = __shfl_sync(0xffffffffu, src, r);
        to[k] = pl + __shfl_sync(0xffffffffu, dst, r) * a.row16 + at;
        if (at >= a.row16 || from < 0) to[k] = nullptr;
        else v[k] = __ldcs(pl + from * a.row16 + at);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (to[k]) *to[k] = v[k];
    }
  }
}

}  // namespace

cudaError_t pages_trim_launch(const PagesArgs& a, cudaStream_t st) {
  prof_begin_launch(st);
  const cudaError_t r = launch_pdl(pages_trim_kernel, dim3((a.max_pages + PT_NT - 1) / PT_NT, a.S), dim3(PT_NT), 0, st, a);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

cudaError_t pages_fork_launch(const PagesArgs& a, const int* parent, cudaStream_t st) {
  const int smem = a.S * (1 + PF_COLS) * 4;
  static std::atomic<unsigned long long> allowed;
  cudaError_t r = allow_smem(pages_fork_kernel, SP_MAX_TABLE_ROWS * (1 + PF_COLS) * 4, allowed);
  if (r != cudaSuccess) return r;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(std::min((a.max_pages + PF_COLS - 1) / PF_COLS, PF_CTAS));
  cfg.blockDim = dim3(PF_NT);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cfg.gridDim.x;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  prof_begin_launch(st);
  r = cudaLaunchKernelEx(&cfg, pages_fork_kernel, a, parent);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

static size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

size_t pages_bytes(int S, int max_pages) {
  return 2 * align256(((size_t)S + 1) * 4) + 2 * align256((size_t)S * max_pages * 4);
}

cudaError_t pages_move_launch(const PagesArgs& a, const int* add, const int* keep, long long ld_keep, int keep_cap, void* ws,
                              cudaStream_t st) {
  const size_t rows = align256(((size_t)a.S + 1) * 4), entries = align256((size_t)a.S * a.max_pages * 4);
  char* base = static_cast<char*>(ws);
  PageMoves mv;
  mv.start = reinterpret_cast<int*>(base);
  mv.old_len = reinterpret_cast<int*>(base + rows);
  mv.old = reinterpret_cast<int*>(base + 2 * rows);
  mv.free = reinterpret_cast<int*>(base + 2 * rows + entries);
  static std::atomic<unsigned long long> allowed[2];
  auto* plan = keep ? pages_plan_kernel<true> : pages_plan_kernel<false>;
  cudaError_t r = allow_smem(plan, SP_MAX_TABLE_ROWS * 12, allowed[keep != nullptr]);
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  r = launch_pdl(plan, dim3(1), dim3(PP_NT), (size_t)a.S * 12, st, a, add, keep, ld_keep, keep_cap, mv);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  if (r != cudaSuccess) return r;
  prof_begin_launch(st);
  r = launch_pdl(keep ? pages_copy_kernel<true> : pages_copy_kernel<false>, dim3(device_sm_count() * 8), dim3(PM_NT),
                 ((size_t)a.S + 1) * 4, st, a, keep, ld_keep, mv);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
