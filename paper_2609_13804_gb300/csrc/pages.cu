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

// Entries behind the page of a row's last position go back.  A thread per entry; atomics on counts commute.  A launch and
// length -> entry -> count: 2.4 us for 64 rows.
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
constexpr int PF_ENTRIES = 1 << 15;  // table entries in shared memory, at most

// A row's new entries are its parent's of the same columns, so a CTA needs the old entries of all rows in its columns and
// no others.  One cluster: the lengths change when all of its CTAs have read them.  Latency: 160 rows of 40 entries 4.5 us, 9 of
// 275 4.1 (by strips of 8 columns 8.7).
__global__ void __launch_bounds__(PF_NT) pages_fork_kernel(const PagesArgs a, const int* __restrict__ parent, int cols_shift) {
  extern __shared__ int fork_s[];  // [S] old lengths, [S] the rows that they continue, [S][columns] old entries
  int *len_s = fork_s, *from_s = fork_s + a.S, *old_s = fork_s + 2 * a.S;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, cols = 1 << cols_shift, n = a.S << cols_shift;
  for (int s = tid; s < a.S; s += PF_NT) {
    len_s[s] = a.lens[s];
    from_s[s] = __ldg(parent + s);
  }
  int c0 = blockIdx.x << cols_shift;
  auto load = [&]() {
    for (int i = tid; i < n; i += PF_NT) {
      const int c = c0 + (i & (cols - 1));
      old_s[i] = c < a.max_pages ? a.table[(size_t)(i >> cols_shift) * a.max_pages + c] : -1;
    }
  };
  load();
  __syncthreads();
  const long long most = (long long)a.max_pages << a.page_shift;
  for (int s = tid; s < a.S; s += PF_NT) {  // a row that stays continues itself
    const int p = from_s[s];
    if (p < 0 || p >= a.S || len_s[p] < 0 || len_s[p] > most) {
      if (p != -1) set_error(a.err, SP_DEVERR_INDEX);
      from_s[s] = s;
    }
  }
  __syncthreads();
  // (release: this CTA's reads of the lengths come before the writes behind the wait)
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  for (;;) {
    for (int i = tid; i < n; i += PF_NT) {
      const int s = i >> cols_shift, k = i & (cols - 1), c = c0 + k, p = from_s[s];
      if (c >= a.max_pages || p == s) continue;
      const int old = old_s[i];
      int now = c < (len_s[p] + (1 << a.page_shift) - 1) >> a.page_shift ? old_s[(p << cols_shift) + k] : -1;
      if (now >= a.n_pages || old >= a.n_pages) set_error(a.err, SP_DEVERR_INDEX);
      if (now >= a.n_pages || now < 0) now = -1;
      if (now == old) continue;
      if (now >= 0) atomicAdd(a.refs + now, 1);
      if (old >= 0 && old < a.n_pages) atomicSub(a.refs + old, 1);
      a.table[(size_t)s * a.max_pages + c] = now;
    }
    c0 += gridDim.x << cols_shift;
    if (c0 >= a.max_pages) break;
    __syncthreads();
    load();
    __syncthreads();
  }
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (blockIdx.x == 0)
    for (int s = tid; s < a.S; s += PF_NT)
      if (from_s[s] != s) a.lens[s] = len_s[from_s[s]];
}

// ------------------------------------------------------------------------- reserve, compact

constexpr int PP_NT = 1024, PP_WARPS = PP_NT / 32, PP_CTAS = 8;
constexpr int PP_LOADS = 4;  // of a lane at once

// What the kernels of a call leave each other.
struct PageMoves {
  int* need;     // [S] pages that a row needs
  int* move;     // [S] positions of it that move
  int* start;    // [S + 1] positions that move before each row's
  int* was;      // [S] compact: the row's length before; reserve: whether shared pages of it are replaced
  int* old;      // [S, max_pages] the entries that rows had (reserve: those of the places that are replaced)
  int* place;    // [S, max_pages] reserve: the places of a row that get pages
  int* count;    // [PP_CTAS] free pages that each CTA of the plan has found
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

// Which free pages the rows take, in order of rows and places, and the tables and counts after it.  One cluster: a warp
// finds what a row needs, while its CTA looks through its share of the counts for free pages; then every CTA knows all
// rows' needs and gives its free pages to the places they fall to.  (A free page finds its row: a list of the free ones, for
// rows to take from, would cost another barrier.)  Latency, about 7 us behind the call before: lengths -> entries -> counts,
// the cluster's barrier, needs -> places -> entries.  256 rows that take 11,500 of 25,000 pages 9 us (one CTA: 38), 64 that
// take 64 of them 7.
template <bool COMPACT>
__global__ void __launch_bounds__(PP_NT, 1)
pages_plan_kernel(const PagesArgs a, const int* __restrict__ add, const int* __restrict__ keep, long long ld_keep, int keep_cap,
                  PageMoves mv) {
  extern __shared__ int before_s[];  // [S + 1] pages that rows before each one need
  __shared__ int warp_s[PP_WARPS], free_s[PP_CTAS];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, rank = blockIdx.x, lane = tid & 31, S = a.S, shift = a.page_shift, page = 1 << shift;
  const int warp = rank * PP_WARPS + (tid >> 5), warps = PP_CTAS * PP_WARPS;
  const long long most = (long long)a.max_pages << shift;
  // this CTA's share of the counts: p0 .. p1 - 1, a piece of four to a thread and turn
  const int share = (((a.n_pages + PP_CTAS - 1) / PP_CTAS) + 3) & ~3;
  const int p0 = min(rank * share, a.n_pages), p1 = min(p0 + share, a.n_pages);
  auto bits = [](const int4& r) -> unsigned int {  // of the free ones of four pages
    return (r.x == 0) | (r.y == 0) << 1 | (r.z == 0) << 2 | (r.w == 0) << 3;
  };
  auto free_at = [&](int p) {
    if (p + 3 < p1) return bits(__ldcg(reinterpret_cast<const int4*>(a.refs + p)));
    unsigned int free = 0;
    for (int k = 0; p + k < p1; ++k) free |= (unsigned)(__ldcg(a.refs + p + k) == 0) << k;
    return free;
  };
  int4 refs0 = make_int4(1, 1, 1, 1);  // (its first piece, looked at behind the rows)
  const bool whole0 = p0 + tid * 4 + 3 < p1;
  if (whole0) refs0 = __ldcg(reinterpret_cast<const int4*>(a.refs + p0 + tid * 4));
  int need0 = 0, released0 = 0;  // of this warp's first row
  for (int s = warp; s < S; s += warps) {
    const int len = a.lens[s], n = __ldg(add + s);
    const int* row = a.table + (size_t)s * a.max_pages;
    int* old = mv.old + (size_t)s * a.max_pages;
    int need = 0, move = 0, released = 0;
    if (COMPACT) {
      if (n < 0 || n > keep_cap || n > most || len < 0 || len > most) {
        if (n != -1 && lane == 0) set_error(a.err, SP_DEVERR_INDEX);
        need = -1;  // the row stays as it is
      } else {
        // the first position that moves (or that the row does not have, which the copy finds)
        const int there = min(n, len);
        int first = there;
        for (int i0 = 0; i0 < there; i0 += 32) {
          const unsigned int other =
              __ballot_sync(0xffffffffu, i0 + lane < there && __ldg(keep + s * ld_keep + i0 + lane) != i0 + lane);
          if (other) {
            first = i0 + __ffs(other) - 1;
            break;
          }
        }
        const int pages = (n + page - 1) >> shift, stay = first == n ? pages : first >> shift;
        need = pages - stay;
        move = first == n ? 0 : n - (stay << shift);
#pragma unroll 4
        for (int c = lane; c < a.max_pages; c += 32) old[c] = row[c];
        released = len;
      }
    } else if (len < 0 || n < 0 || (long long)len + n > most) {
      if (lane == 0) set_error(a.err, SP_DEVERR_INDEX);
    } else if (n > 0) {
      const int lo = len >> shift, hi = (int)(((long long)len + n + page - 1) >> shift);
      int shares = 0;
      for (int c0 = lo; c0 < hi; c0 += 32 * PP_LOADS) {
        int e[PP_LOADS], named[PP_LOADS];
#pragma unroll
        for (int k = 0; k < PP_LOADS; ++k) {
          const int c = c0 + 32 * k + lane;
          e[k] = c < hi ? row[c] : -1;
        }
#pragma unroll
        for (int k = 0; k < PP_LOADS; ++k) {
          if (e[k] >= a.n_pages) {
            set_error(a.err, SP_DEVERR_INDEX);
            e[k] = -1;
          }
          named[k] = e[k] >= 0 ? __ldcg(a.refs + e[k]) : 0;
        }
#pragma unroll
        for (int k = 0; k < PP_LOADS; ++k) {
          const int c = c0 + 32 * k + lane;
          const bool shared = named[k] > 1, gets = c < hi && (e[k] < 0 || shared);
          const unsigned int all = __ballot_sync(0xffffffffu, gets);
          if (gets) {
            mv.place[(size_t)s * a.max_pages + need + __popc(all & ((1u << lane) - 1u))] = c;
            old[c] = shared ? e[k] : -1;
          }
          need += __popc(all);
          shares += shared;
          if (c0 == lo && k == 0 && __shfl_sync(0xffffffffu, (int)shared, 0)) move = len & (page - 1);
        }
      }
      released = __any_sync(0xffffffffu, shares > 0);
    }
    if (lane == 0) {
      mv.need[s] = need;
      mv.move[s] = move;
      mv.was[s] = released;
    }
    if (s == warp) need0 = need, released0 = released;
  }
  const unsigned int free0 = whole0 ? bits(refs0) : p0 + tid * 4 < p1 ? free_at(p0 + tid * 4) : 0u;
  int mine = __popc(free0);
  for (int p = p0 + (tid + PP_NT) * 4; p < p1; p += PP_NT * 4) mine += __popc(free_at(p));
  int sum;
  const int at0 = cta_prefix(mine, warp_s, sum);  // (of its first piece, where it has no more)
  if (tid == 0) mv.count[rank] = sum;
  cluster_sync_all();
  if (tid < PP_CTAS) free_s[tid] = __ldcg(mv.count + tid);
  int total = 0, move0 = 0;
  for (int s0 = 0; s0 < S; s0 += PP_NT) {
    const int s = s0 + tid;
    if (s0 == 0 && rank == 0 && s < S) move0 = __ldcg(mv.move + s);
    const int before = total + cta_prefix(s < S ? max(__ldcg(mv.need + s), 0) : 0, warp_s, sum);
    if (s < S) before_s[s] = before;
    total += sum;
  }
  if (tid == 0) before_s[S] = total;
  __syncthreads();
  int base = 0, found = 0;  // free pages before this CTA's, and all
  for (int i = 0; i < PP_CTAS; ++i) {
    if (i < rank) base += free_s[i];
    found += free_s[i];
  }
  // (rows are served in order until one does not fit)
  // Free pages from the at-th on, of four pages from p: each to the row that needs it, and the place.
  auto give_all = [&](unsigned int free, int at, int p) {
    int x = -1;
    for (; free && at < total; free &= free - 1, ++at) {
      if (x < 0 || before_s[x + 1] <= at) {  // the last row with at most `at` pages before it
        int y = S - 1;
        x = max(x, 0);
        while (x < y) {
          const int mid = (x + y + 1) >> 1;
          if (before_s[mid] <= at) x = mid; else y = mid - 1;
        }
      }
      if (before_s[x + 1] > found) return;
      const int k = at - before_s[x], id = p + __ffs(free) - 1;
      int c;
      if (COMPACT) {
        const int n = __ldg(add + x), pages = (n + page - 1) >> shift;
        c = pages - (before_s[x + 1] - before_s[x]) + k;
      } else {
        c = __ldcg(mv.place + (size_t)x * a.max_pages + k);
      }
      a.refs[id] = 1;
      a.table[(size_t)x * a.max_pages + c] = id;
    }
  };
  const bool again = share > PP_NT * 4;  // counts are looked at a second time
  if (!again) {
    give_all(free0, base + at0, p0 + tid * 4);
  } else {
    for (int q0 = p0; q0 < p1 && base < total; q0 += PP_NT * 4) {
      const unsigned int free = q0 + tid * 4 < p1 ? free_at(q0 + tid * 4) : 0u;
      const int at = base + cta_prefix(__popc(free), warp_s, sum);
      give_all(free, at, q0 + tid * 4);
      base += sum;
    }
  }
  // Only now are pages released: counts must not fall to 0 under the eyes of those who look for free pages.
  if (again) cluster_sync_all();
  for (int s = warp; s < S; s += warps) {
    if ((s == warp ? need0 : __ldcg(mv.need + s)) < (COMPACT ? 0 : 1) || before_s[s + 1] > found) continue;
    const int* old = mv.old + (size_t)s * a.max_pages;
    const int taken = before_s[s + 1] - before_s[s];
    if (COMPACT) {
      const int n = __ldg(add + s), pages = (n + page - 1) >> shift;
#pragma unroll 4
      for (int c = pages - taken + lane; c < a.max_pages; c += 32) {
        const int e = __ldcg(old + c);
        if (e >= 0 && e < a.n_pages) atomicSub(a.refs + e, 1);
        else if (e >= a.n_pages) set_error(a.err, SP_DEVERR_INDEX);
        if (c >= pages) a.table[(size_t)s * a.max_pages + c] = -1;
      }
      if (lane == 0) a.lens[s] = n;
    } else if (s == warp ? released0 : __ldcg(mv.was + s)) {
      for (int i = lane; i < taken; i += 32) {
        const int e = __ldcg(old + __ldcg(mv.place + (size_t)s * a.max_pages + i));
        if (e >= 0) atomicSub(a.refs + e, 1);
      }
    }
  }
  if (rank == 0) {
    int moved = 0;
    for (int s0 = 0; s0 < S; s0 += PP_NT) {
      const int s = s0 + tid;
      const bool on = s < S && before_s[s + 1] <= found;
      const int before = moved + cta_prefix(!on ? 0 : s0 == 0 ? move0 : __ldcg(mv.move + s), warp_s, sum);
      if (s < S) mv.start[s] = before;
      moved += sum;
    }
    if (tid == 0) {
      mv.start[S] = moved;
      if (total > found) set_error(a.err, SP_DEVERR_PAGES);
    }
  }
}

constexpr int PM_NT = 256, PM_WARPS = PM_NT / 32;
constexpr int PM_LOADS = 8;    // 16-byte loads of a lane at once
constexpr int PM_PIECES = 512;  // of a warp's share of a plane, about

// The rows of the positions that move, all planes (a layer's keys or values).  A warp takes a few positions of a few planes
// (positions: about PM_PIECES pieces of 16 bytes; planes: several where enough warps have work): it looks up where they
// were and go once, then copies.  Bound by HBM, which reads and writes mixed: 13,904 positions of 56 planes of 1 KB, 1.6 GB
// read and written, 251 us with the plan's last part, 6.35 TB/s or 94% of a copy (a warp to 8 positions of any size, and
// pieces found by division: 467); 118 positions of 64 planes of 8 KB, 121 MB, 20 us.
template <bool COMPACT>
__global__ void __launch_bounds__(PM_NT, 3)
pages_copy_kernel(const PagesArgs a, const int* __restrict__ keep, long long ld_keep, PageMoves mv, int lanes_shift, int pos_shift) {
  extern __shared__ int start_s[];  // [S + 1]
  pdl_wait();
  pdl_trigger();
  const int S = a.S, lane = threadIdx.x & 31, shift = a.page_shift, mask = (1 << shift) - 1;
  for (int i = threadIdx.x; i <= S; i += PM_NT) start_s[i] = __ldcg(mv.start + i);
  __syncthreads();
  const int total = start_s[S];
  if (total == 0) return;
  const int shares = (total + (1 << pos_shift) - 1) >> pos_shift;
  const int warps = gridDim.x * PM_WARPS;
  // planes at a time: as many as give every warp one turn, where few do
  const int turns = (int)min(((long long)shares * a.planes + warps - 1) / warps, 8ll), planes = turns <= 4 ? turns : 4;
  const long long units = (long long)shares * ((a.planes + planes - 1) / planes);
  const int L = 1 << lanes_shift;  // lanes of a row
  const int steps = (a.row16 + L - 1) >> lanes_shift, groups = ((1 << pos_shift) + (32 >> lanes_shift) - 1) >> (5 - lanes_shift);
  for (long long u = blockIdx.x * (long long)PM_WARPS + (threadIdx.x >> 5); u < units; u += warps) {
    const int plane0 = (int)(u / shares) * planes, pos = ((int)(u % shares) << pos_shift) + lane;
    int src = -1, dst = 0;  // rows of a plane
    if (lane < 1 << pos_shift && pos < total) {
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
        if (from >= 0 && from < __ldcg(mv.was + x)) e = __ldcg(old + (from >> shift));
        if (e >= 0 && e < a.n_pages) src = (e << shift) + (from & mask);
        else if (plane0 == 0) set_error(a.err, SP_DEVERR_INDEX);
        dst = (__ldcg(table + (to >> shift)) << shift) + (to & mask);
      } else {
        src = (__ldcg(old + (len >> shift)) << shift) + at;
        dst = (__ldcg(table + (len >> shift)) << shift) + at;
      }
    }
    for (int plane = plane0; plane < min(plane0 + planes, a.planes); ++plane) {
      uint4* pl = a.kv + ((size_t)plane * a.n_pages << shift) * a.row16;
      for (int g0 = 0, s0 = 0; g0 < groups;) {
        uint4 v[PM_LOADS];
        int group = g0, step = s0;
        unsigned int have = 0;
#pragma unroll
        for (int k = 0; k < PM_LOADS; ++k) {
          const int r = (group << (5 - lanes_shift)) + (lane >> lanes_shift), at = (step << lanes_shift) + (lane & (L - 1));
          const int from = __shfl_sync(0xffffffffu, src, r & 31);
          if (group < groups && at < a.row16 && from >= 0) {
            v[k] = __ldcs(pl + (size_t)from * a.row16 + at);
            have |= 1u << k;
          }
          if (++step == steps) step = 0, ++group;
        }
        group = g0, step = s0;
#pragma unroll
        for (int k = 0; k < PM_LOADS; ++k) {
          const int r = (group << (5 - lanes_shift)) + (lane >> lanes_shift), at = (step << lanes_shift) + (lane & (L - 1));
          const int to = __shfl_sync(0xffffffffu, dst, r & 31);
          if (have >> k & 1) pl[(size_t)to * a.row16 + at] = v[k];
          if (++step == steps) step = 0, ++group;
        }
        g0 = group, s0 = step;
      }
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

// One cluster of `ctas`.
template <typename Kernel, typename... Args>
static cudaError_t launch_cluster(Kernel* k, int ctas, int threads, size_t smem, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = pdl_enabled() ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

cudaError_t pages_fork_launch(const PagesArgs& a, const int* parent, cudaStream_t st) {
  static std::atomic<unsigned long long> allowed;
  cudaError_t r = allow_smem(pages_fork_kernel, (2 * SP_MAX_TABLE_ROWS + PF_ENTRIES) * 4, allowed);
  if (r != cudaSuccess) return r;
  // columns at once: as many as give every CTA of the cluster one turn, where they fit
  int shift = 3;
  while (((long long)PF_CTAS << shift) < a.max_pages && ((long long)a.S << (shift + 1)) <= PF_ENTRIES) ++shift;
  const int ctas = (int)std::min<long long>((a.max_pages + (1ll << shift) - 1) >> shift, PF_CTAS);
  prof_begin_launch(st);
  r = launch_cluster(pages_fork_kernel, ctas, PF_NT, (size_t)a.S * (2 + (1 << shift)) * 4, st, a, parent, shift);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

static size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

size_t pages_bytes(int S, int max_pages) {
  return 4 * align256(((size_t)S + 1) * 4) + 2 * align256((size_t)S * max_pages * 4) + 256;
}

cudaError_t pages_move_launch(const PagesArgs& a, const int* add, const int* keep, long long ld_keep, int keep_cap, void* ws,
                              cudaStream_t st) {
  const size_t rows = align256(((size_t)a.S + 1) * 4), entries = align256((size_t)a.S * a.max_pages * 4);
  char* base = static_cast<char*>(ws);
  PageMoves mv;
  mv.count = reinterpret_cast<int*>(base);
  base += 256;
  mv.need = reinterpret_cast<int*>(base);
  mv.move = reinterpret_cast<int*>(base + rows);
  mv.start = reinterpret_cast<int*>(base + 2 * rows);
  mv.was = reinterpret_cast<int*>(base + 3 * rows);
  mv.old = reinterpret_cast<int*>(base + 4 * rows);
  mv.place = reinterpret_cast<int*>(base + 4 * rows + entries);
  prof_begin_launch(st);
  cudaError_t r = launch_cluster(keep ? pages_plan_kernel<true> : pages_plan_kernel<false>, PP_CTAS, PP_NT,
                                 ((size_t)a.S + 1) * 4, st, a, add, keep, ld_keep, keep_cap, mv);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  if (r != cudaSuccess) return r;
  int lanes = 0, pos = 0;
  while (lanes < 5 && 1 << lanes < a.row16) ++lanes;
  while (pos < 5 && a.row16 << (pos + 1) <= PM_PIECES) ++pos;
  prof_begin_launch(st);
  r = launch_pdl(keep ? pages_copy_kernel<true> : pages_copy_kernel<false>, dim3(device_sm_count() * 3), dim3(PM_NT),
                 ((size_t)a.S + 1) * 4, st, a, keep, ld_keep, mv, lanes, pos);
  prof_end_launch(st, SP_K_MISC, 0.0, 0.0);
  return r;
}

}  // namespace sp
