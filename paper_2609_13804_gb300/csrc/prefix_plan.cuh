// How the attention over shared prefixes (prefix_attn.cu, prefix_attn_tc.cu) is cut into work.
//
// The keys a call reads form entries: entry g < n_groups is group g's prefix, read by all rows of the
// group's sequences; entry n_groups + b is sequence b's own keys, read by its rows.  For one key / value
// head the G = Hq / Hkv query heads of a row read the same keys, so an entry with R rows is a product of
// M = R G query vectors (vector m: row m / G, head m % G of the kv head's G) with the entry's keys.  The M
// vectors are cut into row tiles, the keys into key tiles; an item is (entry, row tile, kv head).  An item
// counts `over` units for what it costs whatever its length (its query vectors in, its result out) and one
// for each of its key tiles, and the items' units, one after the other, are one list of N.  P workers (warps,
// or CTAs of the tensor kernel) take equal consecutive parts of it, whatever the entries' lengths: worker w
// the units [w N / P, (w + 1) N / P).  The key tiles of an item that one worker takes are a segment; it writes
// its running max, sum and weighted values in 32 bits to slot (item index + worker index), which is its own:
// going along the list, each next segment has the next item or the next worker.  prefix_merge_kernel joins
// every row's segments.  All lengths are read on the device; every CTA builds the same plan from them.
#pragma once
#include "common.cuh"

namespace sp {

constexpr int kPlanEntries = 2 * SP_MAX_BATCH;
// Units of a plan, at most: they are counted in 32 bits.  Whether an entry's or all entries' are more is told from
// counts of kCoarse units, rounded up.
constexpr int kCoarse = 1 << 16, kMaxUnits = 32000 * kCoarse;

struct PrefixArgs {
  const __nv_bfloat16* q;
  long long ld_q;
  __nv_bfloat16* out;
  long long ld_out;
  float* lse;              // [T_cap, Hq] or NULL
  const __nv_bfloat16* kv; // [2][n_pages][page][Hkv DH]
  int n_pages, page_shift;
  const int* table;
  int max_pages;
  const int* lens;
  const int* ptable;
  int pmax_pages;
  const int* plens;
  const int* group_cu;
  int n_groups;
  const int* cu_rows;      // NULL: row b is sequence b's
  int B, T_cap, Hq, Hkv;
  float scale_log2;        // scale * log2(e): scores are exponentiated in base 2
  int* err;
};

// One launch's share of the entries, and where its segments go.
struct PlanArgs {
  int tile_rows;           // query vectors of a row tile
  int key_shift;           // log2 of the keys of a key tile
  int over;                // units of an item besides its key tiles
  int min_shift;           // log2 of the units a worker takes at least (while there are enough)
  int workers;
  int max_items;           // items there is room for: no more exist while row and group offsets ascend (else, and
                           // with over kMaxUnits units in all, the launch covers nothing and reports SP_DEVERR_INDEX)
  bool prefix, own;        // which entries this launch covers
  int* unit0;              // [n_groups + B + 1] first unit of each entry, then N      (written for the merge)
  int* item0;              // [n_groups + B + 1] first item of each entry, then the item count
  int4* rows_prefix;       // [T_cap] where a row's prefix items lie (if this launch covers prefixes): the entry's first
  int4* rows_own;          // unit, units per item (0: none), first item, the row's first vector; its own items likewise
  float* part_o;           // [slots][slot_rows][DH]
  float2* part_ml;         // [slots][slot_rows] (max in log2 units, sum)
  int slot_rows;
};

// Rows of sequence b begin here (b in 0..B), clamped to the rows there are.
SP_DEVINL int row_begin(const PrefixArgs& a, int b) {
  return min(max(a.cu_rows ? __ldg(a.cu_rows + b) : b, 0), a.T_cap);
}

struct PlanShared {
  int unit0[kPlanEntries + 1];
  int item0[kPlanEntries + 1];
  int row0[kPlanEntries], rows[kPlanEntries], keys[kPlanEntries];
  uint2 wsum[32];  // a warp's items and units (a CTA has 32 warps at most)
  unsigned int wcoarse[32];  // and its units in kCoarse
};

// (N is at most kMaxUnits)
SP_DEVINL int plan_workers(const PlanArgs& p, int N) { return max(min(p.workers, (N + (1 << p.min_shift) - 1) >> p.min_shift), 1); }
// First unit of worker w's part, floor(w N / P), without products over 32 bits (P is below 2^15).
SP_DEVINL int part_begin(int N, int P, int w) {
  const int q = N / P, r = N - q * P;
  return w * q + w * r / P;
}
// Worker w's units [t0, t1).
SP_DEVINL void part_of_worker(int N, int P, int w, int& t0, int& t1) {
  const int q = N / P, r = N - q * P, a = w * r, f = a / P;
  t0 = w * q + f;
  t1 = t0 + q + (a - f * P + r >= P ? 1 : 0);
}

// Called by all NT threads of the CTA (a multiple of 32, at most 1,024).
template <int NT>
SP_DEVINL void build_plan(const PrefixArgs& a, const PlanArgs& p, PlanShared& s, bool write) {
  const int E = a.n_groups + a.B, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.Hq / a.Hkv;
  constexpr int PER = (kPlanEntries + NT - 1) / NT;
  int i_sum = 0;
  unsigned int t_sum = 0;  // (may wrap where there are too many)
  unsigned int coarse = 0;  // units in kCoarse, an entry's up to kMaxUnits / kCoarse + 1 (so that all entries' fit)
  unsigned int tl[PER];
  int il[PER], r0[PER], r1[PER], len[PER];
  // every thread's loads at once, first those that others depend on (entries beyond the last: the last's again)
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int e = min(tid * PER + k, E - 1), b = e - a.n_groups;
    r0[k] = b < 0 ? __ldg(a.group_cu + e) : b;
    r1[k] = b < 0 ? __ldg(a.group_cu + e + 1) : b + 1;
    len[k] = __ldg(b < 0 ? a.plens + e : a.lens + b);
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    r0[k] = row_begin(a, min(max(r0[k], 0), a.B));
    r1[k] = row_begin(a, min(max(r1[k], 0), a.B));
  }
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int e = tid * PER + k;
    int items = 0;
    unsigned int units = 0;
    if (e < E) {
      const bool pre = e < a.n_groups;
      const int r = max(r1[k] - r0[k], 0);
      const int cap = (pre ? a.pmax_pages : a.max_pages) << a.page_shift;
      if ((len[k] < 0 || len[k] > cap) && write) set_error(a.err, SP_DEVERR_INDEX);
      const int keys = min(max(len[k], 0), cap);
      s.row0[e] = r0[k];
      s.rows[e] = r;
      s.keys[e] = keys;
      if (pre ? p.prefix : p.own) {
        items = (r * G + p.tile_rows - 1) / p.tile_rows * a.Hkv;
        const int kt = (keys + (1 << p.key_shift) - 1) >> p.key_shift;
        const long long n = kt ? (long long)items * (kt + p.over) : 0;
        units = (unsigned int)min(n, (long long)kMaxUnits);
        coarse += (unsigned int)min((n + kCoarse - 1) / kCoarse, (long long)(kMaxUnits / kCoarse + 1));
      }
    }
    il[k] = items;
    tl[k] = units;
    i_sum += items;
    t_sum += units;
  }
  int ix = i_sum;
  unsigned int tx = t_sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int iu = __shfl_up_sync(0xffffffffu, ix, o);
    const unsigned int tu = __shfl_up_sync(0xffffffffu, tx, o);
    if (lane >= o) {
      ix += iu;
      tx += tu;
    }
  }
  coarse = __reduce_add_sync(0xffffffffu, coarse);
  if (lane == 31) {
    s.wsum[warp] = make_uint2(ix, tx);
    s.wcoarse[warp] = coarse;
  }
  __syncthreads();
  ix -= i_sum;
  tx -= t_sum;
  int total = 0;
  coarse = 0;
#pragma unroll
  for (int w = 0; w < NT / 32; ++w) {
    const uint2 x = s.wsum[w];
    total += (int)x.x;
    coarse += s.wcoarse[w];
    ix += w < warp ? (int)x.x : 0;
    tx += w < warp ? x.y : 0;
  }
  const bool fits = total <= p.max_items && coarse <= kMaxUnits / kCoarse;
  if (!fits && write && tid == 0) set_error(a.err, SP_DEVERR_INDEX);
#pragma unroll
  for (int k = 0; k <= PER; ++k) {  // (the total's place follows the last entry, maybe another thread's first)
    const int e = tid * PER + k;
    if (k < PER ? e <= E : (e == E && tid == NT - 1)) {
      const int i = fits ? ix : 0;
      const int t = fits ? (int)tx : 0;
      s.item0[e] = i;
      s.unit0[e] = t;
      if (write) {
        p.item0[e] = i;
        p.unit0[e] = t;
      }
    }
    if (k < PER) {
      ix += il[k];
      tx += tl[k];
    }
  }
  __syncthreads();
}

// Where row `row`'s items lie, of the entries e0 .. e1 - 1 (whose rows ascend).
SP_DEVINL int4 find_row(const PlanShared& s, int e0, int e1, int row, int G) {
  int lo = e0, hi = e1 - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.row0[mid] <= row) lo = mid; else hi = mid - 1;
  }
  const int in = row - s.row0[lo], items = s.item0[lo + 1] - s.item0[lo], units = s.unit0[lo + 1] - s.unit0[lo];
  if (in < 0 || in >= s.rows[lo] || units == 0) return make_int4(0, 0, 0, 0);
  return make_int4(s.unit0[lo], units / items, s.item0[lo], in * G);
}

// The merge's table of rows, by `threads` threads of every CTA (thread t of them).
SP_DEVINL void write_rows(const PrefixArgs& a, const PlanArgs& p, const PlanShared& s, int t, int threads) {
  const int G = a.Hq / a.Hkv;
  for (int row = blockIdx.x * threads + t; row < a.T_cap; row += gridDim.x * threads) {
    if (p.prefix) p.rows_prefix[row] = find_row(s, 0, a.n_groups, row, G);
    if (p.own) p.rows_own[row] = find_row(s, a.n_groups, a.n_groups + a.B, row, G);
  }
}

// A walk along the key tiles of a worker's part, which ends at unit t1.
struct TileCursor {
  int e, item, rt, kvh, j, kt;  // entry, item (over all entries), row tile, kv head, key tile of kt
  int u;                        // the key tile's unit
  SP_DEVINL void set_item(const PlanShared& s, const PlanArgs& p, int Hkv) {
    const int in = item - s.item0[e];
    rt = in / Hkv;
    kvh = in - rt * Hkv;
    kt = (s.keys[e] + (1 << p.key_shift) - 1) >> p.key_shift;
  }
  // to the first key tile at or behind unit t < t1; false: there is none before t1 (called by whole warps)
  SP_DEVINL bool seek(const PlanShared& s, const PlanArgs& p, int E, int Hkv, int t, int t1) {
    // the entry that holds unit t (entries without units are passed over), by the whole warp: every step-th entry,
    // then those between
    const int lane = threadIdx.x & 31, step = (E + 31) >> 5;
    static_assert(kPlanEntries <= 32 * 32, "two rounds of 32");
    const unsigned int coarse = __ballot_sync(0xffffffffu, lane * step < E && s.unit0[min(lane * step, E)] <= t);
    const int from = (31 - __clz(coarse)) * step;
    const unsigned int fine = __ballot_sync(0xffffffffu, lane < step && from + lane < E && s.unit0[min(from + lane, E)] <= t);
    e = from + 31 - __clz(fine);
    const int len = ((s.keys[e] + (1 << p.key_shift) - 1) >> p.key_shift) + p.over;
    const int off = t - s.unit0[e], in = off / len;
    item = s.item0[e] + in;
    j = max(off - in * len - p.over, 0);
    u = s.unit0[e] + in * len + p.over + j;
    set_item(s, p, Hkv);
    return u < t1;
  }
  // to the next key tile; false: there is none before t1
  SP_DEVINL bool next(const PlanShared& s, const PlanArgs& p, int Hkv, int t1) {
    if (++u >= t1) return false;  // (else there are units behind this one)
    if (++j < kt) return true;
    j = 0;
    ++item;
    while (item >= s.item0[e + 1] || s.unit0[e + 1] == s.unit0[e]) {
      ++e;
      item = s.item0[e];
    }
    set_item(s, p, Hkv);
    u += p.over;
    return u < t1;
  }
};

cudaError_t prefix_tc_launch(const PrefixArgs& a, const PlanArgs& p, int dh, cudaStream_t st);

}  // namespace sp
