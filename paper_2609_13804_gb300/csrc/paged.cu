// Rows of a QKV projection into a paged cache: row j of sequence b belongs to position p = lens[b] + j, which
// lies in row p % page of page table[b][p / page].  The rotation is applied on the way: for pair i of a head,
// (x_i, x_{i + dh/2}) -> (x_i c - x_{i + dh/2} s, x_{i + dh/2} c + x_i s) with (c, s) of the row's rotary
// position, in fp32, rounded once to bf16.  Queries go to q_out, keys and values to their pages.
//
// Bound by the rows' bytes.  A thread takes 16 bytes of a head's first half and the 16 bytes they rotate with
// (of a value head: copies them); the threads of a row's heads are consecutive, so a row's (cos, sin) come from
// memory once and from L1 for its other heads.  Measured: 372 MB (7,600 rows of 96 heads of 128) in 59.5 us, 6.3 TB/s
// or 92% of a copy; a row for each of four sequences 2.6 us, a launch.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace sp {

namespace {

constexpr int PA_NT = 256;

__global__ void __launch_bounds__(PA_NT) paged_append_kernel(const PagedAppendArgs a) {
  __shared__ int s_cu[SP_MAX_BATCH + 1];
  pdl_wait();
  pdl_trigger();
  if (a.cu_rows) {
    for (int i = threadIdx.x; i <= a.B; i += PA_NT) s_cu[i] = __ldg(a.cu_rows + i);
    __syncthreads();
  }
  const int first = a.cu_rows ? max(s_cu[0], 0) : 0;
  const int T = a.cu_rows ? min(s_cu[a.B], a.T_cap) : a.B;
  const int cpr = a.dh / 16;  // threads per head
  const int per_row = (a.Hq + 2 * a.Hkv) * cpr;
  const int half = a.dh / 2;
  const size_t W = (size_t)a.Hkv * a.dh;
  const long long n = (long long)(T - first) * per_row;
  for (long long i = blockIdx.x * (long long)PA_NT + threadIdx.x; i < n; i += (long long)gridDim.x * PA_NT) {
    const int row = first + (int)(i / per_row);
    const int u = (int)(i % per_row);
    const int head = u / cpr, c = u - head * cpr;
    const __nv_bfloat16* src = a.qkv + row * a.ld + head * a.dh + c * 8;
    const uint4 lo = *reinterpret_cast<const uint4*>(src), hi = *reinterpret_cast<const uint4*>(src + half);
    __nv_bfloat16* dst;
    if (head < a.Hq) {
      if (!a.q_out) continue;
      dst = a.q_out + row * a.ld_q + head * a.dh;
    } else {
      int b = row, at = 0;
      if (a.cu_rows) {
        int x = 0, y = a.B - 1;
        while (x < y) {
          const int mid = (x + y + 1) >> 1;
          if (s_cu[mid] <= row) x = mid; else y = mid - 1;
        }
        b = x;
        at = row - s_cu[b];
      }
      const long long p = (long long)(a.lens ? __ldg(a.lens + b) : 0) + at;
      const long long pg = p >> a.page_shift;
      int page = -1;
      if (p >= 0 && pg < a.max_pages) page = __ldg(a.table + (size_t)b * a.max_pages + pg);
      if (page < 0 || page >= a.n_pages) {
        if (c == 0) set_error(a.err, SP_DEVERR_INDEX);
        continue;
      }
      const bool v = head >= a.Hq + a.Hkv;
      dst = a.kv + ((((size_t)(v ? a.n_pages : 0) + page) << a.page_shift) + (p & ((1 << a.page_shift) - 1))) * W +
            (size_t)(head - a.Hq - (v ? a.Hkv : 0)) * a.dh;
    }
    dst += c * 8;
    uint4 olo = lo, ohi = hi;
    if (a.pos || a.pos3) {  // (a value head checks the position too: a row is skipped whole)
      int pt, ph, pw;
      if (a.pos3) {
        const int4 q = __ldg(reinterpret_cast<const int4*>(a.pos3) + row);
        pt = q.x; ph = q.y; pw = q.z;
      } else {
        pt = ph = pw = __ldg(a.pos + row);
      }
      if (pt < 0 || pt >= a.max_pos || ph < 0 || ph >= a.max_pos || pw < 0 || pw >= a.max_pos) {
        if (c == 0) set_error(a.err, SP_DEVERR_INDEX);
        continue;
      }
      if (a.rope && head < a.Hq + a.Hkv) {
        const uint32_t xl[4] = {lo.x, lo.y, lo.z, lo.w}, xh[4] = {hi.x, hi.y, hi.z, hi.w};
        uint32_t yl[4], yh[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {  // pairs 8 c + 2 k and the next (sections begin at even pairs)
          const int pair = c * 8 + 2 * k;
          const int q = pair < a.sec1 ? pt : (pair < a.sec2 ? ph : pw);
          const float4 cs = __ldg(reinterpret_cast<const float4*>(a.rope + (size_t)q * half + pair));
          const float2 x = unpack_bf16x2(xl[k]), y = unpack_bf16x2(xh[k]);
          yl[k] = pack_bf16x2(x.x * cs.x - y.x * cs.y, x.y * cs.z - y.y * cs.w);
          yh[k] = pack_bf16x2(y.x * cs.x + x.x * cs.y, y.y * cs.z + x.y * cs.w);
        }
        olo = make_uint4(yl[0], yl[1], yl[2], yl[3]);
        ohi = make_uint4(yh[0], yh[1], yh[2], yh[3]);
      }
    }
    *reinterpret_cast<uint4*>(dst) = olo;
    *reinterpret_cast<uint4*>(dst + half) = ohi;
  }
}

}  // namespace

cudaError_t paged_append_launch(const PagedAppendArgs& a, cudaStream_t st) {
  const int rows = a.cu_rows ? a.T_cap : a.B;
  if (rows == 0) return cudaSuccess;
  const long long n = (long long)rows * (a.Hq + 2 * a.Hkv) * (a.dh / 16);
  const int grid = (int)std::min<long long>((n + PA_NT - 1) / PA_NT, (long long)device_sm_count() * 32);
  prof_begin_launch(st);
  const cudaError_t r = launch_pdl(paged_append_kernel, dim3(grid), dim3(PA_NT), 0, st, a);
  prof_end_launch(st, SP_K_MISC, 0.0, 2.0 * n * 32);
  return r;
}

}  // namespace sp
