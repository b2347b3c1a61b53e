// paged_device.hpp -- device helpers of the paged-cache kernels.
#pragma once

#include "ebd.h"
#include "ebd_device.hpp"

namespace ebd {

// The sequence that owns new token t: the last s with off[s] <= t, or -1 when t lies before off[0] or
// from off[S] on.  A 64-ary search by one wave (t is uniform over it; every lane gets the result), two
// steps of loads for up to 4095 sequences.  Every probe is one of off's S + 1 entries, whatever they hold.
__device__ __forceinline__ int find_seq(const int64_t *off, int S, int64_t t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, width = S + 1;
  while (true) {
    const int step = (width + 63) / 64;
    const int i = lane * step;
    const bool below = i < width && off[lo + i] <= t;
    const int n = __popcll(__ballot(below));
    if (n == 0) return -1;
    lo += (n - 1) * step;
    width = min(step, width - (n - 1) * step);
    if (step == 1) break;
  }
  return lo < S ? lo : -1;
}

// Element offset of row r of sequence s in the pools (head 0), or -1 where the row has no page.
// shift = log2 page_size.
__device__ __forceinline__ int64_t page_row(const ebd_pages &P, int shift, int s, int64_t r) {
  const int64_t e = r >> shift;
  if (r < 0 || e >= P.max_pages) return -1;
  const int pg = P.page_table[(int64_t)s * P.max_pages + e];
  if ((uint32_t)pg >= (uint32_t)P.num_pages) return -1;
  return pg * P.page_stride + (r & (P.page_size - 1)) * P.row_stride;
}

// fp32 -> bf16 pairs, to nearest even (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 v;
  v[0] = (__bf16)lo;
  v[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, v);
}

}  // namespace ebd
