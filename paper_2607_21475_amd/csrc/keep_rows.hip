// keep_rows.hip -- the rows of a tree's accepted path move together behind the rows held before the step.
//
// Row path[i] of a sequence's new rows becomes row i of them, for an increasing path: path[i] >= i, so that a row is read
// before anything is written over it if a thread takes its columns' rows in order, however they overlap.
//
// One work-group per sequence.  Its threads take 16 bytes of a row of K or V of a head each and go along the path, eight
// rows in flight; the rows' places are looked up once, by a thread each, and shared through LDS.  1024 bytes read and
// written per row and head: a few rows a sequence, so that a chain of loads (lengths, path, page numbers, rows) is what a
// small call takes.
#include "ebd.h"
#include "ebd_internal.hpp"
#include "paged_device.hpp"

#include <algorithm>

namespace ebd {

namespace {
constexpr int kKeepThreads = 256;
constexpr int kKeepChunk = 256;  // rows of the path whose places are in LDS at a time
constexpr int kKeepFlight = 8;
}  // namespace

__global__ __launch_bounds__(kKeepThreads) void keep_rows_kernel(KeepRowsLaunch L) {
  __shared__ int64_t from[kKeepChunk], to[kKeepChunk];
  const ebd_keep_rows_params &p = L.p;
  const int s = blockIdx.x;
  const int64_t n = p.new_off[s + 1] - p.new_off[s], len = p.len[s], first = len - n;
  const int kept = p.kept[s];
  const int32_t *path = p.path + (int64_t)s * p.max_kept;
  bool wrong = n < 0 || first < 0 || kept < 0 || kept > p.max_kept || kept > n;
  if (!wrong) {
    for (int i = threadIdx.x; i < kept; i += kKeepThreads) wrong |= path[i] >= n || path[i] <= (i ? path[i - 1] : -1);
  }
  wrong = __syncthreads_or(wrong);
  // (every thread has read len, which may be len_out)
  if (threadIdx.x == 0 && p.len_out) p.len_out[s] = (int32_t)(wrong ? len : first + kept);
  if (wrong) {
    if (threadIdx.x == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_LAYOUT);
    return;
  }
  const int pieces = 2 * p.pages.kv_heads, column = threadIdx.x % 16 * 8;
  for (int c = 0; c < kept; c += kKeepChunk) {
    const int m = min(kKeepChunk, kept - c);
    bool bad = false;
    if (c) __syncthreads();
    if (threadIdx.x < m) {
      const int i = c + threadIdx.x, a = path[i];
      int64_t x = -1, y = -1;
      if (a != i) {
        x = page_row(p.pages, L.shift, s, first + a), y = page_row(p.pages, L.shift, s, first + i);
        bad = x < 0 || y < 0;
        if (bad) x = -1;
      }
      from[threadIdx.x] = x, to[threadIdx.x] = y;
    }
    if (bad && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
    __syncthreads();
    for (int g = threadIdx.x / 16; g < pieces; g += kKeepThreads / 16) {
      uint16_t *pool = (g & 1 ? L.V : L.K) + (int64_t)(g >> 1) * p.pages.head_stride + column;
      for (int i = 0; i < m; i += kKeepFlight) {
        uint4 v[kKeepFlight];
#pragma unroll
        for (int k = 0; k < kKeepFlight; ++k) {
          v[k] = make_uint4(0u, 0u, 0u, 0u);
          if (i + k < m && from[i + k] >= 0) v[k] = *reinterpret_cast<const uint4 *>(pool + from[i + k]);
        }
#pragma unroll
        for (int k = 0; k < kKeepFlight; ++k)
          if (i + k < m && from[i + k] >= 0) *reinterpret_cast<uint4 *>(pool + to[i + k]) = v[k];
      }
    }
  }
}

hipError_t launch_keep_rows(const KeepRowsLaunch &L, hipStream_t s) {
  hipLaunchKernelGGL(keep_rows_kernel, dim3((unsigned)L.p.pages.num_seqs), dim3(kKeepThreads), 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
