// gather_paged.hip -- the pages of every sequence read out as units (one contiguous run of rows per KV
// head), which the scores and the sampler take.
//
// A copy: 512 bytes read and written per row of K and V, bound by the memory.  A work-group takes 64 rows of
// a unit, 16 lanes per 256-byte row, each lane's eight loads issued before its stores.  Calls that move more than the
// last-level cache holds pass it by (non-temporal): 32 sequences of up to 16384 rows, 8 KV heads, 470 -> 439 us (5.6 TB/s
// read and written; torch's copy runs at 4.9); one of 4096 rows 7.2 us without, 8.1 with.
#include "ebd.h"
#include "ebd_internal.hpp"
#include "paged_device.hpp"

namespace ebd {

namespace {
constexpr int kGatherPagedRows = 64;
constexpr int kGatherPagedThreads = 256;
constexpr int64_t kCacheBytes = (int64_t)256 << 20;

template <bool NT>
__device__ __forceinline__ uint4 load(const uint16_t *p) {
  if constexpr (NT) return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
  else return *reinterpret_cast<const uint4 *>(p);
}
template <bool NT>
__device__ __forceinline__ void store(uint16_t *p, const uint4 &v) {
  if constexpr (NT) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(p));
  else *reinterpret_cast<uint4 *>(p) = v;
}
}  // namespace

template <bool NT>
__global__ __launch_bounds__(kGatherPagedThreads) void gather_paged_kernel(GatherPagedLaunch L) {
  const ebd_pages &P = L.p.pages;
  const int u = blockIdx.x / L.chunks, c = blockIdx.x % L.chunks;
  const int s = u / P.kv_heads, h = u % P.kv_heads;
  const int64_t u0 = L.p.seq_off[u], n = L.p.seq_off[u + 1] - u0;
  const int64_t seen = min(n, L.p.max_rows);
  const bool outside = seen > 0 && (u0 < 0 || u0 > L.p.num_rows - seen);  // some rows have no place in Ku and Vu
  if (c == 0 && threadIdx.x == 0 && (n > L.p.max_rows || outside) && L.status)
    atomicOr(&L.status[u], EBD_ST_BAD_LAYOUT);
  const int64_t r0 = (int64_t)c * kGatherPagedRows + threadIdx.x / 16;
  if (r0 - threadIdx.x / 16 >= seen) return;
  const int e = threadIdx.x % 16 * 8;
  uint4 k[4], v[4];
  bool bad = false;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = r0 + 16 * j;
    const int64_t at = r < seen ? page_row(P, L.shift, s, r) : -1;
    k[j] = v[j] = make_uint4(0u, 0u, 0u, 0u);
    if (at >= 0) {
      k[j] = load<NT>(L.K + at + h * P.head_stride + e);
      v[j] = load<NT>(L.V + at + h * P.head_stride + e);
    }
    bad |= r < seen && at < 0;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t r = r0 + 16 * j;
    if (r < seen && (uint64_t)(u0 + r) < (uint64_t)L.p.num_rows) {
      store<NT>(L.Ku + (u0 + r) * kHeadDim + e, k[j]);
      store<NT>(L.Vu + (u0 + r) * kHeadDim + e, v[j]);
    }
  }
  if (bad && e == 0 && L.status) atomicOr(&L.status[u], EBD_ST_BAD_PAGE);
}

int64_t gather_paged_groups(const ebd_gather_paged_params &p) {
  return (int64_t)p.pages.num_seqs * p.pages.kv_heads * ((p.max_rows + kGatherPagedRows - 1) / kGatherPagedRows);
}

hipError_t launch_gather_paged(GatherPagedLaunch L, hipStream_t s) {
  L.chunks = (int32_t)((L.p.max_rows + kGatherPagedRows - 1) / kGatherPagedRows);
  const dim3 grid((unsigned)gather_paged_groups(L.p)), block(kGatherPagedThreads);
  const int64_t rows = (int64_t)L.p.pages.num_seqs * L.p.pages.kv_heads * L.p.max_rows;
  if (rows * 8 * kHeadDim > kCacheBytes) hipLaunchKernelGGL(gather_paged_kernel<true>, grid, block, 0, s, L);
  else hipLaunchKernelGGL(gather_paged_kernel<false>, grid, block, 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
