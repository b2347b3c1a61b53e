// plan_step.hip -- page tables, slots, positions and tree masks of a serving step, from the sequences' new token counts.
//
// Sequence s holds first rows and gets n: its entries first / P .. (first + n - 1) / P that name no page take the next pages
// of the free ring, in the order of the sequences (so that a sequence needs to know how many the ones before it take); the
// pages of ended sequences go behind the ring's last.  Then token j's slot is its row's page times P and the row's place in
// it, its position first + j, or first + its depth in a tree, whose mask is its own bit and its parent's mask.
//
// Three launches, each of which needs all that the one before it found: plan_count (a wave per sequence: what it needs
// and gives back), plan_fill (a wave per sequence: sums over the sequences before it, its entries), plan_tokens (a thread per
// token) or plan_trees (a work-group per sequence, its parents in LDS, where each token walks up to its root).
#include "ebd.h"
#include "ebd_internal.hpp"
#include "paged_device.hpp"

#include <algorithm>

namespace ebd {

namespace {

constexpr int kPlanThreads = 256;
constexpr int kPlanWaves = kPlanThreads / 64;
constexpr int kTreeMost = 64 * 64;       // tokens of a tree: mask_words times 64
constexpr int64_t kRowsHeld = (int64_t)1 << 30;

__device__ __forceinline__ bool in_pool(const ebd_plan_step_params &p, int page) {
  return (uint32_t)page < (uint32_t)p.num_pages;
}

// What a sequence gets: its new tokens n (-1: it has ended), the rows it holds, and the entries of its new rows.
struct Request {
  int n, first;
  int e0, e1;     // entries e0 .. e1 - 1, as far as the table goes
  uint32_t status;
};
__device__ __forceinline__ Request request(const ebd_plan_step_params &p, int shift, int count, int len) {
  Request q;
  q.n = count < 0 ? -1 : count;
  q.first = max(len, 0);
  q.status = 0;
  if (q.n > 0 && (int64_t)q.first + q.n > kRowsHeld) q.n = 0, q.status = EBD_ST_BAD_LAYOUT;
  q.e0 = q.e1 = 0;
  if (q.n > 0) {
    q.e0 = q.first >> shift;
    const int end = ((q.first + q.n - 1) >> shift) + 1;
    q.e1 = min(end, p.max_pages);
    if (end > p.max_pages) q.status |= EBD_ST_BAD_PAGE;
  }
  return q;
}

struct FreePages {
  int head, count;
};
__device__ __forceinline__ FreePages free_pages(const ebd_plan_step_params &p, int head, int count) {
  const bool ok = (uint32_t)head < (uint32_t)p.num_pages && count >= 0 && count <= p.num_pages;
  return ok ? FreePages{head, count} : FreePages{0, 0};
}
// The i'th place of the ring behind its head, i < 2 num_pages.
__device__ __forceinline__ int ring_at(const ebd_plan_step_params &p, int head, int64_t i) {
  int64_t at = head + i;
  at -= at >= p.num_pages ? p.num_pages : 0;
  at -= at >= p.num_pages ? p.num_pages : 0;
  return (int)at;
}

__device__ __forceinline__ int64_t wave_sum64(int64_t x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// Slot of row `row` of sequence s, or -1.
__device__ __forceinline__ int64_t slot_of(const ebd_plan_step_params &p, int shift, int s, int row) {
  const int e = row >> shift;
  if (e >= p.max_pages) return -1;
  const int pg = p.page_table[(int64_t)s * p.max_pages + e];
  return in_pool(p, pg) ? ((int64_t)pg << shift) + (row & (p.page_size - 1)) : -1;
}

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void plan_count_kernel(PlanStepLaunch L) {
  const ebd_plan_step_params &p = L.p;
  const int s = blockIdx.x * kPlanWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const FreePages f = free_pages(p, p.free_state[0], p.free_state[1]);
    *L.state = make_int2(f.head, f.count);
  }
  if (s >= p.num_seqs) return;
  const Request q = request(p, L.shift, p.count[s], p.len[s]);
  const int32_t *row = p.page_table + (int64_t)s * p.max_pages;
  const int e0 = q.n < 0 ? 0 : q.e0, e1 = q.n < 0 ? p.max_pages : q.e1;
  int found = 0;  // entries without a page, or (ended) with one
  for (int e = e0 + lane; e < e1; e += 64) found += in_pool(p, row[e]) == (q.n < 0);
  found = wave_sum(found);
  if (lane == 0) {
    L.info[s] = make_int4(q.n, q.first, q.n < 0 ? 0 : found, q.n < 0 ? found : 0);
    if (q.status && L.status) atomicOr(&L.status[s], q.status);
  }
}

__global__ __launch_bounds__(kPlanThreads) void plan_fill_kernel(PlanStepLaunch L) {
  __shared__ int64_t sums[kPlanWaves][3];
  const ebd_plan_step_params &p = L.p;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, s0 = blockIdx.x * kPlanWaves, s = s0 + wave;
  // tokens, pages taken and pages given back by the sequences before this one
  int64_t t = 0, take = 0, back = 0;
  for (int i = threadIdx.x; i < s0; i += kPlanThreads) {
    const int4 v = L.info[i];
    t += max(v.x, 0), take += v.z, back += v.w;
  }
  t = wave_sum64(t), take = wave_sum64(take), back = wave_sum64(back);
  if (lane == 0) sums[wave][0] = t, sums[wave][1] = take, sums[wave][2] = back;
  __syncthreads();
  t = take = back = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) t += sums[w][0], take += sums[w][1], back += sums[w][2];
  for (int i = s0; i < s && i < p.num_seqs; ++i) {
    const int4 v = L.info[i];
    t += max(v.x, 0), take += v.z, back += v.w;
  }
  if (s >= p.num_seqs) return;
  const int4 me = L.info[s];
  const int2 f = *L.state;
  const int n = max(me.x, 0);
  if (lane == 0) {
    p.new_off[s] = t;
    if (me.x != 0) p.len[s] = me.x < 0 ? 0 : me.y + n;
    const bool beyond = t + n > p.num_tokens && n > 0 && (p.slots || p.pos || p.mask);
    if (beyond && L.status) atomicOr(&L.status[s], EBD_ST_BAD_LAYOUT);
    if (s == p.num_seqs - 1) {
      p.new_off[s + 1] = t + n;
      const int64_t taken = min(take + me.z, (int64_t)f.y);
      p.free_state[0] = ring_at(p, f.x, taken);
      p.free_state[1] = (int)min(f.y - taken + back + me.w, (int64_t)p.num_pages);
    }
  }
  int32_t *row = p.page_table + (int64_t)s * p.max_pages;
  if (me.x < 0) {
    for (int base = 0; base < p.max_pages; base += 64) {
      const int e = base + lane;
      const int pg = e < p.max_pages ? row[e] : -1;
      const uint64_t has = __ballot(in_pool(p, pg));
      const int64_t at = f.y + back + __popcll(has & ((1ull << lane) - 1));
      if (in_pool(p, pg) && at < p.num_pages) p.free_pages[ring_at(p, f.x, at)] = pg;
      if (e < p.max_pages && pg != -1) row[e] = -1;
      back += __popcll(has);
    }
    return;
  }
  if (me.z == 0) return;
  const int e0 = me.y >> L.shift, e1 = min(((me.y + n - 1) >> L.shift) + 1, p.max_pages);
  bool none = false;
  for (int base = e0; base < e1; base += 64) {
    const int e = base + lane;
    const bool hole = e < e1 && !in_pool(p, row[e]);
    const uint64_t holes = __ballot(hole);
    const int64_t at = take + __popcll(holes & ((1ull << lane) - 1));
    if (hole && at < f.y) row[e] = p.free_pages[ring_at(p, f.x, at)];
    none |= hole && at >= f.y;
    take += __popcll(holes);
  }
  if (__any(none) && lane == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
}

__global__ __launch_bounds__(kPlanThreads) void plan_tokens_kernel(PlanStepLaunch L) {
  const ebd_plan_step_params &p = L.p;
  const int64_t t = (int64_t)blockIdx.x * kPlanThreads + threadIdx.x;
  if (t >= p.num_tokens) return;
  // the last sequence whose first token is not behind t (those without tokens start where the next one does)
  int lo = 0, hi = p.num_seqs;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.new_off[mid + 1] <= t) lo = mid + 1;
    else hi = mid;
  }
  int64_t slot = -1;
  int pos = -1;
  if (lo < p.num_seqs) {
    pos = L.info[lo].y + (int)(t - p.new_off[lo]);
    slot = slot_of(p, L.shift, lo, pos);
  }
  if (p.slots) p.slots[t] = slot;
  if (p.pos) p.pos[t] = pos;
}

// Work-group s < num_seqs: the tokens of sequence s; the ones behind those: padding.
__global__ __launch_bounds__(kPlanThreads) void plan_trees_kernel(PlanStepLaunch L) {
  __shared__ int32_t parent[kTreeMost];
  const ebd_plan_step_params &p = L.p;
  const int s = blockIdx.x, W = p.mask_words;
  if (s >= p.num_seqs) {
    const int64_t step = (int64_t)(gridDim.x - p.num_seqs) * kPlanThreads;
    for (int64_t t = p.new_off[p.num_seqs] + (int64_t)(s - p.num_seqs) * kPlanThreads + threadIdx.x; t < p.num_tokens; t += step) {
      if (p.slots) p.slots[t] = -1;
      if (p.pos) p.pos[t] = -1;
      for (int w = 0; w < W; ++w) p.mask[t * W + w] = 0;
    }
    return;
  }
  const int64_t t0 = p.new_off[s];
  const int first = L.info[s].y, all = max(L.info[s].x, 0);
  const int n = (int)max((int64_t)0, min((int64_t)all, p.num_tokens - t0)), in = min(n, 64 * W);
  bool bad = n > in;
  for (int j = threadIdx.x; j < in; j += kPlanThreads) {
    int up = p.parent[t0 + j];
    if (up < -1 || up >= j) up = -1, bad = true;
    parent[j] = up;
  }
  if (__any(bad) && (threadIdx.x & 63) == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_LAYOUT);
  __syncthreads();
  for (int j = threadIdx.x; j < n; j += kPlanThreads) {
    uint64_t *mask = p.mask + (t0 + j) * W;
    int depth = 0;
    if (j < in) {
      // words from the last down to the one a bit falls into are finished: parents come before their children
      int w = W - 1;
      uint64_t bits = 0;
      for (int i = j; i >= 0; i = parent[i], ++depth) {
        for (; w > i >> 6; --w, bits = 0) mask[w] = bits;
        bits |= 1ull << (i & 63);
      }
      for (; w >= 0; --w, bits = 0) mask[w] = bits;
    } else {
      for (int w = 0; w < W; ++w) mask[w] = 0;
    }
    if (p.pos) p.pos[t0 + j] = j < in ? first + depth - 1 : -1;
    if (p.slots) p.slots[t0 + j] = slot_of(p, L.shift, s, first + j);
  }
}

size_t plan_step_bytes(const ebd_plan_step_params &p) { return 256 + (size_t)p.num_seqs * sizeof(int4); }

hipError_t launch_plan_step(const PlanStepLaunch &L, hipStream_t s) {
  const ebd_plan_step_params &p = L.p;
  const dim3 block(kPlanThreads), seqs((unsigned)((p.num_seqs + kPlanWaves - 1) / kPlanWaves));
  hipLaunchKernelGGL(plan_count_kernel, seqs, block, 0, s, L);
  hipLaunchKernelGGL(plan_fill_kernel, seqs, block, 0, s, L);
  if (p.num_tokens > 0 && p.parent) {
    hipLaunchKernelGGL(plan_trees_kernel, dim3((unsigned)p.num_seqs + 4), block, 0, s, L);
  } else if (p.num_tokens > 0 && (p.slots || p.pos)) {
    hipLaunchKernelGGL(plan_tokens_kernel, dim3((unsigned)((p.num_tokens + kPlanThreads - 1) / kPlanThreads)), block, 0, s, L);
  }
  return hipGetLastError();
}

}  // namespace ebd
