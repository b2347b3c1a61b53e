// plan_step.hip -- page tables, slots, positions and tree masks of a serving step, from the sequences' new token counts.
//
// Sequence s holds first rows and gets n: its entries first / P .. (first + n - 1) / P that name no page take the next pages
// of the free ring, in the order of the sequences (so that a sequence needs to know how many the ones before it take); the
// pages of ended sequences go behind the ring's last.  Then token j's slot is its row's page times P and the row's place in
// it, its position first + j, or first + its depth in a tree, whose mask is its own bit and its parent's mask.
//
// Few sequences: one launch (plan_one).  Others: three, each of which needs all that the one before it found: plan_count (a
// wave per sequence: what it needs and gives back), plan_fill (a wave per sequence: sums over the sequences before it, its
// entries), plan_tokens (a thread per token) or plan_trees (a work-group per sequence, its parents in LDS, where each token
// walks up to its root).  Latency bounds a step of some hundred sequences and shallow trees: 512 sequences and 66 thousand
// tokens, 1.1 MB read and written, 6.3 + 9.6 + 4.1 us.  Two parts grow faster than the step.  Each work-group of plan_fill adds
// up all sequences before its own: 512 sequences of one token 9 us, 4096 13, 16384 69, 65536 764.  And a walk is as long as its
// token is deep, so that chains are quadratic: of 4096 tokens 1200 us in one launch and 3150 in three (as random trees 155 and
// 164), two of 512 beside 62 trees of 30 58 (14).
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

// f(entry, its page, whether there is such an entry) for the entries e0 .. e1 - 1 of a sequence, in order, 64 at a time by a
// wave's lanes, 512 of them in flight (512 sequences, of which 20 with 2049 entries have ended, with the copy that puts the tables
// back, 3 us: 34.1 in all one by one, 22.8 so).
template <class F>
__device__ __forceinline__ void scan(const int32_t *row, int e0, int e1, const F &f) {
  constexpr int kFlight = 8;
  const int lane = threadIdx.x & 63;
  for (int base = e0; base < e1; base += 64 * kFlight) {
    int pg[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      const int e = base + 64 * k + lane;
      pg[k] = -1;
      if (e < e1) pg[k] = row[e];
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k)
      if (base + 64 * k < e1) f(base + 64 * k + lane, pg[k], base + 64 * k + lane < e1);
  }
}

// Slot of row `row` of sequence s, or -1.
__device__ __forceinline__ int64_t slot_of(const ebd_plan_step_params &p, int shift, int s, int row) {
  const int e = row >> shift;
  if (e >= p.max_pages) return -1;
  const int pg = p.page_table[(int64_t)s * p.max_pages + e];
  return in_pool(p, pg) ? ((int64_t)pg << shift) + (row & (p.page_size - 1)) : -1;
}

// A wave fills sequence s's entries: holes from the ring's `take`'th page on, or (n < 0: ended) its pages to the ring, from
// the `back`'th place behind its last; whether a hole is left.
__device__ __forceinline__ bool fill(const ebd_plan_step_params &p, const FreePages &f, int s, int n, int first, int shift,
                                     int64_t take, int64_t back) {
  const uint64_t below = (1ull << (threadIdx.x & 63)) - 1;
  int32_t *row = p.page_table + (int64_t)s * p.max_pages;
  if (n < 0) {
    scan(row, 0, p.max_pages, [&](int e, int pg, bool here) {
      const uint64_t has = __ballot(here && in_pool(p, pg));
      const int64_t at = f.count + back + __popcll(has & below);
      if (here && in_pool(p, pg) && at < p.num_pages) p.free_pages[ring_at(p, f.head, at)] = pg;
      if (here && pg != -1) row[e] = -1;
      back += __popcll(has);
    });
    return false;
  }
  bool none = false;
  if (n > 0) {
    scan(row, first >> shift, min(((first + n - 1) >> shift) + 1, p.max_pages), [&](int e, int pg, bool here) {
      const bool hole = here && !in_pool(p, pg);
      const uint64_t holes = __ballot(hole);
      const int64_t at = take + __popcll(holes & below);
      const int got = hole && at < f.count ? p.free_pages[ring_at(p, f.head, at)] : -1;
      if (hole && at < f.count) row[e] = got;
      none |= hole && !in_pool(p, got);
      take += __popcll(holes);
    });
  }
  return __any(none);
}

// The state behind the step.
__device__ __forceinline__ void finish(const ebd_plan_step_params &p, const FreePages &f, int64_t take, int64_t back) {
  const int64_t taken = min(take, (int64_t)f.count);
  p.free_state[0] = ring_at(p, f.head, taken);
  p.free_state[1] = (int)min(f.count - taken + back, (int64_t)p.num_pages);
}

// Position and mask of token j of a tree, whose parents are in LDS; its depth.
__device__ __forceinline__ int walk(const int32_t *parent, int j, uint64_t *mask, int W) {
  // words from the last down to the one a bit falls into are finished: parents come before their children
  int w = W - 1, depth = 0;
  uint64_t bits = 0;
  for (int i = j; i >= 0; i = parent[i], ++depth) {
    for (; w > i >> 6; --w, bits = 0) mask[w] = bits;
    bits |= 1ull << (i & 63);
  }
  for (; w >= 0; --w, bits = 0) mask[w] = bits;
  return depth - 1;
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
  scan(row, e0, e1, [&](int, int pg, bool here) { found += here && in_pool(p, pg) == (q.n < 0); });
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
  if (p.num_seqs == 0 && threadIdx.x == 0) p.new_off[0] = 0;
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
  const FreePages f = {L.state->x, L.state->y};
  const int n = max(me.x, 0);
  if (lane == 0) {
    p.new_off[s] = t;
    if (me.x != 0) p.len[s] = me.x < 0 ? 0 : me.y + n;
    const bool beyond = t + n > p.num_tokens && n > 0 && (p.slots || p.pos || p.mask);
    if (beyond && L.status) atomicOr(&L.status[s], EBD_ST_BAD_LAYOUT);
    if (s == p.num_seqs - 1) {
      p.new_off[s + 1] = t + n;
      finish(p, f, take + me.z, back + me.w);
    }
  }
  const bool none = fill(p, f, s, me.x, me.y, L.shift, take, back);
  if (none && lane == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
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
      depth = walk(parent, j, mask, W);
    } else {
      for (int w = 0; w < W; ++w) mask[w] = 0;
    }
    if (p.pos) p.pos[t0 + j] = j < in ? first + depth : -1;
    if (p.slots) p.slots[t0 + j] = slot_of(p, L.shift, s, first + j);
  }
}

// All of it by one work-group, for up to 128 sequences, of which eight lanes each take the entries, and four tokens a thread.
// us by one launch / by three: 64 sequences of one token 5.0 / 9.7, 64 trees of 30 6.4 / 9.5, 128 trees of 15 7.2 / 9.6, of 30
// 9.2 / 9.6, 16 of 130 8.2 / 9.5.  Not taken: one sequence of 4000 tokens in pages of 16, whose 250 entries eight lanes would
// take, 14.6 / 10.0; 256 sequences of one token, by a version that takes sequences in turns, 10.5 / 9.8; tables of many
// entries, which a wave each gives back when their sequences end, 64 of 8200 163 / 39.
constexpr int kOneThreads = 1024;
constexpr int kOneLanes = 8;
constexpr int kOneSeqs = kOneThreads / kOneLanes;
constexpr int kOneTokens = 4;
constexpr int64_t kOneEntries = (int64_t)1 << 17;  // of all sequences' tables
constexpr int64_t kOnePages = 128;                // of a sequence's new rows
__global__ __launch_bounds__(kOneThreads) void plan_one_kernel(PlanStepLaunch L) {
  __shared__ int new_of[kOneSeqs], first_of[kOneSeqs], take_of[kOneSeqs], back_of[kOneSeqs];
  __shared__ int64_t off[kOneSeqs + 1];
  __shared__ int32_t parent[kOneThreads * kOneTokens];
  const ebd_plan_step_params &p = L.p;
  const int S = p.num_seqs, me = threadIdx.x, lane = me & 63, wave = me >> 6, s = me / kOneLanes, own = lane % kOneLanes;
  int32_t up[kOneTokens];  // asked for first, used last
#pragma unroll
  for (int k = 0; k < kOneTokens; ++k) {
    const int t = me + k * kOneThreads;
    up[k] = -1;
    if (p.parent && t < p.num_tokens) up[k] = p.parent[t];
  }
  const FreePages f = free_pages(p, p.free_state[0], p.free_state[1]);
  // eight lanes' sequence: what it needs; a wave for what an ended one gives back
  Request q = {0, 0, 0, 0, 0};
  if (s < S) q = request(p, L.shift, p.count[s], p.len[s]);
  int32_t *row = p.page_table + (int64_t)s * p.max_pages;
  int found = 0;
  for (int e = q.e0 + own; e < q.e1; e += kOneLanes) found += !in_pool(p, row[e]);
#pragma unroll
  for (int o = kOneLanes / 2; o; o >>= 1) found += __shfl_xor(found, o);
  if (own == 0) new_of[s] = q.n, first_of[s] = q.first, take_of[s] = found, back_of[s] = 0;
  const uint64_t ended = __ballot(own == 0 && q.n < 0);
  for (uint64_t rest = ended; rest; rest &= rest - 1) {
    const int e = (64 * wave + __builtin_ctzll(rest)) / kOneLanes;
    int held = 0;
    scan(p.page_table + (int64_t)e * p.max_pages, 0, p.max_pages, [&](int, int pg, bool here) { held += here && in_pool(p, pg); });
    held = wave_sum(held);
    if (lane == 0) back_of[e] = held;
  }
  __syncthreads();
  if (wave == 0) {  // the sums over the sequences before each (counts pass 32 bits, pages do not)
    static_assert(kOneSeqs == 128, "two sequences a lane");
    const int a = 2 * lane, b = a + 1, n0 = max(new_of[a], 0), t0 = take_of[a], b0 = back_of[a];
    int64_t upto = (int64_t)n0 + max(new_of[b], 0);
    int take = t0 + take_of[b], back = b0 + back_of[b];
    const int64_t n2 = upto;
    const int t2 = take, b2 = back;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int64_t x = __shfl_up(upto, o);
      const int y = __shfl_up(take, o), z = __shfl_up(back, o);
      if (lane >= o) upto += x, take += y, back += z;
    }
    if (lane == 0) off[0] = 0, p.new_off[0] = 0;
    if (lane == 63) finish(p, f, take, back);  // (sequences that are not there take and give nothing)
    const int64_t before = upto - n2;
    off[a + 1] = before + n0, off[b + 1] = upto;
    if (a < S) p.new_off[a + 1] = before + n0;
    if (b < S) p.new_off[b + 1] = upto;
    take_of[a] = take - t2, take_of[b] = take - t2 + t0;
    back_of[a] = back - b2, back_of[b] = back - b2 + b0;
  }
  __syncthreads();
  if (own == 0 && s < S) {
    if (q.n != 0) p.len[s] = q.n < 0 ? 0 : q.first + q.n;
    if (off[s + 1] > p.num_tokens && q.n > 0 && (p.slots || p.pos || p.mask)) q.status |= EBD_ST_BAD_LAYOUT;
    if (q.status && L.status) atomicOr(&L.status[s], q.status);
  }
  bool none = false;
  int take = take_of[s];
  for (int base = q.e0; base < q.e1; base += kOneLanes) {
    const int e = base + own;
    const bool hole = e < q.e1 && !in_pool(p, row[e]);
    const uint32_t holes = (uint32_t)(__ballot(hole) >> (lane - own)) & ((1u << kOneLanes) - 1u);
    const int at = take + __popc(holes & ((1u << own) - 1u));
    const int got = hole && at < f.count ? p.free_pages[ring_at(p, f.head, at)] : -1;
    if (hole && at < f.count) row[e] = got;
    none |= hole && !in_pool(p, got);
    take += __popc(holes);
  }
  if (none && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  for (uint64_t rest = ended; rest; rest &= rest - 1) {
    const int e = (64 * wave + __builtin_ctzll(rest)) / kOneLanes;
    fill(p, f, e, -1, 0, L.shift, 0, back_of[e]);
  }
  __syncthreads();  // the entries are written
  int seq[kOneTokens];
#pragma unroll
  for (int k = 0; k < kOneTokens; ++k) {
    const int t = me + k * kOneThreads;
    int lo = 0, hi = S;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (off[mid + 1] <= t) lo = mid + 1;
      else hi = mid;
    }
    seq[k] = t < p.num_tokens ? lo : S;
    if (p.mask && seq[k] < S) {
      const int j = t - (int)off[lo];
      const bool bad = j >= 64 * p.mask_words || up[k] < -1 || up[k] >= j;
      if (bad && L.status) atomicOr(&L.status[lo], EBD_ST_BAD_LAYOUT);
      parent[t] = bad ? -1 : up[k];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kOneTokens; ++k) {
    const int t = me + k * kOneThreads, u = seq[k];
    if (t >= p.num_tokens) break;
    const int t0 = u < S ? (int)off[u] : 0, j = t - t0, at = u < S ? first_of[u] + j : -1;
    int pos = at;
    if (p.mask) {
      uint64_t *mask = p.mask + (int64_t)t * p.mask_words;
      if (u < S && j < 64 * p.mask_words) {
        pos = first_of[u] + walk(parent + t0, j, mask, p.mask_words);
      } else {
        pos = -1;
        for (int w = 0; w < p.mask_words; ++w) mask[w] = 0;
      }
    }
    if (p.pos) p.pos[t] = pos;
    if (p.slots) p.slots[t] = u < S ? slot_of(p, L.shift, u, at) : -1;
  }
}

size_t plan_step_bytes(const ebd_plan_step_params &p) { return 256 + (size_t)p.num_seqs * sizeof(int4); }

hipError_t launch_plan_step(const PlanStepLaunch &L, hipStream_t s) {
  const ebd_plan_step_params &p = L.p;
  if (p.num_seqs <= kOneSeqs && p.num_tokens <= kOneThreads * kOneTokens &&
      p.num_tokens <= kOnePages * p.page_size && (int64_t)p.num_seqs * p.max_pages <= kOneEntries) {
    hipLaunchKernelGGL(plan_one_kernel, dim3(1), dim3(kOneThreads), 0, s, L);
    return hipGetLastError();
  }
  const dim3 block(kPlanThreads), seqs((unsigned)std::max(1, (p.num_seqs + kPlanWaves - 1) / kPlanWaves));
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
