// rope.hip -- rotary positions, and the append of new tokens to a paged cache with the rotation on the way.
//
// Pair i of a row at position pos is turned by the angle pos freq_i:
//   y1 = a (x1 cos - x2 sin),  y2 = a (x2 cos + x1 sin).
// The angle is taken in turns, pos freq_i / 2 pi, in 64 bits, and only its distance to the nearest whole
// turn (exact in 64 bits, below 1/2) becomes fp32, so that a position of a million costs no accuracy.  cos
// and sin are made once per token and work-group, by one lane per pair, and shared by its rows through LDS.
//
// Both kernels read and write each row once: the memory's rate bounds large calls, the chain of dependent
// loads (sequence, length, page, row) small ones.  Eight lanes take a row, 32 bytes each in two 16-byte
// accesses that hold both elements of its pairs.  A work-group has as many waves as a token's rows need (up to 128 of
// them), so that a token's sines are made once, by one wave's worth of work, and no lane idles over rows that are not
// there; tokens of few rows share a work-group.
#include "ebd.h"
#include "ebd_internal.hpp"
#include "rope_device.hpp"

namespace ebd {

namespace {

// Eight pairs whose first elements are in a and second ones in b.
__device__ __forceinline__ void rotate8(uint4 &a, uint4 &b, const float2 *cs) {
  uint32_t *pa = &a.x, *pb = &b.x;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float a0 = bf16_lo(pa[w]), a1 = bf16_hi(pa[w]), b0 = bf16_lo(pb[w]), b1 = bf16_hi(pb[w]);
    const float2 t0 = cs[2 * w], t1 = cs[2 * w + 1];
    pa[w] = pack_bf16(a0 * t0.x - b0 * t0.y, a1 * t1.x - b1 * t1.y);
    pb[w] = pack_bf16(b0 * t0.x + a0 * t0.y, b1 * t1.x + a1 * t1.y);
  }
}

// Four neighbouring pairs (one per 32-bit word), those from `n` on copied.
__device__ __forceinline__ void rotate_pairs(uint4 &a, const float2 *cs, int n) {
  uint32_t *p = &a.x;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float x = bf16_lo(p[w]), y = bf16_hi(p[w]);
    const float2 t = cs[w];
    const uint32_t r = pack_bf16(x * t.x - y * t.y, y * t.x + x * t.y);
    p[w] = w < n ? r : p[w];
  }
}

// A rotary half that is no multiple of eight elements: lane l takes every eighth pair, then every eighth
// of the elements behind them (8191 tokens of 32 rows, 34 of their elements rotated: 62 us, 64 of them 32).
__device__ __forceinline__ void rotate_odd(const ebd_rotary &R, const uint16_t *x, uint16_t *y,
                                           const float2 *cs, int l) {
  const int n = R.rot_dim / 2;
  for (int i = l; i < n; i += 8) {
    const float a = bf16_lo(x[i]), b = bf16_lo(x[i + n]);
    const uint32_t r = pack_bf16(a * cs[i].x - b * cs[i].y, b * cs[i].x + a * cs[i].y);
    y[i] = (uint16_t)r;
    y[i + n] = (uint16_t)(r >> 16);
  }
  for (int i = R.rot_dim + l; i < kHeadDim; i += 8) y[i] = x[i];
}

__device__ __forceinline__ void turn_row(const ebd_rotary &R, const Split &S, uint4 &a, uint4 &b,
                                         const float2 *cs) {
  if (S.how == kHalf) rotate8(a, b, cs + S.e0);
  if (S.how == kPairs) {
    const int i = S.e0 / 2, n = R.rot_dim / 2;
    rotate_pairs(a, cs + i, n - i);
    rotate_pairs(b, cs + i + 4, n - i - 4);
  }
}

}  // namespace

__global__ __launch_bounds__(8 * kRopeRows) void rope_kernel(RopeLaunch L) {
  __shared__ float2 cs[4][kHeadDim / 2];
  const ebd_rope_params &p = L.p;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per;
  const int64_t t = token_group(blockIdx.x, blockIdx.z) * L.tpb + slot;
  const int h = blockIdx.y * kRopeRows + i / 8;
  const bool live = t < p.num_tokens && h < p.num_heads;
  const Split sp = split_row(p.rot, i % 8, true);
  const uint16_t *x = L.x + t * p.x.token_stride + h * p.x.head_stride;
  uint16_t *y = L.y + t * p.y.token_stride + h * p.y.head_stride;
  uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
  if (live && sp.how != kOdd) {
    a = load16(x + sp.e0);
    b = load16(x + sp.e1);
  }
  if (t < p.num_tokens && i < p.rot.rot_dim / 2) cs[slot][i] = turn(p.rot, i, p.pos[t]);
  __syncthreads();
  if (!live) return;
  if (sp.how == kOdd) {
    rotate_odd(p.rot, x, y, cs[slot], i % 8);
    return;
  }
  turn_row(p.rot, sp, a, b, cs[slot]);
  store16(y + sp.e0, a);
  store16(y + sp.e1, b);
}

// Rows of a token in order: its keys, its queries, its values.
__global__ __launch_bounds__(8 * kRopeRows) void append_paged_kernel(AppendPagedLaunch L) {
  __shared__ float2 cs[4][kHeadDim / 2];
  const ebd_append_paged_params &p = L.p;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per;
  const int64_t t = token_group(blockIdx.x, blockIdx.z) * L.tpb + slot;
  const int row = blockIdx.y * kRopeRows + i / 8;
  const int kv = p.pages.kv_heads, S = p.pages.num_seqs;
  const bool isk = row < kv, isq = !isk && row < kv + p.q_heads;
  const bool here = t < p.num_tokens && row < 2 * kv + p.q_heads;
  const int h = isk ? row : (isq ? row - kv : row - kv - p.q_heads);
  const Split sp = split_row(p.rot, i % 8, isk || isq);
  const ebd_rows &in = isq ? p.q_rows : (isk ? p.k_rows : p.v_rows);
  const uint16_t *x = (isq ? L.q : (isk ? L.k_new : L.v_new)) + t * in.token_stride + h * in.head_stride;
  uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
  if (here && sp.how != kOdd) {  // asked for before the token's place is known
    a = load16(x + sp.e0);
    b = load16(x + sp.e1);
  }
  // the wave's token: its sequence, row and page
  const int s = t < p.num_tokens ? find_seq(p.new_off, S, t) : -1;
  const bool live = here && s >= 0;
  int64_t base = -1;
  if (s >= 0) {
    const int64_t r = (int64_t)p.len[s] - p.new_off[s + 1] + t;
    if (p.rot.freq && i < p.rot.rot_dim / 2) cs[slot][i] = turn(p.rot, i, p.pos ? p.pos[t] : r);
    base = page_row(p.pages, L.shift, s, r);
    if (base < 0 && i == 0 && blockIdx.y == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  }
  __syncthreads();
  if (!live || (!isq && base < 0)) return;
  uint16_t *y = isq ? L.q_out + t * p.q_out_rows.token_stride + h * p.q_out_rows.head_stride
                    : (isk ? L.K : L.V) + base + h * p.pages.head_stride;
  if (sp.how == kOdd) {
    rotate_odd(p.rot, x, y, cs[slot], i % 8);
    return;
  }
  turn_row(p.rot, sp, a, b, cs[slot]);
  store16(y + sp.e0, a);
  store16(y + sp.e1, b);
}

hipError_t launch_rope(RopeLaunch L, hipStream_t s) {
  cut_tokens(L.p.num_heads, &L.per, &L.tpb);
  hipLaunchKernelGGL(rope_kernel, rope_grid(L.p.num_tokens, L.p.num_heads, L.tpb), dim3(L.per * L.tpb), 0, s, L);
  return hipGetLastError();
}

hipError_t launch_append_paged(AppendPagedLaunch L, hipStream_t s) {
  const int64_t rows = 2 * (int64_t)L.p.pages.kv_heads + L.p.q_heads;
  cut_tokens(rows, &L.per, &L.tpb);
  hipLaunchKernelGGL(append_paged_kernel, rope_grid(L.p.num_tokens, rows, L.tpb), dim3(L.per * L.tpb), 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
