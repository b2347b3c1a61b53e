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
#include "paged_device.hpp"

#include <algorithm>

namespace ebd {

namespace {

constexpr int kRopeRows = 128;  // most rows of a work-group: 8 lanes each

// cos and sin (times the amplitude) of pair `i` at position `pos`.
__device__ __forceinline__ float2 turn(const ebd_rotary &R, int i, int64_t pos) {
  const double t = (double)pos * R.freq[i] * 0.15915494309189535;  // 1 / 2 pi
  float s, c;
  sincospif(2.0f * (float)(t - rint(t)), &s, &c);
  if (R.flags & EBD_ROPE_INVERSE) s = -s;
  return make_float2(R.amplitude * c, R.amplitude * s);
}

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

// How the eight lanes of a row split it: lane l's two 16-byte chunks (elements), and whether the second
// elements of the first chunk's pairs are the second chunk (halves), which needs rot_dim / 2 to be whole
// chunks.  Other halves go element by element (kOdd).
enum { kCopy, kHalf, kPairs, kOdd };
struct Split {
  int how, e0, e1;
};
__device__ __forceinline__ Split split_row(const ebd_rotary &R, int l, bool rotated) {
  if (!rotated || !R.freq) return {kCopy, 16 * l, 16 * l + 8};
  if (R.layout == EBD_ROPE_PAIRS) return {kPairs, 16 * l, 16 * l + 8};
  if (R.rot_dim % 16) return {kOdd, 0, 0};
  if (16 * l < R.rot_dim) return {kHalf, 8 * l, R.rot_dim / 2 + 8 * l};
  return {kCopy, 16 * l, 16 * l + 8};
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

// Rows are read once, so that they leave no trace in the caches (8191 tokens of 32 rows 31.2 -> 28.9 us, append of 13k
// tokens of 36 rows 53 -> 52); what is written stays there for the attention that reads it next.
__device__ __forceinline__ uint4 load16(const uint16_t *p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
}
__device__ __forceinline__ void store16(uint16_t *p, const uint4 &v) { *reinterpret_cast<uint4 *>(p) = v; }

}  // namespace

// Work-group (token group, block of rows): `per` threads, whole waves, for each of up to four tokens.  A dimension of the
// grid holds fewer than 2^32 threads, which 2^24 tokens of up to 1024 pass, so token groups fill x and go on in z.
constexpr int kAcross = 1 << 21;
__device__ __forceinline__ int64_t token_group(int x, int z) { return (int64_t)z * kAcross + x; }
__device__ __forceinline__ int token_slot(int per) {
  const int t = threadIdx.x;
  return (t >= per) + (t >= 2 * per) + (t >= 3 * per);
}

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

namespace {
// Threads of a token and tokens of a work-group.
void cut(int64_t rows, int32_t *per, int32_t *tpb) {
  *per = (int32_t)((std::min<int64_t>(rows, kRopeRows) * 8 + 63) / 64 * 64);
  *tpb = std::max(1, std::min(4, 256 / *per));
}
dim3 rope_grid(int64_t tokens, int64_t rows, int tpb) {
  const int64_t groups = (tokens + tpb - 1) / tpb;
  return dim3((unsigned)std::min<int64_t>(groups, kAcross), (unsigned)((rows + kRopeRows - 1) / kRopeRows),
              (unsigned)((groups + kAcross - 1) / kAcross));
}
}  // namespace

hipError_t launch_rope(RopeLaunch L, hipStream_t s) {
  cut(L.p.num_heads, &L.per, &L.tpb);
  hipLaunchKernelGGL(rope_kernel, rope_grid(L.p.num_tokens, L.p.num_heads, L.tpb), dim3(L.per * L.tpb), 0, s, L);
  return hipGetLastError();
}

hipError_t launch_append_paged(AppendPagedLaunch L, hipStream_t s) {
  const int64_t rows = 2 * (int64_t)L.p.pages.kv_heads + L.p.q_heads;
  cut(rows, &L.per, &L.tpb);
  hipLaunchKernelGGL(append_paged_kernel, rope_grid(L.p.num_tokens, rows, L.tpb), dim3(L.per * L.tpb), 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
