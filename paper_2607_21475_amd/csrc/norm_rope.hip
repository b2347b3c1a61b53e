// norm_rope.hip -- norms of heads with the rotary positions in the same pass, forward and backward, and the append of
// new tokens to a paged cache with both on the way.
//
// A row x of 128 elements at position pos, its head's weights w, the rotation R (rope_device.hpp):
//   y = R (r w x),  r = 1 / sqrt(mean x^2 + eps)
// and from dy, with g = R^T dy (pairs turned back), h = g w, n = r x:
//   dx = r (h - n mean(h n)),  dw = sum g n over the rows that share w.
//
// Eight lanes take a row, 16 elements each: as the rotation pairs them (rope_device.hpp), so that norm, rotation and
// gradients stay in registers and a row's sums are three exchanges between neighbouring lanes.  All steps are fp32, and an
// output is rounded once.  Each row is read and written once: memory bounds large calls, a chain of loads small ones.
#include "ebd.h"
#include "ebd_internal.hpp"
#include "rope_device.hpp"

namespace ebd {

namespace {

// A lane's two chunks of a row.
struct Part {
  float a[8], b[8];
};

// As split_row, but where halves are no whole chunks, each lane takes neighbouring ones, and the pairs meet in LDS.
__device__ __forceinline__ Split part_of(const ebd_rotary &R, int l, bool rotated) {
  Split sp = split_row(R, l, rotated);
  if (sp.how == kOdd) sp.e0 = 16 * l, sp.e1 = 16 * l + 8;
  return sp;
}

__device__ __forceinline__ void unpack8(const uint4 &v, float (&x)[8]) {
  const uint32_t *p = &v.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(p[i]), x[2 * i + 1] = bf16_hi(p[i]);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ Part load_row(const Split &S, const uint16_t *p) {
  Part x;
  unpack8(load16(p + S.e0), x.a);
  unpack8(load16(p + S.e1), x.b);
  return x;
}
__device__ __forceinline__ void store_part(const Split &S, uint16_t *p, const Part &x) {
  store16(p + S.e0, pack8(x.a));
  store16(p + S.e1, pack8(x.b));
}
__device__ __forceinline__ Part load_weights(const Split &S, const float *w) {
  Part x;
#pragma unroll
  for (int i = 0; i < 8; i += 4) {
    const f32x4 u = *reinterpret_cast<const f32x4 *>(w + S.e0 + i), v = *reinterpret_cast<const f32x4 *>(w + S.e1 + i);
#pragma unroll
    for (int k = 0; k < 4; ++k) x.a[i + k] = u[k], x.b[i + k] = v[k];
  }
  return x;
}

// Sum over a row's eight lanes, the same in each.
__device__ __forceinline__ float sum8(float x) {
  x += dpp_f<0xB1>(x);   // quad_perm [1,0,3,2]
  x += dpp_f<0x4E>(x);   // quad_perm [2,3,0,1]
  x += dpp_f<0x141>(x);  // row_half_mirror
  return x;
}

// x becomes n = r x; returns r = scale / sqrt(mean (scale x)^2 + scale^2 eps).  The scale is 1, or 2^-80 where the squares'
// sum passes fp32 (elements beyond 1e18); below, squares that vanish are nothing beside eps.
__device__ __forceinline__ float normalise(Part &x, float eps) {
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += x.a[i] * x.a[i] + x.b[i] * x.b[i];
  s = sum8(s);
  float scale = 1.0f;
  if (!(s < INFINITY)) {
    scale = 0x1p-80f;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x.a[i] *= scale, x.b[i] *= scale;
      s += x.a[i] * x.a[i] + x.b[i] * x.b[i];
    }
    s = sum8(s);
    eps *= scale * scale;
  }
  const float r = rsqrtf(s * (1.0f / kHeadDim) + eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) x.a[i] *= r, x.b[i] *= r;
  return r * scale;
}

// The pairs of a lane's part of a row turned; SIGN -1: back.  `row`: the row's place in LDS, of 128 elements, for pairs that
// lie in different lanes (which are those of one wave).
template <bool ODD, int SIGN>
__device__ __forceinline__ void turn_part(const ebd_rotary &R, const Split &S, Part &x, const float2 *cs, float *row) {
  auto pair = [&](float &u, float &v, const float2 &t) {
    const float c = t.x, s = SIGN * t.y, y = u * c - v * s;
    v = v * c + u * s;
    u = y;
  };
  const int n = R.rot_dim / 2;
  if (S.how == kHalf) {
#pragma unroll
    for (int i = 0; i < 8; ++i) pair(x.a[i], x.b[i], cs[S.e0 + i]);
  } else if (S.how == kPairs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int u = S.e0 / 2 + i, v = u + 4;
      if (u < n) pair(x.a[2 * i], x.a[2 * i + 1], cs[u]);
      if (v < n) pair(x.b[2 * i], x.b[2 * i + 1], cs[v]);
    }
  }
  if constexpr (ODD) {
    if (S.how == kOdd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) row[S.e0 + i] = x.a[i], row[S.e1 + i] = x.b[i];
    }
    wave_sync();
    if (S.how == kOdd) {
      auto one = [&](float &u, int e) {
        if (e >= 2 * n) return;
        const float2 t = cs[e < n ? e : e - n];
        const float v = row[e < n ? e + n : e - n], s = SIGN * t.y;
        u = u * t.x + (e < n ? -v : v) * s;
      };
#pragma unroll
      for (int i = 0; i < 8; ++i) one(x.a[i], S.e0 + i), one(x.b[i], S.e1 + i);
    }
    wave_sync();  // (before the next row is written)
  }
}

__device__ __forceinline__ void multiply(Part &x, const Part &w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x.a[i] *= w.a[i], x.b[i] *= w.b[i];
}

constexpr int kOddRow = kHeadDim + 4;  // a row in LDS, padded

}  // namespace

template <bool ODD>
__global__ __launch_bounds__(8 * kRopeRows) void norm_rope_kernel(NormRopeLaunch L) {
  __shared__ float2 cs[4][kHeadDim / 2];
  __shared__ float rows[ODD ? kRopeRows : 1][kOddRow];
  const ebd_norm_rope_params &p = L.p;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per, l = i % 8, n = p.rot.rot_dim / 2;
  const int64_t t = token_group(blockIdx.x, blockIdx.z) * L.tpb + slot;
  const int h = blockIdx.y * kRopeRows + i / 8;
  const bool live = t < p.num_tokens && h < p.num_heads;
  const Split sp = part_of(p.rot, l, true);
  Part x = {}, w = {};
  if (live) {
    x = load_row(sp, L.x + t * p.x.token_stride + h * p.x.head_stride);
    w = load_weights(sp, p.norm.weight + h * p.norm.head_stride);
  }
  if (t < p.num_tokens && p.rot.freq && i < n) cs[slot][i] = turn(p.rot, i, p.pos[t]);
  __syncthreads();
  if (!live) return;
  normalise(x, p.norm.eps);
  multiply(x, w);
  turn_part<ODD, 1>(p.rot, sp, x, cs[slot], rows[ODD ? threadIdx.x / 8 : 0]);
  store_part(sp, L.y + t * p.y.token_stride + h * p.y.head_stride, x);
}

constexpr int kBackwardRows = 64;  // (128 of them leave too few registers)

// A work-group takes every gridDim.x'th group of tokens; a thread's head stays the same, so that its share of dw waits in
// registers.  Shared weights: the work-group's rows are added up (within a wave, then through LDS) and leave one row of
// sums; weights of each head's own: each token slot leaves a row for every head.
template <bool ODD, bool SHARED>
__global__ __launch_bounds__(8 * kBackwardRows) void norm_rope_backward_kernel(NormRopeBackwardLaunch L) {
  __shared__ float2 cs[2][4][kHeadDim / 2];
  __shared__ float rows[ODD ? kBackwardRows : 1][kOddRow];
  __shared__ float sums[SHARED ? kBackwardRows / 8 : 1][kHeadDim];
  const ebd_norm_rope_backward_params &p = L.p;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per, l = i % 8, n = p.rot.rot_dim / 2;
  const int h = blockIdx.y * kBackwardRows + i / 8;
  const Split sp = part_of(p.rot, l, true);
  Part w = {}, dw = {};
  if (h < p.num_heads) w = load_weights(sp, p.norm.weight + h * p.norm.head_stride);
  int par = 0;
  for (int64_t g = blockIdx.x; g * L.tpb < p.num_tokens; g += gridDim.x, par ^= 1) {
    const int64_t t = g * L.tpb + slot;
    const bool live = t < p.num_tokens && h < p.num_heads;
    Part x = {}, d = {};
    if (live) {
      x = load_row(sp, L.x + t * p.x.token_stride + h * p.x.head_stride);
      d = load_row(sp, L.dy + t * p.dy.token_stride + h * p.dy.head_stride);
    }
    if (t < p.num_tokens && p.rot.freq && i < n) cs[par][slot][i] = turn(p.rot, i, p.pos[t]);
    __syncthreads();  // (the other half is written by the next group's tokens, which every wave reaches after this one's)
    if (live) {
      const float r = normalise(x, p.norm.eps);
      turn_part<ODD, -1>(p.rot, sp, d, cs[par][slot], rows[ODD ? threadIdx.x / 8 : 0]);
      float m = 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        dw.a[k] += d.a[k] * x.a[k], dw.b[k] += d.b[k] * x.b[k];
        d.a[k] *= w.a[k], d.b[k] *= w.b[k];
        m += d.a[k] * x.a[k] + d.b[k] * x.b[k];
      }
      m = sum8(m) * (1.0f / kHeadDim);
#pragma unroll
      for (int k = 0; k < 8; ++k) d.a[k] = r * (d.a[k] - x.a[k] * m), d.b[k] = r * (d.b[k] - x.b[k] * m);
      store_part(sp, L.dx + t * p.dx.token_stride + h * p.dx.head_stride, d);
    }
  }
  if constexpr (SHARED) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      dw.a[k] = add_xor32(add_xor16(add_xor8(dw.a[k])));
      dw.b[k] = add_xor32(add_xor16(add_xor8(dw.b[k])));
    }
    if (lane < 8) {
#pragma unroll
      for (int k = 0; k < 8; ++k) sums[wave][sp.e0 + k] = dw.a[k], sums[wave][sp.e1 + k] = dw.b[k];
    }
    __syncthreads();
    const int waves = blockDim.x >> 6;
    for (int e = threadIdx.x; e < kHeadDim; e += blockDim.x) {
      float s = 0.0f;
      for (int v = 0; v < waves; ++v) s += sums[v][e];
      L.part[((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * kHeadDim + e] = s;
    }
  } else if (h < p.num_heads) {
    float *out = L.part + (((int64_t)blockIdx.x * L.tpb + slot) * p.num_heads + h) * kHeadDim;
#pragma unroll
    for (int k = 0; k < 8; ++k) out[sp.e0 + k] = dw.a[k], out[sp.e1 + k] = dw.b[k];
  }
}

// dw of a head: its rows of sums, added in a fixed order in 64 bits: 32 lanes take four elements each of every 32nd row,
// then the 32 sums meet (512 rows of 40 heads: 20.9 us with a thread an element and 8 of the rows at a time, 5.6 so).
__global__ __launch_bounds__(1024) void norm_rope_join_kernel(NormRopeBackwardLaunch L) {
  constexpr int kFlight = 8;
  __shared__ double sums[16][kHeadDim];
  const int e = threadIdx.x % 32 * 4, g = threadIdx.x / 32, h = blockIdx.x;
  const float *part = L.part + (int64_t)h * kHeadDim + e;
  const int64_t step = (int64_t)gridDim.x * kHeadDim;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = g; i < L.parts; i += 32 * kFlight) {
    f32x4 v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      v[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i + 32 * k < L.parts) v[k] = *reinterpret_cast<const f32x4 *>(part + (i + 32 * k) * step);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
#pragma unroll
      for (int c = 0; c < 4; ++c) s[c] += v[k][c];
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) s[c] += __shfl_xor(s[c], 32);
  if (threadIdx.x % 64 < 32) {
#pragma unroll
    for (int c = 0; c < 4; ++c) sums[g / 2][e + c] = s[c];
  }
  __syncthreads();
  if (threadIdx.x >= kHeadDim) return;
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) all += sums[i][threadIdx.x];
  L.dweight[(int64_t)h * kHeadDim + threadIdx.x] = (float)all;
}

// Rows of a token in order: its keys, its queries, its values.
template <bool ODD>
__global__ __launch_bounds__(8 * kRopeRows) void append_norm_kernel(AppendNormLaunch L) {
  __shared__ float2 cs[4][kHeadDim / 2];
  __shared__ float rows[ODD ? kRopeRows : 1][kOddRow];
  const ebd_append_paged_params &p = L.p.append;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per, l = i % 8, n = p.rot.rot_dim / 2;
  const int64_t t = token_group(blockIdx.x, blockIdx.z) * L.tpb + slot;
  const int row = blockIdx.y * kRopeRows + i / 8;
  const int kv = p.pages.kv_heads, S = p.pages.num_seqs;
  const bool isk = row < kv, isq = !isk && row < kv + p.q_heads;
  const bool here = t < p.num_tokens && row < 2 * kv + p.q_heads;
  const int h = isk ? row : (isq ? row - kv : row - kv - p.q_heads);
  const Split sp = part_of(p.rot, l, isk || isq);
  const ebd_rows &in = isq ? p.q_rows : (isk ? p.k_rows : p.v_rows);
  const ebd_norm &norm = isq ? L.p.q_norm : L.p.k_norm;
  const bool normed = (isk || isq) && norm.weight;
  Part x = {}, w = {};
  if (here) {  // asked for before the token's place is known
    x = load_row(sp, (isq ? L.q : (isk ? L.k_new : L.v_new)) + t * in.token_stride + h * in.head_stride);
    if (normed) w = load_weights(sp, norm.weight + h * norm.head_stride);
  }
  // the wave's token: its place
  bool live = here;
  int64_t base = -1;
  if (L.p.slots) {
    const int64_t at = t < p.num_tokens ? L.p.slots[t] : -1;
    live &= at >= 0 && (at >> L.shift) < p.pages.num_pages;
    if (t < p.num_tokens && p.rot.freq && i < n) cs[slot][i] = turn(p.rot, i, p.pos[t]);
    base = (at >> L.shift) * p.pages.page_stride + (at & (p.pages.page_size - 1)) * p.pages.row_stride;
    if (!live) base = -1;
  } else {
    const int s = t < p.num_tokens ? find_seq(p.new_off, S, t) : -1;
    live &= s >= 0;
    if (s >= 0) {
      const int64_t r = (int64_t)p.len[s] - p.new_off[s + 1] + t;
      if (p.rot.freq && i < n) cs[slot][i] = turn(p.rot, i, p.pos ? p.pos[t] : r);
      base = page_row(p.pages, L.shift, s, r);
      if (base < 0 && i == 0 && blockIdx.y == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
    }
  }
  __syncthreads();
  if (!live || (!isq && base < 0)) return;
  uint16_t *y = isq ? L.q_out + t * p.q_out_rows.token_stride + h * p.q_out_rows.head_stride
                    : (isk ? L.K : L.V) + base + h * p.pages.head_stride;
  if (normed) {
    normalise(x, norm.eps);
    multiply(x, w);
  }
  turn_part<ODD, 1>(p.rot, sp, x, cs[slot], rows[ODD ? threadIdx.x / 8 : 0]);
  store_part(sp, y, x);
}

namespace {
bool odd(const ebd_rotary &R) { return R.freq && R.layout == EBD_ROPE_HALF && R.rot_dim % 16; }
constexpr int64_t kBackwardGroups = 512;
constexpr int64_t kBackwardChain = 256;  // most token groups of a work-group: as many fp32 additions in a row
}  // namespace

hipError_t launch_norm_rope(NormRopeLaunch L, hipStream_t s) {
  cut_tokens(L.p.num_heads, &L.per, &L.tpb);
  const dim3 grid = rope_grid(L.p.num_tokens, L.p.num_heads, L.tpb), block(L.per * L.tpb);
  if (odd(L.p.rot)) hipLaunchKernelGGL(norm_rope_kernel<true>, grid, block, 0, s, L);
  else hipLaunchKernelGGL(norm_rope_kernel<false>, grid, block, 0, s, L);
  return hipGetLastError();
}

NormRopeBackwardLaunch norm_rope_backward_plan(const ebd_norm_rope_backward_params &p) {
  NormRopeBackwardLaunch L{};
  L.p = p;
  cut_tokens(p.num_heads, &L.per, &L.tpb, kBackwardRows);
  const int64_t groups = ((int64_t)p.num_tokens + L.tpb - 1) / L.tpb, blocks = (p.num_heads + kBackwardRows - 1) / kBackwardRows;
  L.groups = (int32_t)std::min<int64_t>(groups, std::max<int64_t>(std::max<int64_t>(1, kBackwardGroups / blocks),
                                                                  (groups + kBackwardChain - 1) / kBackwardChain));
  L.parts = p.norm.head_stride ? L.groups * L.tpb : (int32_t)(L.groups * blocks);
  return L;
}

size_t norm_rope_backward_bytes(const NormRopeBackwardLaunch &L) {
  return (size_t)L.parts * (L.p.norm.head_stride ? L.p.num_heads : 1) * kHeadDim * sizeof(float);
}

hipError_t launch_norm_rope_backward(const NormRopeBackwardLaunch &L, hipStream_t s) {
  const dim3 grid((unsigned)L.groups, (unsigned)((L.p.num_heads + kBackwardRows - 1) / kBackwardRows)), block(L.per * L.tpb);
  const bool shared = L.p.norm.head_stride == 0;
  if (odd(L.p.rot) && shared) hipLaunchKernelGGL((norm_rope_backward_kernel<true, true>), grid, block, 0, s, L);
  else if (odd(L.p.rot)) hipLaunchKernelGGL((norm_rope_backward_kernel<true, false>), grid, block, 0, s, L);
  else if (shared) hipLaunchKernelGGL((norm_rope_backward_kernel<false, true>), grid, block, 0, s, L);
  else hipLaunchKernelGGL((norm_rope_backward_kernel<false, false>), grid, block, 0, s, L);
  return hipGetLastError();
}

hipError_t launch_norm_rope_join(const NormRopeBackwardLaunch &L, hipStream_t s) {
  const unsigned heads = L.p.norm.head_stride ? L.p.num_heads : 1;
  hipLaunchKernelGGL(norm_rope_join_kernel, dim3(heads), dim3(1024), 0, s, L);
  return hipGetLastError();
}

hipError_t launch_append_norm(AppendNormLaunch L, hipStream_t s) {
  const ebd_append_paged_params &p = L.p.append;
  const int64_t rows = 2 * (int64_t)p.pages.kv_heads + p.q_heads;
  cut_tokens(rows, &L.per, &L.tpb);
  const dim3 grid = rope_grid(p.num_tokens, rows, L.tpb), block(L.per * L.tpb);
  if (odd(p.rot)) hipLaunchKernelGGL(append_norm_kernel<true>, grid, block, 0, s, L);
  else hipLaunchKernelGGL(append_norm_kernel<false>, grid, block, 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
