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
//
// Forward, a wave takes a token, eight of its rows at a time and the next eight on their way, or (few tokens) a share of its
// rows: it makes the token's sines itself, a pair a lane, and finds the token's place itself, so that waves never wait for
// each other, and both cost one wave's instructions whatever the rows.  (A work-group a token, a wave for each eight rows and
// the sines shared behind a barrier, issues twice the instructions: 8191 tokens of 40 rows 34.4 us, so 33.0; 5.1 TB/s, of 32
// rows with shared weights 24 us, 5.5 TB/s, the rate of a copy.)  Halves that are no whole chunks (kOdd) meet in LDS: 8191
// tokens of 32 rows, 34 or 126 of 128 elements rotated, 35 us forward and 54 backward with the join, by whole chunks 27 and 44;
// an append of 8192 tokens, 8 KV heads of 4 query heads, 48 and 40.
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
  const bool half = rotated && R.freq && R.layout == EBD_ROPE_HALF, whole = R.rot_dim % 16 == 0;
  const bool pairs = half && whole && 16 * l < R.rot_dim;
  const int how = !rotated || !R.freq ? kCopy : !half ? kPairs : !whole ? kOdd : pairs ? kHalf : kCopy;
  return {how, pairs ? 8 * l : 16 * l, pairs ? R.rot_dim / 2 + 8 * l : 16 * l + 8};
}

__device__ __forceinline__ void unpack8(const uint4 &v, float (&x)[8]) {
  const uint32_t *p = &v.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[2 * i] = bf16_lo(p[i]), x[2 * i + 1] = bf16_hi(p[i]);
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
struct Raw {
  uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const Split &S, const uint16_t *p) { return {load16(p + S.e0), load16(p + S.e1)}; }
__device__ __forceinline__ Part unpack(const Raw &r) {
  Part x;
  unpack8(r.a, x.a);
  unpack8(r.b, x.b);
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

// The sines that a lane's part of a row is turned by: its eight pairs, or (ODD) those of each of its sixteen elements.
template <bool ODD>
struct Turns {
  float2 t[8];
};
template <>
struct Turns<true> {
  float2 t[16];
};

// ... from cs, the token's (those past the last pair are not used).
template <bool ODD>
__device__ __forceinline__ Turns<ODD> turns_of(const ebd_rotary &R, const Split &S, const float2 *cs) {
  Turns<ODD> T;
  if constexpr (ODD) {
    const int n = R.rot_dim / 2;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int e = i < 8 ? S.e0 + i : S.e1 + i - 8;
      const float2 t = cs[e < n ? e : max(0, min(e - n, kHeadDim / 2 - 1))];
      T.t[i] = make_float2(t.x, e < n ? -t.y : t.y);
    }
  } else {
    const int l = threadIdx.x & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) T.t[i] = cs[8 * l + i];
  }
  return T;
}

// A part of a row turned; SIGN -1: back.  row: a place in LDS for it where its pairs lie in different lanes (ODD).
template <bool ODD, int SIGN>
__device__ __forceinline__ void turn_part(const ebd_rotary &R, const Split &S, Part &x, const Turns<ODD> &T, float *row) {
  const int n = R.rot_dim / 2;
  if constexpr (ODD) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      *reinterpret_cast<f32x4 *>(row + S.e0 + i) = f32x4{x.a[i], x.a[i + 1], x.a[i + 2], x.a[i + 3]};
      *reinterpret_cast<f32x4 *>(row + S.e1 + i) = f32x4{x.b[i], x.b[i + 1], x.b[i + 2], x.b[i + 3]};
    }
    wave_sync();
    auto one = [&](float u, int e, float2 t) {
      const float v = row[e < n ? e + n : max(0, e - n)];
      const float y = u * t.x + v * (SIGN * t.y);
      return e < 2 * n ? y : u;
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) x.a[i] = one(x.a[i], S.e0 + i, T.t[i]), x.b[i] = one(x.b[i], S.e1 + i, T.t[8 + i]);
    wave_sync();  // (before the next row is written)
  } else {
    // (by value: from references the compiler makes addresses)
    auto pair = [](float u, float v, float2 t) {
      const float s = SIGN * t.y;
      return make_float2(u * t.x - v * s, v * t.x + u * s);
    };
    if (S.how == kHalf) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 y = pair(x.a[i], x.b[i], T.t[i]);
        x.a[i] = y.x, x.b[i] = y.y;
      }
    } else if (S.how == kPairs) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = S.e0 / 2 + i, v = u + 4;
        const float2 y = pair(x.a[2 * i], x.a[2 * i + 1], T.t[i]), z = pair(x.b[2 * i], x.b[2 * i + 1], T.t[i + 4]);
        x.a[2 * i] = u < n ? y.x : x.a[2 * i], x.a[2 * i + 1] = u < n ? y.y : x.a[2 * i + 1];
        x.b[2 * i] = v < n ? z.x : x.b[2 * i], x.b[2 * i + 1] = v < n ? z.y : x.b[2 * i + 1];
      }
    }
  }
}

__device__ __forceinline__ void multiply(Part &x, const Part &w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x.a[i] *= w.a[i], x.b[i] *= w.b[i];
}

constexpr int kOddRow = kHeadDim + 4;  // a row in LDS, padded
constexpr int kForwardWaves = 4;       // waves of a work-group, which have nothing to do with each other
typedef __attribute__((address_space(4))) int32_t const_i32;  // read through the scalar cache
typedef __attribute__((address_space(4))) int64_t const_i64;

}  // namespace

// A wave's token and its share of the token's rows: every `waves`'th block of eight, from `part` on.
struct Share {
  int64_t t;
  int part, waves;
};
__device__ __forceinline__ Share share_of(int shift) {
  const uint32_t w = blockIdx.x * kForwardWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  return {(int64_t)(w >> shift), (int)(w & ((1u << shift) - 1u)), 1 << shift};
}

// The wave's sines, pair i by lane i.
__device__ __forceinline__ void make_turns(const ebd_rotary &R, int64_t pos, float2 *cs) {
  const int lane = threadIdx.x & 63;
  if (lane < R.rot_dim / 2) cs[lane] = turn(R, lane, pos);
  wave_sync();
}

template <bool ODD>
__global__ __launch_bounds__(64 * kForwardWaves) void norm_rope_kernel(NormRopeLaunch L) {
  __shared__ float2 cs[kForwardWaves][kHeadDim / 2];
  __shared__ float rows[ODD ? 8 * kForwardWaves : 1][kOddRow];
  const ebd_norm_rope_params &p = L.p;
  const Share w = share_of(L.shift);
  if (w.t >= p.num_tokens) return;
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 7, r0 = (threadIdx.x >> 3) & 7;
  const Split sp = part_of(p.rot, l, true);
  const uint16_t *x0 = L.x + w.t * p.x.token_stride;
  uint16_t *y0 = L.y + w.t * p.y.token_stride;
  float *odd = rows[ODD ? threadIdx.x >> 3 : 0];
  int h = 8 * w.part + r0;
  Raw x = {}, next = {};
  Part g = {};
  if (h < p.num_heads) {
    x = load_raw(sp, x0 + h * p.x.head_stride);
    g = load_weights(sp, p.norm.weight + h * p.norm.head_stride);
  }
  Turns<ODD> turns = {};
  if (p.rot.freq) {
    make_turns(p.rot, ((const const_i32 *)p.pos)[w.t], cs[wave]);
    turns = turns_of<ODD>(p.rot, sp, cs[wave]);
  }
  for (; h - r0 < p.num_heads; h += 8 * w.waves, x = next) {
    const int after = h + 8 * w.waves;
    if (after < p.num_heads) next = load_raw(sp, x0 + after * p.x.head_stride);
    Part v = unpack(x);
    normalise(v, p.norm.eps);
    multiply(v, g);
    if (p.norm.head_stride && after < p.num_heads) g = load_weights(sp, p.norm.weight + after * p.norm.head_stride);
    turn_part<ODD, 1>(p.rot, sp, v, turns, odd);
    if (h < p.num_heads) store_part(sp, y0 + h * p.y.head_stride, v);
  }
}

constexpr int kBackwardRows = 64;  // (128 of them leave too few registers)

// A work-group takes every gridDim.x'th group of tokens; a thread's head stays the same, so that its share of dw waits in
// registers; the next group's rows are on their way meanwhile.  Shared weights: the work-group's rows are added up (within a
// wave, then through LDS) and leave one row of sums; weights of each head's own: the token slots' rows are added up, and leave
// one for every head.
template <bool ODD, bool SHARED>
__global__ __launch_bounds__(8 * kBackwardRows) void norm_rope_backward_kernel(NormRopeBackwardLaunch L) {
  __shared__ float2 cs[2][4][kHeadDim / 2];
  __shared__ float rows[ODD ? kBackwardRows : 1][kOddRow];
  __shared__ float sums[SHARED ? kBackwardRows / 8 : 32][kHeadDim];
  const ebd_norm_rope_backward_params &p = L.p;
  const int slot = token_slot(L.per), i = threadIdx.x - slot * L.per, l = i % 8, n = p.rot.rot_dim / 2;
  const int h = blockIdx.y * kBackwardRows + i / 8;
  const Split sp = part_of(p.rot, l, true);
  Part w = {}, dw = {};
  if (h < p.num_heads) w = load_weights(sp, p.norm.weight + h * p.norm.head_stride);
  // The rows of the token after this one's, and its position, are on their way meanwhile.  Nothing else is loaded in the
  // loop, since a wait for it would be one for these; past the last token or head, that one's are asked for, and not used
  // (conditions would cost more).  Two sets of registers in turn, without copies at the loop's end, were no faster: they
  // leave a wave less on a SIMD.
  struct Token {
    Raw x, d;
    int pos;
  };
  const bool turns = p.rot.freq && i < n;
  const double freq = turns ? p.rot.freq[i] : 0.0;
  const int row = min(h, p.num_heads - 1);
  const uint16_t *xs = L.x + row * p.x.head_stride, *ds = L.dy + row * p.dy.head_stride;
  auto ask = [&](int64_t g, Token &to) {
    const int64_t t = min(g * L.tpb + slot, (int64_t)p.num_tokens - 1);
    to.x = load_raw(sp, xs + t * p.x.token_stride);
    to.d = load_raw(sp, ds + t * p.dy.token_stride);
    to.pos = *(turns ? p.pos + t : reinterpret_cast<const int32_t *>(p.norm.weight));
  };
  auto take = [&](int64_t g, int par, const Token &now) {
    if (turns) cs[par][slot][i] = turn_by(p.rot, freq, now.pos);
    __syncthreads();  // (the other half is written by the next group's tokens, which every wave reaches after this one's)
    const int64_t t = g * L.tpb + slot;
    if (t >= p.num_tokens || h >= p.num_heads) return;
    Part x = unpack(now.x), d = unpack(now.d);
    const float r = normalise(x, p.norm.eps);
    turn_part<ODD, -1>(p.rot, sp, d, turns_of<ODD>(p.rot, sp, cs[par][slot]), rows[ODD ? threadIdx.x / 8 : 0]);
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
  };
  Token next;
  ask(blockIdx.x, next);
  int par = 0;
  for (int64_t g = blockIdx.x; g * L.tpb < p.num_tokens; g += gridDim.x, par ^= 1) {
    const Token now = next;
    ask(g + gridDim.x, next);
    take(g, par, now);
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
  } else {
    // (token slots of a work-group have up to 16 rows each, 32 in all)
    if (L.tpb > 1) {
#pragma unroll
      for (int k = 0; k < 8; ++k) sums[threadIdx.x / 8][sp.e0 + k] = dw.a[k], sums[threadIdx.x / 8][sp.e1 + k] = dw.b[k];
      __syncthreads();
      for (int t = 1; slot == 0 && t < L.tpb; ++t) {
        const float *other = sums[(threadIdx.x + t * L.per) / 8];
#pragma unroll
        for (int k = 0; k < 8; ++k) dw.a[k] += other[sp.e0 + k], dw.b[k] += other[sp.e1 + k];
      }
    }
    if (slot == 0 && h < p.num_heads) {
      float *out = L.part + ((int64_t)blockIdx.x * p.num_heads + h) * kHeadDim;
#pragma unroll
      for (int k = 0; k < 8; ++k) out[sp.e0 + k] = dw.a[k], out[sp.e1 + k] = dw.b[k];
    }
  }
}

// A quarter of a head's dw: its rows of sums, added in a fixed order in 64 bits.  Eight lanes take four elements each of
// every 128th row, and the 128 sums meet (512 rows of 40 heads: 20.9 us by a thread an element and eight rows at a time, 5.6
// by whole rows, 32 at a time, 4.9 so; of few heads the work-groups are what lacks).
__global__ __launch_bounds__(1024) void norm_rope_join_kernel(NormRopeBackwardLaunch L) {
  constexpr int kFlight = 4;
  __shared__ double sums[16][32];
  const int quarter = blockIdx.x & 3, h = blockIdx.x >> 2, e = threadIdx.x % 8 * 4, g = threadIdx.x / 8;
  const float *part = L.part + (int64_t)h * kHeadDim + 32 * quarter + e;
  const int64_t step = (int64_t)(gridDim.x / 4) * kHeadDim;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  for (int i = g; i < L.parts; i += 128 * kFlight) {
    f32x4 v[kFlight];
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
      v[k] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i + 128 * k < L.parts) v[k] = *reinterpret_cast<const f32x4 *>(part + (i + 128 * k) * step);
    }
#pragma unroll
    for (int k = 0; k < kFlight; ++k) {
#pragma unroll
      for (int c = 0; c < 4; ++c) s[c] += v[k][c];
    }
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
#pragma unroll
    for (int o = 8; o < 64; o <<= 1) s[c] += __shfl_xor(s[c], o);
  }
  if (threadIdx.x % 64 < 8) {
#pragma unroll
    for (int c = 0; c < 4; ++c) sums[threadIdx.x / 64][e + c] = s[c];
  }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  double all = 0.0;
#pragma unroll
  for (int i = 0; i < 16; ++i) all += sums[i][threadIdx.x];
  L.dweight[(int64_t)h * kHeadDim + 32 * quarter + threadIdx.x] = (float)all;
}

// Blocks of eight rows of a token in order: of its keys, its queries, its values.  A block holds rows of one kind, so that
// the kind, its pointers and strides are the wave's, not the lanes' (blocks of neighbouring rows whatever their kind: 8192
// tokens, 8 KV heads of 4 query heads, 53 us, so 41; a barrier and a wave
// for each block 54).
template <bool ODD>
__global__ __launch_bounds__(64 * kForwardWaves) void append_norm_kernel(AppendNormLaunch L) {
  __shared__ float2 cs[kForwardWaves][kHeadDim / 2];
  __shared__ float rows[ODD ? 8 * kForwardWaves : 1][kOddRow];
  const ebd_append_paged_params &p = L.p.append;
  const Share w = share_of(L.waves);
  if (w.t >= p.num_tokens) return;
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 7, r0 = (threadIdx.x >> 3) & 7;
  const int kv = p.pages.kv_heads, nk = (kv + 7) / 8, nq = (p.q_heads + 7) / 8, blocks = 2 * nk + nq;
  float *odd = rows[ODD ? threadIdx.x >> 3 : 0];
  const Split turned = part_of(p.rot, l, true), copied = {kCopy, 16 * l, 16 * l + 8};
  enum { kKey, kQuery, kValue };
  auto kind_of = [&](int b) { return b < nk ? kKey : b < nk + nq ? kQuery : kValue; };
  auto head_of = [&](int b) { return 8 * (b < nk ? b : b < nk + nq ? b - nk : b - nk - nq) + r0; };
  auto load = [&](int b) -> Raw {
    const int kind = kind_of(b), h = head_of(b);
    const ebd_rows &in = kind == kKey ? p.k_rows : kind == kQuery ? p.q_rows : p.v_rows;
    const uint16_t *x = (kind == kKey ? L.k_new : kind == kQuery ? L.q : L.v_new) + w.t * in.token_stride;
    if (h >= (kind == kQuery ? p.q_heads : kv)) return {};
    return load_raw(kind == kValue ? copied : turned, x + h * in.head_stride);
  };
  auto weights = [&](int b) -> Part {  // (asked for with the rows: behind them, a wait would be one for the next rows, too)
    const int kind = kind_of(b), h = head_of(b);
    const ebd_norm &norm = kind == kKey ? L.p.k_norm : L.p.q_norm;
    if (kind == kValue || !norm.weight || h >= (kind == kQuery ? p.q_heads : kv)) return {};
    return load_weights(turned, norm.weight + h * norm.head_stride);
  };
  Raw x = {}, next = {};
  Part g = {}, next_g = {};
  int b = w.part;
  if (b < blocks) x = load(b), g = weights(b);  // asked for before the token's place is known
  int64_t base = -1, pos = 0;
  if (L.p.slots) {
    const int64_t at = ((const const_i64 *)L.p.slots)[w.t];
    if (at < 0 || (at >> L.shift) >= p.pages.num_pages) return;
    base = (at >> L.shift) * p.pages.page_stride + (at & (p.pages.page_size - 1)) * p.pages.row_stride;
  } else {
    const int s = __builtin_amdgcn_readfirstlane(find_seq(p.new_off, p.pages.num_seqs, w.t));
    if (s < 0) return;
    pos = (int64_t)((const const_i32 *)p.len)[s] - ((const const_i64 *)p.new_off)[s + 1] + w.t;
    const int64_t e = pos >> L.shift;  // (as page_row, by scalar loads)
    const int pg = pos >= 0 && e < p.pages.max_pages
                       ? ((const const_i32 *)p.pages.page_table)[(int64_t)s * p.pages.max_pages + e] : -1;
    if ((uint32_t)pg < (uint32_t)p.pages.num_pages)
      base = pg * p.pages.page_stride + (pos & (p.pages.page_size - 1)) * p.pages.row_stride;
    else if (w.part == 0 && (threadIdx.x & 63) == 0 && L.status)
      atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  }
  Turns<ODD> turns = {};
  if (p.rot.freq) {
    make_turns(p.rot, p.pos ? (int64_t)((const const_i32 *)p.pos)[w.t] : pos, cs[wave]);
    turns = turns_of<ODD>(p.rot, turned, cs[wave]);
  }
  for (; b < blocks; b += w.waves, x = next, g = next_g) {
    if (b + w.waves < blocks) next = load(b + w.waves), next_g = weights(b + w.waves);
    const int kind = kind_of(b), h = head_of(b);
    if (kind != kQuery && base < 0) continue;
    const bool here = h < (kind == kQuery ? p.q_heads : kv);
    if (kind == kValue) {
      uint16_t *y = L.V + base + h * p.pages.head_stride;
      if (here) store16(y + copied.e0, x.a), store16(y + copied.e1, x.b);
      continue;
    }
    const ebd_norm &norm = kind == kKey ? L.p.k_norm : L.p.q_norm;
    Part v = unpack(x);
    if (norm.weight) {
      normalise(v, norm.eps);
      multiply(v, g);
    }
    turn_part<ODD, 1>(p.rot, turned, v, turns, odd);
    if (here)
      store_part(turned, kind == kKey ? L.K + base + h * p.pages.head_stride
                                      : L.q_out + w.t * p.q_out_rows.token_stride + h * p.q_out_rows.head_stride, v);
  }
}

namespace {
bool odd(const ebd_rotary &R) { return R.freq && R.layout == EBD_ROPE_HALF && R.rot_dim % 16; }
// Work-groups of more than four waves: one a CU, since a wave that shares its SIMD with another of its group keeps the others
// waiting at the barrier.  us with the join, by 128 / 256 / 384 / 512 / 768 work-groups: 8191 tokens of 40 rows, weights of
// their own (five waves) 85 / 51 / 65 / 57 / 62, 1000 of 40 18.9 / 15.8 / 20.5 / 21.3 / 25.6, 8191 of 32 with shared ones (four
// waves) 79 / 46 / 42 / 38 / 39, 4212 of 7 with their own 18.3 / 13.8 / 12.7 / 12.0 / 12.9.
constexpr int64_t kBackwardGroups = 512, kBackwardWide = 256;
constexpr int64_t kBackwardChain = 256;  // most token groups of a work-group: as many fp32 additions in a row
}  // namespace

// Waves of a token (their logarithm): one where the tokens are enough to fill the chip, else as many as there are blocks of
// eight rows, or as fill it.
// us by one wave a token below / at / above the line: norms of 8191 tokens of 32 rows 23.6 / 24.8, 2048 of 32 - / 7.6 / 8.0;
// appends, whose waves each find the token's place, of 8192 tokens of 48 rows 41.8 / 41.4 / 40.3, of 2000 of 36 rows
// 12.0 / 13.4 / 18.3.
constexpr int64_t kNormFill = 4096, kAppendFill = 2048;
int32_t forward_shift(int64_t tokens, int64_t rows, int64_t fill) {
  int32_t s = 0;
  while ((tokens << s) < fill && (8 << s) < rows) ++s;
  return s;
}
dim3 forward_grid(int64_t tokens, int32_t shift) {
  return dim3((unsigned)(((tokens << shift) + kForwardWaves - 1) / kForwardWaves));
}

hipError_t launch_norm_rope(NormRopeLaunch L, hipStream_t s) {
  L.shift = forward_shift(L.p.num_tokens, L.p.num_heads, kNormFill);
  const dim3 grid = forward_grid(L.p.num_tokens, L.shift), block(64 * kForwardWaves);
  if (odd(L.p.rot)) hipLaunchKernelGGL(norm_rope_kernel<true>, grid, block, 0, s, L);
  else hipLaunchKernelGGL(norm_rope_kernel<false>, grid, block, 0, s, L);
  return hipGetLastError();
}

NormRopeBackwardLaunch norm_rope_backward_plan(const ebd_norm_rope_backward_params &p) {
  NormRopeBackwardLaunch L{};
  L.p = p;
  const int32_t heads = std::max(p.num_heads, 1);  // (without heads the sums of shared weights are written, as zeros)
  cut_tokens(heads, &L.per, &L.tpb, kBackwardRows);
  const int64_t groups = ((int64_t)p.num_tokens + L.tpb - 1) / L.tpb, blocks = (heads + kBackwardRows - 1) / kBackwardRows;
  const int64_t fill = std::max<int64_t>(1, (L.per > 256 ? kBackwardWide : kBackwardGroups) / blocks);
  L.groups = (int32_t)std::min<int64_t>(groups, std::max<int64_t>(fill, (groups + kBackwardChain - 1) / kBackwardChain));
  L.parts = p.norm.head_stride ? L.groups : (int32_t)(L.groups * blocks);
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
  hipLaunchKernelGGL(norm_rope_join_kernel, dim3(4 * heads), dim3(1024), 0, s, L);
  return hipGetLastError();
}

hipError_t launch_append_norm(AppendNormLaunch L, hipStream_t s) {
  const ebd_append_paged_params &p = L.p.append;
  L.waves = forward_shift(p.num_tokens, 8 * (2 * ((p.pages.kv_heads + 7) / 8) + (int64_t)(p.q_heads + 7) / 8), kAppendFill);
  const dim3 grid = forward_grid(p.num_tokens, L.waves), block(64 * kForwardWaves);
  if (odd(p.rot)) hipLaunchKernelGGL(append_norm_kernel<true>, grid, block, 0, s, L);
  else hipLaunchKernelGGL(append_norm_kernel<false>, grid, block, 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
