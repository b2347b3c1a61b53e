// rope_device.hpp -- what the kernels that rotate rows share: the sines of a token, how eight lanes split a row, the
// work-groups' tokens.
#pragma once

#include "ebd.h"
#include "ebd_internal.hpp"
#include "paged_device.hpp"

#include <algorithm>

namespace ebd {

constexpr int kRopeRows = 128;  // most rows of a work-group: 8 lanes each

// cos and sin (times the amplitude) of the pair of frequency `freq` at position `pos`.
__device__ __forceinline__ float2 turn_by(const ebd_rotary &R, double freq, int64_t pos) {
  const double t = (double)pos * freq * 0.15915494309189535;  // 1 / 2 pi
  float s, c;
  sincospif(2.0f * (float)(t - rint(t)), &s, &c);
  if (R.flags & EBD_ROPE_INVERSE) s = -s;
  return make_float2(R.amplitude * c, R.amplitude * s);
}
__device__ __forceinline__ float2 turn(const ebd_rotary &R, int i, int64_t pos) { return turn_by(R, R.freq[i], pos); }

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

// Rows are read once, so that they leave no trace in the caches (8191 tokens of 32 rows 31.2 -> 28.9 us, append of 13k
// tokens of 36 rows 53 -> 52); what is written stays there for the attention that reads it next.
__device__ __forceinline__ uint4 load16(const uint16_t *p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)));
}
__device__ __forceinline__ void store16(uint16_t *p, const uint4 &v) { *reinterpret_cast<uint4 *>(p) = v; }

// Work-group (token group, block of rows): `per` threads, whole waves, for each of up to four tokens.  A dimension of the
// grid holds fewer than 2^32 threads, which 2^24 tokens of up to 1024 pass, so token groups fill x and go on in z.
constexpr int kAcross = 1 << 21;
__device__ __forceinline__ int64_t token_group(int x, int z) { return (int64_t)z * kAcross + x; }
__device__ __forceinline__ int token_slot(int per) {
  const int t = threadIdx.x;
  return (t >= per) + (t >= 2 * per) + (t >= 3 * per);
}

// Threads of a token and tokens of a work-group.
inline void cut_tokens(int64_t rows, int32_t *per, int32_t *tpb, int64_t most = kRopeRows) {
  *per = (int32_t)((std::min<int64_t>(rows, most) * 8 + 63) / 64 * 64);
  *tpb = std::max(1, std::min(4, 256 / *per));
}
inline dim3 rope_grid(int64_t tokens, int64_t rows, int tpb) {
  const int64_t groups = (tokens + tpb - 1) / tpb;
  return dim3((unsigned)std::min<int64_t>(groups, kAcross), (unsigned)((rows + kRopeRows - 1) / kRopeRows),
              (unsigned)((groups + kAcross - 1) / kAcross));
}

}  // namespace ebd
