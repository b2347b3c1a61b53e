// attend_paged.hpp -- what the kernels of the paged attention share: a launch's sequences and the rows their
// queries see, loads that write LDS directly, transposing LDS reads, and the finished rows' store.
#pragma once

#include "ebd.h"
#include "ebd_internal.hpp"
#include "paged_device.hpp"

namespace ebd {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(4))) int32_t const_i32;  // read through the scalar cache
typedef __attribute__((address_space(4))) int64_t const_i64;

constexpr int kRowBytes = 2 * kHeadDim;

__device__ __forceinline__ uint32_t lds_at(const void *p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_u8 *)(uint8_t *)p);
}

// 16 bytes per lane from base + off straight into LDS at `to` + 16 lane; NT: the non-temporal hint.  Written as
// assembly because the compiler would wait for all of them before any read of LDS; it holds no result register, and
// the waits below order it.  It writes m0, which cannot be named as clobbered (the register is reserved); nothing else in
// these kernels uses it, which the build's tests look at.
template <bool NT>
__device__ __forceinline__ void load_lds16(uint32_t to, const uint8_t *base, uint32_t off) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(to), "v"(off), "s"(base)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base)
                 : "memory");
}
// ... from an address of each lane's own.
__device__ __forceinline__ void load_lds16_from(uint32_t to, const void *from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(from) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

__device__ __forceinline__ bf16x8 join8(s16x4 lo, s16x4 hi) {
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ s16x4 read_transposed(const uint8_t *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(lds_u8 *)p);
}

// A sequence's part of a launch.
struct Seq {
  int64_t t0;       // its first new token
  int tokens;       // new tokens that get an output
  int64_t first;    // row of its first new token
  int64_t len;      // rows it holds
  int64_t held;     // ... of which the host's bound lets the launch see
  int64_t seen;     // ... and the page table holds
  uint32_t status;
};
// New tokens of a sequence that get an output: tokens t0 .. t1 - 1, as far as the bounds allow.
__device__ __forceinline__ int tokens_of(const ebd_attend_paged_params &p, int64_t t0, int64_t t1) {
  if (t0 < 0) return 0;
  return (int)max((int64_t)0, min(min(t1 - t0, (int64_t)p.max_new), p.num_tokens - t0));
}
__device__ __forceinline__ Seq sequence(const ebd_attend_paged_params &p, int s) {
  Seq q;
  const const_i64 *off = (const const_i64 *)p.new_off;
  q.t0 = off[s];
  const int64_t t1 = off[s + 1], n = t1 - q.t0;
  q.len = ((const const_i32 *)p.len)[s];
  q.first = q.len - n;
  q.status = (n > p.max_new || q.len > p.max_rows) ? EBD_ST_BAD_LAYOUT : 0u;
  q.held = min(q.len, p.max_rows);
  q.seen = min(q.held, (int64_t)p.pages.max_pages * p.pages.page_size);
  q.tokens = tokens_of(p, q.t0, t1);
  return q;
}

// Whether a launch takes a sequence with this many query rows.
__device__ __forceinline__ bool takes(const AttendPagedLaunch &L, int64_t rows) {
  return rows > L.more_than && rows <= L.at_most;
}

// The u'th block of query rows of a launch: its sequence (-1: there is none) and which of its blocks.  With
// L.blocks blocks set aside for each sequence that is a division; otherwise (sequences of very different
// lengths, of which most would stay empty) the sequences' own blocks are counted, 64 sequences at a time.
// u is uniform over the wave, and so is the result.
struct Place {
  int s, rb;
};
__device__ __forceinline__ Place place_of(const AttendPagedLaunch &L, int u) {
  if (L.blocks > 0) {
    const int s = L.by_blocks.quotient(u);
    return {s, u - s * L.blocks};
  }
  const ebd_attend_paged_params &p = L.p;
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < p.pages.num_seqs; base += 64) {
    const int s = base + lane;
    int n = 0;
    if (s < p.pages.num_seqs) {
      const int64_t rows = (int64_t)tokens_of(p, p.new_off[s], p.new_off[s + 1]) * p.group;
      if (takes(L, rows)) n = (int)((rows + L.rows - 1) / L.rows);
    }
    int upto = n;  // blocks of the sequences up to this lane's
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t behind = __ballot(upto > u);
    if (behind) {
      const int l = __builtin_ctzll(behind);
      return {base + l, u - __builtin_amdgcn_readlane(upto - n, l)};
    }
    u -= __builtin_amdgcn_readlane(upto, 63);
  }
  return {-1, 0};
}

// The keys of split sp of a block that sees the rows lo .. hi - 1: its own rows, from a tile's border on, dealt
// evenly over the splits, at least L.least (a multiple of 128) each.
struct Keys {
  int beg, end;
};
__device__ __forceinline__ Keys split_of(const AttendPagedLaunch &L, int lo, int hi, int tile, int sp) {
  if (lo >= hi) return {0, 0};
  lo &= -tile;
  int rows = hi - lo;
  if (L.nsplit > 1) rows = max(L.least, ((rows + L.nsplit - 1) / L.nsplit + 127) / 128 * 128);
  const int64_t beg = lo + (int64_t)sp * rows;
  if (beg >= hi) return {0, 0};
  return {(int)beg, (int)min((int64_t)hi, beg + rows)};
}

// The rows lo .. hi - 1 that query row `row` sees (lo >= hi: none).
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span span_of(const AttendPagedLaunch &L, const Seq &q, int row) {
  const ebd_attend_paged_params &p = L.p;
  const int j = L.by_group.quotient(row);
  if (j >= q.tokens) return {0, 0};
  int64_t last = q.first + j;
  if (p.qpos) last = min((int64_t)p.qpos[q.t0 + j], q.len - 1);
  const int64_t lo = p.window > 0 ? max((int64_t)0, last - p.window + 1) : 0;
  const int64_t hi = min(last + 1, q.seen);
  return lo < hi ? Span{(int)lo, (int)hi} : Span{0, 0};
}

// Whether query row `row` would see rows behind the page table's end.
__device__ __forceinline__ bool past_table(const AttendPagedLaunch &L, const Seq &q, int row) {
  const ebd_attend_paged_params &p = L.p;
  const int j = L.by_group.quotient(row);
  if (j >= q.tokens) return false;
  int64_t last = q.first + j;
  if (p.qpos) last = min((int64_t)p.qpos[q.t0 + j], q.len - 1);
  const int64_t lo = p.window > 0 ? last - p.window + 1 : 0;
  return min(last + 1, q.held) > max(lo, q.seen);
}

// The range a block of query rows sees (the same in every lane of a wave that holds them all), and
// whether a tile needs masks: inside [every_lo, every_hi) every row that sees anything sees all.
struct Range {
  int lo, hi, every_lo, every_hi;
};
template <int N>
__device__ __forceinline__ Range range_of(const Span (&s)[N]) {
  int lo = INT32_MAX, hi = 0, elo = 0, ehi = INT32_MAX;
#pragma unroll
  for (int b = 0; b < N; ++b) {
    if (s[b].lo >= s[b].hi) continue;
    lo = min(lo, s[b].lo), hi = max(hi, s[b].hi);
    elo = max(elo, s[b].lo), ehi = min(ehi, s[b].hi);
  }
  return {wave_min(lo), -wave_min(-hi), -wave_min(-elo), wave_min(ehi)};
}

// A bf16 value in a word's upper half: whether it is an infinity or NaN, and its note (bit 0: +inf, bit 1:
// -inf, both: NaN); what a note adds to a sum.
__device__ __forceinline__ bool not_finite(uint32_t v) { return (v & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t poison_of(uint32_t v) {
  return !not_finite(v) ? 0u : (v & 0x007f0000u) ? 3u : (v >> 31) ? 2u : 1u;
}
__device__ __forceinline__ float poison_value(uint32_t note) {
  return note == 0u ? 0.0f : note == 1u ? INFINITY : note == 2u ? -INFINITY : NAN;
}

// Whether any value of the rows k .. end - 1 (at most 32) of a sequence's KV head is not finite; `head`: its offset.
__device__ __forceinline__ bool any_not_finite(const AttendPagedLaunch &L, int s, int64_t head, int k, int end) {
  const int lane = threadIdx.x & 63;
  bool found = false;
#pragma unroll 2
  for (int r = lane >> 4; r < 32; r += 4) {
    const int64_t at = k + r < end ? page_row(L.p.pages, L.shift, s, k + r) : -1;
    if (at < 0) continue;
    const u32x4 v = reinterpret_cast<const u32x4 *>(L.V + at + head)[lane & 15];
#pragma unroll
    for (int e = 0; e < 4; ++e) found |= not_finite(v[e]) | not_finite(v[e] << 16);
  }
  return __any(found);
}

// range_of the query rows of tokens j0 .. j1 without positions of their own (p.qpos is NULL): what they see moves
// on with the token, so the first and the last that see anything tell.
__device__ __forceinline__ Range range_of_tokens(const ebd_attend_paged_params &p, const Seq &q, int j0, int j1) {
  const int64_t w = p.window > 0 ? p.window : INT64_MAX / 2;
  const int64_t a = max(q.first + j0, (int64_t)0), b = min(q.first + min(j1, q.tokens - 1), q.seen - 2 + w);
  if (a > b || q.seen <= 0) return {INT32_MAX, 0, 0, INT32_MAX};
  return {(int)max((int64_t)0, a - w + 1), (int)min(b + 1, q.seen), (int)max((int64_t)0, b - w + 1),
          (int)min(a + 1, q.seen)};
}

// Elements e .. e+7 of a finished row: token t, query head hq, sums o over weights that total Z with the
// maximum M.  A row, or a part of one, that saw nothing has Z = 0, and no other: the key at the maximum weighs 1, and a
// logit that is NaN makes Z NaN, though no maximum shows it (M stays -inf where there are no others).
__device__ __forceinline__ void store_row(const AttendPagedLaunch &L, int64_t t, int hq, int e, float M, float Z,
                                          const float (&o)[8]) {
  const bool any = Z != 0.0f;
  const float a = any ? 1.0f / Z : 0.0f;
  uint4 v;
  v.x = any ? pack_bf16(o[0] * a, o[1] * a) : 0u;
  v.y = any ? pack_bf16(o[2] * a, o[3] * a) : 0u;
  v.z = any ? pack_bf16(o[4] * a, o[5] * a) : 0u;
  v.w = any ? pack_bf16(o[6] * a, o[7] * a) : 0u;
  *reinterpret_cast<uint4 *>(L.y + t * L.p.y_rows.token_stride + hq * L.p.y_rows.head_stride + e) = v;
  if (e == 0 && L.lse)
    L.lse[t * ((int64_t)L.p.pages.kv_heads * L.p.group) + hq] = any ? (M + fast_log2(Z)) * kLn2 : -INFINITY;
}

}  // namespace ebd
