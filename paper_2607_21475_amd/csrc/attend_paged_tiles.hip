// attend_paged_tiles.hip -- attention of many query rows over a paged cache on gfx950 (prompts, chunks).
//
// attend_tiles: one work-group per (sequence, KV head, block of query rows, split of the rows they see), a wave for
//   each 32 query rows.  Tiles of keys and values pass through LDS, the next one on its way (loads that write LDS
//   directly) while the waves compute the present one; one barrier a tile.
//   S^T = K Q^T on MFMA 32x32x16 bf16 (exact products, fp32 sums): a lane holds half of the scores of one query row,
//   so maxima and sums are register operations and one swap of the wave's halves, and the weights, rounded to
//   bf16, are the B operand of O^T = V^T W^T as they stand, with the keys of a k block in the order 4h .. 4h+3,
//   8+4h .. 8+4h+3 of half h.  V^T comes from the row-major tile by transposing LDS reads.
//   The 16-byte chunks of a tile's row r are stored at chunk ^ turn(r): rows that are read together (eight by
//   the transposing reads, 32 by the key reads) then spread over all banks (no conflicts counted).
//   The running maximum moves only when a score exceeds it by 2^8 (weights stay below that; fp32 and
//   bf16 keep their relative precision), so that most tiles scale nothing.
//   Three shapes.  128 query rows by four waves, tiles of 64 keys, two work-groups a CU: they are out of step by
//   themselves, so that one's weights run under the other's products and its start under the other's loop.  256 query
//   rows by eight waves, one work-group a CU, for one sequence's long chunks: each tile is loaded half as often.
//   64 query rows by eight waves, in four groups of two that take every fourth tile of 32 keys: 33 to 64 rows are
//   too few to hide the memory with 128-row blocks, and too much work for attend_rows' one wave a SIMD (16 sequences
//   of up to 6144 rows, 56 query rows: 40 us, attend_rows 58).
//   Trees (a mask says which new tokens a token sees): a lane reads its row's bits for a tile of new rows from the mask's words,
//   the first of which wait in LDS; tiles of held rows are as above.  They have a shape more: 128 query rows by eight waves in
//   two groups of four, tiles of 64 keys, one work-group a CU.  Alone on its CU a work-group of four waves takes 1.9 us a
//   tile, whatever the depth of its loads (three or four tiles on their way: the same), a chain of products, weights and
//   products; two groups take two tiles in that time, as two work-groups would, but leave half as many partial sums.  Four
//   sequences of up to 300 tokens, 4 heads of 7, under a window of 2048: 51 to 53 us, with work-groups of four waves 58 (three
//   splits).  32 sequences of 64 tokens over 16384 rows, 8 heads of 4, by blocks of 256: 605 to 650 us (0.85 to 0.91 PFLOP/s,
//   keys read once at 3.4 to 3.6 TB/s), by 128: 687; from keys that caches hold 502, as far as the power limit goes.
//   The matrix products bound it: 4 x 128 operations per (query row, key).  So the weights of the first two shapes are
//   rounded to bf16 (half a step, 2^-8, which averages out where many keys share a row); a second product with their tails, 16 bits in all,
//   costs 20 to 40% (8192 tokens over 8192 rows 770 us with it, 566 without, 1024 over 131072 2930 / 2070, 1024 over 1024
//   38.7 / 32.0).  Each key's rounding is its own, and few keys rule many rows, so that trees divide by the sum of the rounded
//   weights (dot products of their pairs with ones; lse keeps the exact sum): y is then off by 2^-8 of the weighted mean of |v - y|,
//   not of |v|, nothing where one key rules or values are alike.  Costs 1 to 4%, a second product 25 to 45% (the trees above 634 us,
//   621 without, 891 with tails; the four sequences 53, 51, 72).  The third shape is bound by memory and has it (the call above with its join 42.0 / 40.9).  1024 tokens, 32
//   heads, over 131072 rows: 1.95 to 2.06 ms, 1.06 to 1.12 PFLOP/s; the matrix cores are busy 54% of the
//   cycles, of which the power limit leaves about 2.0 to 2.1 GHz (a large product runs at 1.34 PFLOP/s there).
#include "attend_paged.hpp"

namespace ebd {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLazy = 8.0f;

// The order of N operands from LDS, READS reads each, and the PRODUCTS of each: four operands on their way, no more, so
// that the registers suffice.
template <int N, int READS, int PRODUCTS = 1>
__device__ __forceinline__ void feed() {
  constexpr int kRead = 0x100, kProduct = 0x008;
  __builtin_amdgcn_sched_group_barrier(kRead, 4 * READS, 0);
#pragma unroll
  for (int i = 0; i < N - 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(kProduct, PRODUCTS, 0);
    __builtin_amdgcn_sched_group_barrier(kRead, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(kProduct, 4 * PRODUCTS, 0);
}

__device__ __forceinline__ Range uniform(const Range &r) {
  return {__builtin_amdgcn_readfirstlane(r.lo), __builtin_amdgcn_readfirstlane(r.hi),
          __builtin_amdgcn_readfirstlane(r.every_lo), __builtin_amdgcn_readfirstlane(r.every_hi)};
}

template <class T>
__device__ __forceinline__ T lds_read(uint32_t at) {
  return *reinterpret_cast<const __attribute__((address_space(3))) T *>(at);
}
template <class T>
__device__ __forceinline__ void lds_write(uint32_t at, const T &v) {
  *reinterpret_cast<__attribute__((address_space(3))) T *>(at) = v;
}
__device__ __forceinline__ s16x4 lds_read_transposed(uint32_t at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4 *>(at));
}

__device__ __forceinline__ int chunk_turn(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

// Written out: from fmaxf the compiler makes three instructions, two of them to quiet NaN.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

__device__ __forceinline__ float max_halves(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace

// RW waves of 32 query rows each, KG groups of them that take every KG'th tile of KEYS keys.  TREE: the new tokens see each
// other by a mask.
template <int RW, int KG, int KEYS, bool NT, bool TREE, bool TAILS = (KG > 1)>
__global__ __launch_bounds__(64 * RW * KG, 2) void attend_tiles_kernel(AttendPagedLaunch L) {
  constexpr int kWaves = RW * KG, kRows = 32 * RW;
  constexpr int kSub = KEYS / 32;             // blocks of 32 keys of a tile
  constexpr bool kRounded = TREE && !TAILS;   // the sums are divided by the rounded weights' total
  constexpr bool kTails = TAILS;              // weights as a bf16 head and a bf16 tail, not a head alone
  constexpr int kPart = KEYS / RW;            // rows of a tile that a wave loads
  constexpr int kTile = KEYS * kRowBytes;     // bytes of a tile's K, or of its V
  constexpr int kStage = KG * 2 * kTile;
  constexpr int kMergeRow = 132;              // floats of a row's sums in LDS, padded
  constexpr int kMerge = KG > 1 ? KG * kRows * kMergeRow * 4 : 0;
  // two stages; the query rows pass through the second, and past its end where they are more than it holds
  constexpr int kThrough = kStage + kWaves * 32 * kRowBytes, kHeld = 2 * kStage > kThrough ? 2 * kStage : kThrough;
  __shared__ __align__(1024) uint8_t tiles[kHeld > kMerge ? kHeld : kMerge];
  static_assert(kThrough <= sizeof(tiles) && kWaves * 32 * kRowBytes <= sizeof(tiles), "query rows, finished rows");
  __shared__ uint32_t poisons[kWaves][32][8];   // of each query row, two bits an element
  __shared__ uint16_t notes[2][KG][KEYS][16];   // of a tile's values, 16 bits a chunk
  __shared__ int noted[2][KG][RW];              // ... whether a wave noted any
  __shared__ Range ranges[kWaves];
  __shared__ int bad_pages[kWaves];
  __shared__ float2 merged[KG > 1 ? KG : 1][kRows];  // maximum and total weight of a group's rows
  constexpr int kMaskHeld = 4;
  __shared__ uint64_t held_words[TREE ? kWaves : 1][32][kMaskHeld];
  const ebd_attend_paged_params &p = L.p;
  const int H = p.pages.kv_heads, G = p.group;
  // heads vary fastest (work-groups go round the XCDs: a head's stay together for 8, 4, 2 heads and
  // share its keys through the XCD's L2), then splits, then query blocks, the last (which see most) first
  auto token = [&](int row) { return L.by_group.quotient(row); };  // of a query row, in its sequence
  const int us = L.by_heads.quotient(blockIdx.x), h = blockIdx.x - us * H;
  const int back = L.by_nsplit.quotient(us), sp = us - back * L.nsplit, u = (int)L.units - 1 - back;
  const Place place = place_of(L, u);
  if (place.s < 0) return;
  const int s = place.s, rb = place.rb;
  const int lane = threadIdx.x & 63, half = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const int rw = wave % RW, kg = wave / RW;

  const Seq sq = sequence(p, s);
  const int row0 = rb * kRows, nrow = min(kRows, sq.tokens * G - row0);
  if (nrow <= 0 || !takes(L, (int64_t)sq.tokens * G)) return;
  if (threadIdx.x == 0 && rb == 0 && sp == 0 && h == 0 && L.status && sq.status) atomicOr(&L.status[s], sq.status);

  // what this wave's rows see, and the work-group's
  const int row = row0 + 32 * rw + c;
  Span span[1] = {TREE ? tree_span_of(L, sq, row) : span_of(L, sq, row)};
  const bool sees = span[0].lo < span[0].hi;
  if (sq.held > sq.seen && __any(TREE ? tree_past_table(L, sq, row) : past_table(L, sq, row)) && lane == 0 && L.status)
    atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  Range R, all;
  if (TREE && p.window == 0) {
    all = tree_range_of(sq);
    R = 32 * rw < nrow ? all : Range{0, 0, 0, 0};
  } else if (!TREE && !p.qpos) {
    R = range_of_tokens(p, sq, token(row0 + 32 * rw), token(row0 + 32 * rw + 31));
    all = range_of_tokens(p, sq, token(row0), token(row0 + nrow - 1));
  } else {
    R = range_of<1>(span);
    if constexpr (TREE) R.every_hi = (int)min((int64_t)R.every_hi, max((int64_t)0, sq.first));
    if (lane == 0) ranges[wave] = R;
    __syncthreads();
    all = ranges[0];
#pragma unroll
    for (int w = 1; w < RW; ++w) {
      all.lo = min(all.lo, ranges[w].lo), all.hi = max(all.hi, ranges[w].hi);
      all.every_lo = max(all.every_lo, ranges[w].every_lo), all.every_hi = min(all.every_hi, ranges[w].every_hi);
    }
  }
  R = uniform(R);
  all = uniform(all);
  const Keys split = split_of(L, all.lo, all.hi, KEYS, sp);
  const int k_beg = split.beg, k_end = split.end;
  const int every_lo = all.every_lo, every_hi = min(all.every_hi, k_end);
  const const_i32 *table = (const const_i32 *)(p.pages.page_table + (int64_t)s * p.pages.max_pages);
  const int slots = p.pages.page_size - 1;

  // this wave's part of a tile: kPart rows, four rows a load, of K and of V
  const uint32_t rs = (uint32_t)p.pages.row_stride * 2u;
  uint32_t off[kPart / 4];
#pragma unroll
  for (int i = 0; i < kPart / 4; ++i) {
    const int r = kPart * rw + 4 * i + (lane >> 4);
    off[i] = (uint32_t)(lane >> 4) * rs + (uint32_t)((lane & 15) ^ chunk_turn(r)) * 16u;
  }
  const int64_t head = (int64_t)h * p.pages.head_stride;
  // (past the range: some page of it; what a group loads there is not used)
  auto page_of = [&](int k) -> int { return table[min(k, k_end - 1) >> L.shift]; };
  const uint32_t part = kPart * rw * kRowBytes;
  auto address = [&](int k, int pg) {
    if ((uint32_t)pg >= (uint32_t)p.pages.num_pages) pg = 0;  // its rows are masked
    return 2 * ((int64_t)pg * p.pages.page_stride + head) + (int64_t)((k + kPart * rw) & slots) * rs;
  };
  auto load_tile = [&](const uint16_t *pool, int64_t at, uint32_t to) {
    const uint8_t *x = reinterpret_cast<const uint8_t *>(pool) + at;
#pragma unroll
    for (int i = 0; i < kPart / 4; ++i) load_lds16<NT>(to + i * 4 * kRowBytes, x + (int64_t)(4 * i) * rs, off[i]);
  };

  // LDS addresses within a tile: K operand row c, dims 16 kb + 8 half at ka ^ 32 kb; V operand rows
  // 4 half + c16 / 4 (+ 8), dims 32 d + .. at va ^ 64 d (tiles are aligned to 1024 bytes)
  const int c16 = lane & 15, q16 = (lane >> 4) & 1;
  const uint32_t ka = c * kRowBytes + (half ^ chunk_turn(c)) * 16;
  uint32_t va[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = 4 * half + (c16 >> 2) + 8 * u;
    va[u] = r * kRowBytes + ((2 * q16 + ((c16 & 3) >> 1)) ^ chunk_turn(r)) * 16 + 8 * (c16 & 1);
  }

  f32x16 O[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) O[d] = f32x16{};
  float m = -INFINITY, z = 0.0f, zr = 0.0f;  // zr: of the weights as they are rounded (kRounded)
  const float sc2 = L.scale * kLog2e;

  const uint32_t tiles_at = lds_at(tiles);
  auto tile_of = [&](int stage) { return tiles_at + stage * kStage + kg * 2 * kTile; };  // this group's
  const int own_hi = min(span[0].hi, k_end);
  // of a lane's row: whether it sees the keys k .. k + 31 inside its span; the first words of the wave's masks wait in LDS,
  // since a load from memory would be waited for together with the tiles on their way
  const int64_t mask_at = TREE ? (sq.t0 + token(min(row, row0 + nrow - 1))) * L.mask_words : 0;
  auto masked = [&](int k) {
    return mask_bits(L, sq, k, [&](int i) { return i < kMaskHeld ? held_words[wave][c][i] : L.mask[mask_at + i]; });
  };
  uint32_t(*poison)[8] = poisons[wave];
  bool poisoned = false;
  f32x16 S[kSub];
  bf16x8 Q[8];  // B operand: column c is this lane's query row, dims 16 kb + 8 half .. + 7
  bf16x8 W[2 * kSub];  // weights, the B operand of the sums
  bf16x8 X[kTails ? 2 * kSub : 1];  // ... their tails
  bool any_bad = false;

  auto keys = [&](uint32_t Kt, int i) {
    return lds_read<bf16x8>(((Kt + ka) ^ (32 * (i / kSub))) + (i % kSub) * 32 * kRowBytes);
  };
  auto values = [&](uint32_t Vt, int i) {
    const uint32_t d = 64 * (i % 4), ks = (i / 4) * 16 * kRowBytes;
    return join8(lds_read_transposed(((Vt + va[0]) ^ d) + ks), lds_read_transposed(((Vt + va[1]) ^ d) + ks));
  };
  auto scores = [&](uint32_t Kt) {
#pragma unroll
    for (int b = 0; b < kSub; ++b) S[b] = f32x16{};
#pragma unroll
    for (int i = 0; i < 8 * kSub; ++i)
      S[i % kSub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(keys(Kt, i), Q[i / kSub], S[i % kSub], 0, 0, 0);
  };
  auto sums = [&](uint32_t Vt) {
#pragma unroll
    for (int i = 0; i < 8 * kSub; ++i) {
      const bf16x8 A = values(Vt, i);
      if constexpr (kTails) O[i % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, X[i / 4], O[i % 4], 0, 0, 0);
      O[i % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A, W[i / 4], O[i % 4], 0, 0, 0);
    }
  };
  auto mixed = [&](int k, uint32_t bad) { return bad || k < R.every_lo || k + KEYS > min(R.every_hi, k_end); };
  auto softmax = [&](int k, uint32_t bad) {
    if (mixed(k, bad)) {
#pragma unroll
      for (int b = 0; b < kSub; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = k + 32 * b + 8 * (i / 4) + 4 * half + i % 4;
          const bool ok = (key >= span[0].lo) & (key < own_hi) & !((bad >> (2 * b + i / 8)) & 1u);
          S[b][i] = ok ? S[b][i] : -INFINITY;
        }
        if (TREE && k + KEYS > R.every_hi) {
          const uint32_t bits = masked(k + 32 * b) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i) S[b][i] = (bits >> (8 * (i / 4) + i % 4)) & 1u ? S[b][i] : -INFINITY;
        }
      }
    }
    // (the first maximum reads every accumulator's last products, which the compiler waits for, and the rest
    // depend on it)
    float t0 = fmaxf(S[0][0], S[kSub - 1][1]), t1 = fmaxf(fmaxf(S[0][1], S[kSub - 1][0]), t0);
#pragma unroll
    for (int i = 2; i < 16 * kSub; i += 4) {
      t0 = max3(t0, S[i / 16][i % 16], S[i / 16][i % 16 + 1]);
      if (i + 2 < 16 * kSub) t1 = max3(t1, S[(i + 2) / 16][(i + 2) % 16], S[(i + 2) / 16][(i + 2) % 16 + 1]);
    }
    const float t = max_halves(fmaxf(t0, t1)) * sc2;
    if (__any(t > m + kLazy)) {
      const float mn = fmaxf(m, t);
      const float a = mn == -INFINITY ? 1.0f : fast_exp2(m - mn);
      m = mn;
      z *= a;
      if constexpr (kRounded) zr *= a;
#pragma unroll
      for (int d = 0; d < 4; ++d) O[d] *= a;
    }
    const float mu = m == -INFINITY ? 0.0f : m;  // nothing seen yet: every score is -inf
    // a tile's weights are added up by themselves: z takes one rounding a tile
    float part_z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int b = 0; b < kSub; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = fast_exp2(__builtin_fmaf(S[b][i], sc2, -mu));
        part_z[i % 4] += w;
        W[2 * b + i / 8][i % 8] = (__bf16)w;
        if constexpr (kTails) X[2 * b + i / 8][i % 8] = (__bf16)(w - (float)W[2 * b + i / 8][i % 8]);
      }
    }
    z += (part_z[0] + part_z[1]) + (part_z[2] + part_z[3]);
    if constexpr (kRounded) {
      const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
      float part_r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int b = 0; b < 2 * kSub; ++b) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          part_r[i] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{W[b][2 * i], W[b][2 * i + 1]}, ones, part_r[i], false);
      }
      zr += (part_r[0] + part_r[1]) + (part_r[2] + part_r[3]);
    }
  };
  auto bad_of = [&](int k) {
    uint32_t bad = 0;
    if (any_bad) {
#pragma unroll
      for (int b = 0; b < 2 * kSub; ++b) bad |= (uint32_t)((uint32_t)page_of(k + 16 * b) >= (uint32_t)p.pages.num_pages) << b;
    }
    return bad;
  };
  // Infinities and NaN must not reach the sums of query rows that do not see them (0 x NaN).  In tiles that some
  // query row sees in part, each wave looks through the values that it loaded: rows that none may see become
  // zeros, and elsewhere what is not finite becomes zero and is noted, two bits an element; then
  // the waves whose query rows see such a key keep the notes (poison), and add them to their sums at the end.
  auto partial = [&](int k, uint32_t bad) { return bad || k < every_lo || k + KEYS > every_hi; };
  auto inspect = [&](int stage, int k) {
    const uint32_t bad = bad_of(k);
    if (!partial(k, bad)) return;
    bool any = false;
    // (all tiles of new rows come here; most hold nothing that a weight of zero would not hide, and are only looked at: 22
    // sequences of 304 tokens over 3 rows 64.5 us noting always, 55.5 so, four of up to 300 under a window 54.5 / 52)
    if constexpr (TREE) {
#pragma unroll
      for (int i = 0; i < kPart / 4; ++i) {
        const u32x4 v = lds_read<u32x4>(tile_of(stage) + kTile + (kPart * rw + (lane >> 4) + 4 * i) * kRowBytes + (lane & 15) * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) any |= not_finite(v[e]) | not_finite(v[e] << 16);
      }
      any = __any(any);
      if (lane == 0) noted[stage][kg][rw] = any;
      if (!any) return;
      any = false;
    }
#pragma unroll
    for (int i = 0; i < kPart / 4; ++i) {
      const int r = kPart * rw + (lane >> 4) + 4 * i;
      const uint32_t at = tile_of(stage) + kTile + r * kRowBytes + (lane & 15) * 16;
      u32x4 v = lds_read<u32x4>(at);
      uint32_t note = 0;
      if (k + r >= k_end || ((bad >> (r / 16)) & 1u)) {
        v = u32x4{0u, 0u, 0u, 0u};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t n0 = poison_of(v[e] << 16), n1 = poison_of(v[e] & 0xffff0000u);
          v[e] &= (n0 ? 0u : 0xffffu) | (n1 ? 0u : 0xffff0000u);
          note |= (n0 | n1 << 2) << (4 * e);
        }
      }
      notes[stage][kg][r][(lane & 15) ^ chunk_turn(r)] = (uint16_t)note;
      lds_write(at, v);
      any |= note != 0u;
    }
    any = __any(any);
    if (lane == 0) noted[stage][kg][rw] = any;
  };
  auto start_notes = [&]() {
    if (!poisoned) {
      for (int i = lane; i < 256; i += 64) poison[0][i] = 0u;
      poisoned = true;
    }
    wave_sync();
  };
  auto keep_note = [&](int key, uint32_t note) {  // 16 bits in each of the first 16 lanes
    if (!__any(note)) return;
    uint32_t bit = 1u;
    if constexpr (TREE) bit = masked(key) & 1u;
#pragma unroll 1
    for (int j = 0; j < 32; ++j) {
      bool hit = (key >= __shfl(span[0].lo, j)) & (key < __shfl(own_hi, j));
      if constexpr (TREE) hit &= __shfl(bit, j) != 0u;
      if (hit && note) atomicOr(&poison[j][lane >> 1], note << (16 * (lane & 1)));
    }
  };
  auto keep_notes = [&](int stage, int k, uint32_t bad) {
    if (!partial(k, bad) || !__any(lane < RW && noted[stage][kg][lane & (RW - 1)])) return;
    start_notes();
#pragma unroll 1
    for (int r = 0; r < KEYS; ++r) {
      if (TREE && !noted[stage][kg][r / kPart]) continue;  // (that wave wrote none)
      keep_note(k + r, lane < 16 ? notes[stage][kg][r][lane] : 0u);
    }
    wave_sync();
  };
  auto mine = [&](int k) { return k < min(R.hi, k_end) && k + KEYS > R.lo; };  // whether this wave's rows see the tile
  auto barrier = [&]() {
    wait_lds();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");  // nothing behind the barrier is read before it
  };

  if (k_beg < k_end) {
    const int step = KG * KEYS;
    int k = k_beg + kg * KEYS;  // this group's tile
    int pg = page_of(k + kPart * rw);
    auto load = [&](int k, int stage) {
      const int64_t at = address(k, pg);
      load_tile(L.K, at, tile_of(stage) + part);
      load_tile(L.V, at, tile_of(stage) + kTile + part);
      pg = page_of(k + step + kPart * rw);
    };
    load(k, 0);
    if constexpr (TREE) {
#pragma unroll
      for (int i = half; i < kMaskHeld; i += 2) held_words[wave][c][i] = i < L.mask_words ? L.mask[mask_at + i] : 0;
    }
    {
      // the wave's query rows come the same way, into the stage that is still free: whole rows, where operand loads
      // would gather 16 bytes from each
      const uint32_t to = tiles_at + kStage + wave * 32 * kRowBytes;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 4), x = min(row0 + 32 * rw + r, row0 + nrow - 1), j = token(x);
        const uint16_t *q = L.q + (sq.t0 + j) * p.q_rows.token_stride + (h * G + x - j * G) * p.q_rows.head_stride;
        load_lds16_from(to + i * 4 * kRowBytes, q + ((lane & 15) ^ chunk_turn(r)) * 8);
      }
      bool bad = false;  // (rows before the first that is seen may have no page any more)
      for (int e = (max(k_beg, all.lo) >> L.shift) + (int)threadIdx.x; e <= (k_end - 1) >> L.shift; e += 64 * kWaves)
        bad |= (uint32_t)p.pages.page_table[(int64_t)s * p.pages.max_pages + e] >= (uint32_t)p.pages.num_pages;
      bad = __any(bad);
      if (lane == 0) bad_pages[wave] = bad;
      wait_loads<0>();
#pragma unroll
      for (int kb = 0; kb < 8; ++kb) Q[kb] = lds_read<bf16x8>(to + (ka ^ (32 * kb)));
    }
    barrier();
    any_bad = __any(lane < kWaves && bad_pages[lane & (kWaves - 1)]);
    if (any_bad && L.status) {  // whether one of this wave's rows sees such a page
      bool gone = false;
#pragma unroll 1
      for (int e = max(k_beg, R.lo) >> L.shift; (e << L.shift) < min(k_end, R.hi); ++e) {
        const int at = e << L.shift;
        if ((uint32_t)table[e] >= (uint32_t)p.pages.num_pages) {
          if constexpr (TREE)
            gone |= __any(sees && sees_any(L, sq, sq.t0 + token(row), span[0].lo, max(at, k_beg),
                                           min((int64_t)at + p.pages.page_size, (int64_t)own_hi)));
          else
            gone |= __any((max(span[0].lo, k_beg) < at + p.pages.page_size) & (own_hi > at));
        }
      }
      if (gone && lane == 0) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
    }
    int st = 0;
    for (int first = k_beg; first < k_end; first += step, k += step, st ^= 1) {
      wait_loads<0>();
      inspect(st, k);
      barrier();  // the tiles are here, and the other stage has been read
      if (first + step < k_end) load(k + step, st ^ 1);
      if (!mine(k)) continue;
      const uint32_t bad = bad_of(k), T = tile_of(st);
      keep_notes(st, k, bad);
      __builtin_amdgcn_s_setprio(1);
      scores(T);
      feed<8 * kSub, 1>();
      __builtin_amdgcn_s_setprio(0);
      softmax(k, bad);
      __builtin_amdgcn_s_setprio(1);
      sums(T + kTile);
      feed<8 * kSub, 2, kTails ? 2 : 1>();
      __builtin_amdgcn_s_setprio(0);
    }
    if constexpr (kTails) {
      static_assert(KEYS == 32, "tiles of any_not_finite");
      // An infinity's products with a weight's head and tail differ in sign, or are infinity times zero: in tiles that
      // every row sees whole the sum is NaN where it should be infinite.  If a sum is NaN over weights that are not, the
      // wave looks through its values once more.
      f32x16 all = (O[0] + O[1]) + (O[2] + O[3]);
#pragma unroll
      for (int n = 8; n; n /= 2) {
#pragma unroll
        for (int i = 0; i < n; ++i) all[i] += all[i + n];
      }
      const float total = add_xor32(z);
      if (__any((all[0] != all[0]) & (total == total))) {
        start_notes();
#pragma unroll 1
        for (int k0 = k_beg + kg * KEYS; k0 < k_end; k0 += step) {
          if (!any_not_finite(L, s, head, k0, k_end)) continue;
#pragma unroll 1
          for (int key = k0; key < min(k0 + KEYS, k_end); ++key) {
            const int64_t at = page_row(p.pages, L.shift, s, key);
            if (at < 0) continue;
            const u32x4 v = reinterpret_cast<const u32x4 *>(L.V + at + head)[lane & 15];
            uint32_t note = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) note |= (poison_of(v[e] << 16) | poison_of(v[e] & 0xffff0000u) << 2) << (4 * e);
            keep_note(key, lane < 16 ? note : 0u);
          }
        }
        wave_sync();
      }
    }
    if constexpr (kRounded) {
      // as if the rounded weights had the exact ones' total, by which the rest divides (the key at the maximum weighs about 1)
      const float exact = add_xor32(z), rounded = add_xor32(zr), a = rounded != 0.0f ? exact / rounded : 1.0f;
#pragma unroll
      for (int d = 0; d < 4; ++d) O[d] *= a;
    }
    // (a NaN weight makes the row's total NaN, and with it what is noted)
    if (poisoned) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t note = poison[c][2 * d + j / 2] >> (16 * (j % 2) + 8 * half);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = (note >> (2 * i)) & 3u;
            if (x) O[d][4 * j + i] = poison_value(x);
          }
        }
      }
    }
  }

  z += __shfl_xor(z, 32);
  const int64_t slot = (((int64_t)u * H + h) * L.nsplit + sp) * kRows;
  if constexpr (KG > 1) {
    // the groups' sums, combined in order
    __syncthreads();
    float *sums_of = reinterpret_cast<float *>(tiles);  // [KG][kRows][kMergeRow]
    float *Ow = sums_of + (kg * kRows + 32 * rw + c) * kMergeRow + 4 * half;
    if (half == 0) merged[kg][32 * rw + c] = sees ? make_float2(m, z) : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4 *>(Ow + 32 * d + 8 * j) = f32x4{O[d][4 * j], O[d][4 * j + 1], O[d][4 * j + 2], O[d][4 * j + 3]};
    }
    __syncthreads();
    const int e = (threadIdx.x & 15) * 8;
    for (int r = threadIdx.x >> 4; r < nrow; r += 4 * kWaves) {
      float M = -INFINITY, Z = 0.0f, o[8] = {};
#pragma unroll
      for (int v = 0; v < KG; ++v) M = fmaxf(M, merged[v][r].x);
#pragma unroll
      for (int v = 0; v < KG; ++v) {
        const float2 t = merged[v][r];
        if (t.y == 0.0f) continue;  // this group saw nothing of the row
        const float a = fast_exp2(t.x - M);
        Z += a * t.y;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] += a * sums_of[(v * kRows + r) * kMergeRow + e + i];
      }
      if (L.nsplit > 1) {
        if (e == 0) L.stats[slot + r] = make_float2(M, Z);
        if (Z == 0.0f) continue;
        float *part_of = L.part + (slot + r) * kHeadDim + e;
        *reinterpret_cast<f32x4 *>(part_of) = f32x4{o[0], o[1], o[2], o[3]};
        *reinterpret_cast<f32x4 *>(part_of + 4) = f32x4{o[4], o[5], o[6], o[7]};
      } else {
        const int j = token(row0 + r);
        store_row(L, sq.t0 + j, h * G + row0 + r - j * G, e, M, Z, o);
      }
    }
    return;
  }
  const int r = 32 * rw + c;
  if (L.nsplit > 1) {
    if (r >= nrow) return;
    if (half == 0) L.stats[slot + r] = sees ? make_float2(m, z) : make_float2(-INFINITY, 0.0f);
    if (!sees || z == 0.0f) return;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4 *>(L.part + (slot + r) * kHeadDim + 32 * d + 8 * j + 4 * half) =
            f32x4{O[d][4 * j], O[d][4 * j + 1], O[d][4 * j + 2], O[d][4 * j + 3]};
    }
    return;
  }
  // finished rows go through LDS, so that they leave as whole rows
  const bool any = sees && z != 0.0f;
  const float a = any ? 1.0f / z : 0.0f;
  const int64_t j = token(row);
  if (half == 0 && L.lse && r < nrow)
    L.lse[(sq.t0 + j) * ((int64_t)H * G) + h * G + (row - j * G)] = any ? (m + fast_log2(z)) * kLn2 : -INFINITY;
  __syncthreads();  // every wave has read its tiles
  const uint32_t at = tiles_at + wave * 32 * kRowBytes;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x2 v;
      v[0] = any ? pack_bf16(O[d][4 * i] * a, O[d][4 * i + 1] * a) : 0u;
      v[1] = any ? pack_bf16(O[d][4 * i + 2] * a, O[d][4 * i + 3] * a) : 0u;
      lds_write(at + c * kRowBytes + ((4 * d + i) ^ chunk_turn(c)) * 16 + 8 * half, v);
    }
  }
  wave_sync();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int x = 4 * i + (lane >> 4), out = 32 * rw + x;
    const u32x4 v = lds_read<u32x4>(at + x * kRowBytes + ((lane & 15) ^ chunk_turn(x)) * 16);
    const int jo = token(row0 + out);
    if (out < nrow)
      *reinterpret_cast<u32x4 *>(L.y + (sq.t0 + jo) * p.y_rows.token_stride + (h * G + row0 + out - jo * G) * p.y_rows.head_stride + (lane & 15) * 8) = v;
  }
}

namespace {
template <bool TREE>
hipError_t launch_tiles(const AttendPagedLaunch &L, hipStream_t s) {
  const dim3 grid((unsigned)attend_paged_groups(L));
  if (L.rows == kFewRows && L.once) hipLaunchKernelGGL((attend_tiles_kernel<2, 4, 32, true, TREE>), grid, dim3(512), 0, s, L);
  else if (L.rows == kFewRows) hipLaunchKernelGGL((attend_tiles_kernel<2, 4, 32, false, TREE>), grid, dim3(512), 0, s, L);
  else if (L.rows == kTileRows) hipLaunchKernelGGL((attend_tiles_kernel<4, 1, 64, false, TREE>), grid, dim3(256), 0, s, L);
  else hipLaunchKernelGGL((attend_tiles_kernel<8, 1, 64, false, TREE>), grid, dim3(512), 0, s, L);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_attend_tiles(const AttendPagedLaunch &L, hipStream_t s) {
  if (L.mask && L.rows == kTileRows && L.pairs) {
    const dim3 grid((unsigned)attend_paged_groups(L));
    hipLaunchKernelGGL((attend_tiles_kernel<4, 2, 64, false, true, false>), grid, dim3(512), 0, s, L);
    return hipGetLastError();
  }
  return L.mask ? launch_tiles<true>(L, s) : launch_tiles<false>(L, s);
}

}  // namespace ebd
