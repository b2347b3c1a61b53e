// attend_paged.hip -- attention of a chunk of new tokens over a paged cache on gfx950.
//
// Query rows: token j and query head g of the heads that share a KV head make row j group + g, so that one
// pass over the KV head's keys serves all of them.  Per row, over the rows lo .. hi it sees, in base-2
// logits l = scale log2e q.k:
//   m = max l,  w = 2^(l - m),  y = sum w v / sum w,  lse = m ln 2 + ln sum w
// in one pass, m running (what was summed is scaled down when it grows).
//
// attend_rows (up to 32 query rows of a sequence): one work-group per (sequence, KV head, split of the rows that its
//   block of 16 or 32 query rows sees), four waves that take its tiles of 32 keys in turn, each on its own.  A wave keeps the
//   next tile's keys and values on their way into its share of LDS (loads that write LDS directly, 16 bytes a
//   lane) while it computes the present one; nothing in the loop waits for another wave.
//   Scores are formed transposed, S^T = K Q^T (MFMA 16x16x32 bf16: exact products, fp32 sums): lane (g, c) then
//   holds keys 4g .. 4g+3 of query row c, so a row's maximum is a maximum over registers and two lane swaps,
//   and its weights are, as they stand, the B operand of O^T = V^T W^T with the keys of the k slots in the order
//   4g .. 4g+3, 16+4g .. 16+4g+3.  V^T comes from the row-major tile by transposing LDS reads.
//   The 16-byte chunks of a tile's row r are stored at chunk ^ (r mod 16): without that, the rows a
//   read gathers from would all lie in the same banks.
//   Weights enter as a bf16 head and a bf16 tail (16 bits of each): the memory bounds these launches, and
//   the second product costs nothing beside it.  A decode step of 32 sequences of 16384 rows, 8 KV heads of 4 query
//   heads: 317 us, 6.8 TB/s, its keys and values read exactly once; of one of 4096 rows, 8 heads: 6.3 us and the join
//   3.5, a chain of loads (lengths, pages, the tile) of half a microsecond each.
//   Under a mask the same shapes serve trees of up to 32 query rows, us with the mask / in order: 8 KV heads of 4 query heads, 32
//   sequences of 4 tokens over 16384 rows 327 / 324, of 8 336 / 329 (6.4 TB/s), 64 of 4 over 4096 171 / 167, of 8 183 / 178, one
//   of 8 over 4096 15.7 / 14.4 (of 4, one block of 16 rows, 12.2 / 11.5).
// attend_join: the splits of each row, combined in order.
#include "attend_paged.hpp"

namespace ebd {

namespace {

constexpr int kTileKeys = 32;
constexpr int kTileBytes = kTileKeys * 2 * kHeadDim;  // of K, or of V
constexpr int kRowsStages = 2;
constexpr int kMergeRow = 132;  // floats of a row's sums in LDS, padded

__device__ __forceinline__ float max_xor16_32(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace

// TREE: the new tokens see each other by a mask.
template <int NQ, bool NT, bool TREE>
__global__ __launch_bounds__(256, 1) void attend_rows_kernel(AttendPagedLaunch L) {
  constexpr int kRows = 16 * NQ;
  constexpr int kMerge = kRows * (kMergeRow * 4 + 8);  // a wave's sums and statistics, when the waves combine
  constexpr int kPoison = kRowsStages * 2 * kTileBytes;  // (read before the waves combine)
  constexpr int kWaveLds = kPoison + kRows * kHeadDim > kMerge ? kPoison + kRows * kHeadDim : kMerge;
  __shared__ __align__(1024) uint8_t lds[kRowsWaves * kWaveLds];
  const ebd_attend_paged_params &p = L.p;
  const int H = p.pages.kv_heads, G = p.group;
  auto token = [&](int row) { return L.by_group.quotient(row); };  // of a query row, in its sequence
  const int uh = L.by_nsplit.quotient(blockIdx.x), sp = blockIdx.x - uh * L.nsplit;
  const int s = L.by_heads.quotient(uh), h = uh - s * H;  // a block holds all query rows of a sequence
  const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const Seq sq = sequence(p, s);
  const int nrow = min(kRows, sq.tokens * G);
  if (nrow <= 0 || !takes(L, (int64_t)sq.tokens * G)) return;
  if (threadIdx.x == 0 && sp == 0 && h == 0 && L.status && sq.status) atomicOr(&L.status[s], sq.status);

  Span span[NQ];
#pragma unroll
  for (int b = 0; b < NQ; ++b) span[b] = TREE ? tree_span_of(L, sq, 16 * b + c) : span_of(L, sq, 16 * b + c);
  if (sq.held > sq.seen && L.status && sp == 0 && wave == 0) {
#pragma unroll
    for (int b = 0; b < NQ; ++b)
      if (__any(TREE ? tree_past_table(L, sq, 16 * b + c) : past_table(L, sq, 16 * b + c)) && lane == 0)
        atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  }
  Range R;
  uint64_t word0[NQ];  // of a row's mask: few rows have few tokens
  if constexpr (TREE) {
    R = p.window > 0 ? range_of<NQ>(span) : tree_range_of(sq);
    if (p.window > 0) R.every_hi = (int)min((int64_t)R.every_hi, max((int64_t)0, sq.first));
#pragma unroll
    for (int b = 0; b < NQ; ++b) word0[b] = L.mask[(sq.t0 + token(min(16 * b + c, nrow - 1))) * L.mask_words];
  } else {
    R = p.qpos ? range_of<NQ>(span) : range_of_tokens(p, sq, 0, token(nrow - 1));
  }
  // whether this lane's row of a block sees a key inside its span
  auto masked = [&](int b, int k) {
    return mask_bits(L, sq, k, [&](int i) {
      return i == 0 ? word0[b] : L.mask[(sq.t0 + token(min(16 * b + c, nrow - 1))) * L.mask_words + i];
    });
  };
  const Keys split = split_of(L, R.lo, R.hi, kTileKeys, sp);
  const int k_beg = split.beg, k_end = split.end;  // (below 2^30: no sum below overflows)

  f32x4 O[NQ][8];
  float m[NQ], z[NQ];
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    m[b] = -INFINITY;
    z[b] = 0.0f;
#pragma unroll
    for (int d = 0; d < 8; ++d) O[b][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // lane offsets (bytes) of rows 4i + g of a 16-row slab, chunks permuted
  uint8_t *my = lds + wave * kWaveLds;
  const uint32_t rs = (uint32_t)p.pages.row_stride * 2u;
  uint32_t off[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) off[i] = (uint32_t)g * rs + (uint32_t)(c ^ (4 * i + g)) * 16u;
  const int64_t head = (int64_t)h * p.pages.head_stride;
  const const_i32 *table = (const const_i32 *)(p.pages.page_table + (int64_t)s * p.pages.max_pages);
  const int slots = p.pages.page_size - 1;

  // page numbers of the two slabs of the tile at key k (uniform); -1: none
  auto page_of = [&](int k) -> int {
    if (k >= k_end) return 0;  // past the range: never loaded, or masked
    return table[k >> L.shift];
  };
  auto issue = [&](int k, int pg0, int pg1, int stage) -> uint32_t {
    uint32_t bad = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      int pg = b ? pg1 : pg0;
      if ((uint32_t)pg >= (uint32_t)p.pages.num_pages) {
        pg = 0;
        if (k + 16 * b + 16 > R.lo) bad |= 1u << b;  // (rows before the first that is seen may have no page any more)
      }
      const int slot = (k + 16 * b) & slots;
      const int64_t at = 2 * ((int64_t)pg * p.pages.page_stride + head) + (int64_t)slot * rs;
      const uint8_t *pk = reinterpret_cast<const uint8_t *>(L.K) + at;
      const uint8_t *pv = reinterpret_cast<const uint8_t *>(L.V) + at;
      const uint32_t to = lds_at(my + stage * 2 * kTileBytes + b * 16 * kRowBytes);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        load_lds16<NT>(to + i * 4 * kRowBytes, pk + (int64_t)(4 * i) * rs, off[i]);
        load_lds16<NT>(to + kTileBytes + i * 4 * kRowBytes, pv + (int64_t)(4 * i) * rs, off[i]);
      }
    }
    return bad;
  };

  bool gone = false;  // whether a row sees one on a bad page

  // what a row got from values that are not finite, a byte per element (1: +inf, 2: -inf, 3: NaN)
  uint8_t *poison = my + kPoison;
  bool poisoned = false;
  auto start_notes = [&]() {
    if (!poisoned) {
#pragma unroll 1
      for (int i = lane; i < kRows * kHeadDim / 4; i += 64) reinterpret_cast<uint32_t *>(poison)[i] = 0u;
      poisoned = true;
    }
    wave_sync();
  };
  // dims 2 lane .. 2 lane + 1 of a key's value: the rows that see it note what they get; whether any lane noted
  auto note = [&](int key, uint32_t v) {
    const uint32_t v0 = v << 16, v1 = v & 0xffff0000u;
    if (!__any(not_finite(v0) | not_finite(v1))) return false;
    const uint32_t what = poison_of(v0) | poison_of(v1) << 8;
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      uint32_t bit = 1u;
      if constexpr (TREE) bit = masked(b, key) & 1u;
#pragma unroll 1
      for (int j = 0; j < 16; ++j) {
        bool sees = (key >= __shfl(span[b].lo, j)) & (key < __shfl(span[b].hi, j));
        if constexpr (TREE) sees &= __shfl(bit, j) != 0u;
        if (sees) reinterpret_cast<uint16_t *>(poison)[(16 * b + j) * 64 + lane] |= (uint16_t)what;
      }
    }
    return true;
  };

  const float sc2 = L.scale * kLog2e;
  const int stride = kRowsWaves * kTileKeys;
  int k = k_beg + wave * kTileKeys, stage = 0;
  uint32_t bad = 0;
  int pg0 = 0, pg1 = 0;
  if (k < k_end) {
    bad = issue(k, page_of(k), page_of(k + 16), 0);
    pg0 = page_of(k + stride), pg1 = page_of(k + stride + 16);
  }
  bf16x8 Q[NQ][4];  // B operand: column c of block b is query row 16 b + c
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const int row = 16 * b + c;
    const bool ok = span[b].lo < span[b].hi;
    const int j = ok ? token(row) : 0, hq = h * G + (ok ? row - j * G : 0);
    const uint16_t *q = L.q + (sq.t0 + j) * p.q_rows.token_stride + hq * p.q_rows.head_stride;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
      Q[b][kb] = __builtin_bit_cast(bf16x8, ok ? reinterpret_cast<const uint4 *>(q)[4 * kb + g] : make_uint4(0u, 0u, 0u, 0u));
  }

  // (asked for behind the first tile, and here before the next: a wait for them in the loop would be one for all loads)
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) asm volatile("" : "+v"(Q[b][kb]));
    if constexpr (TREE) asm volatile("" : "+v"(word0[b]));
  }

  for (; k < k_end; k += stride, stage ^= 1) {
    uint32_t next_bad = 0;
    if (k + stride < k_end) {
      wait_lds();
      next_bad = issue(k + stride, pg0, pg1, stage ^ 1);
      pg0 = page_of(k + 2 * stride), pg1 = page_of(k + 2 * stride + 16);
      wait_loads<16>();
    } else {
      wait_loads<0>();
    }
    uint8_t *Kt = my + stage * 2 * kTileBytes, *Vt = Kt + kTileBytes;
    // values of rows that no query row may see must not reach a product: 0 x NaN
    if (k + kTileKeys > k_end || bad) {
      const int keep = k_end - k;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + g;
        if (r >= keep || ((bad >> (i / 4)) & 1u))
          *reinterpret_cast<uint4 *>(Vt + r * kRowBytes + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    const bool mixed = bad || k < R.every_lo || k + kTileKeys > min(R.every_hi, k_end);

    // V^T operand of dims 16 d .. + 15
    auto values = [&](int d) {
      const int r = 4 * g + (c >> 2);
      const uint8_t *a = Vt + r * kRowBytes + (((2 * d + ((c & 3) >> 1)) ^ r) * 16) + 8 * (c & 1);
      return join8(read_transposed(a), read_transposed(a + 16 * kRowBytes));
    };
    if (mixed) {
      // some row may not see a key that another sees: an infinity or NaN there must not reach it
      bool top = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(Vt + lane * 16 + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) top |= not_finite(v[e]) | not_finite(v[e] << 16);
      }
      if (__any(top)) {
        start_notes();
#pragma unroll 1
        for (int r = 0; r < kTileKeys; ++r) {  // (rows of bad pages are zeros here)
          uint32_t *at = reinterpret_cast<uint32_t *>(Vt + r * kRowBytes + (((lane >> 2) ^ (r & 15)) * 16) + 4 * (lane & 3));
          const uint32_t v = *at;
          if (note(k + r, v)) *at = (not_finite(v << 16) ? 0u : v & 0xffffu) | (not_finite(v) ? 0u : v & 0xffff0000u);
        }
        wave_sync();
      }
    }
    f32x4 S[NQ][2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int b = 0; b < NQ; ++b) S[b][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        const bf16x8 A = *reinterpret_cast<const bf16x8 *>(Kt + (16 * t + c) * kRowBytes + ((4 * kb + g) ^ c) * 16);
#pragma unroll
        for (int b = 0; b < NQ; ++b)
          S[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, Q[b][kb], S[b][t], 0, 0, 0);
      }
    }
    float w[NQ][8];
    bf16x8 hi[NQ], lo[NQ];
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
      const int own_hi = min(span[b].hi, k_end);
      auto visible = [&](int i) {
        const int key = k + 16 * (i / 4) + 4 * g + i % 4;
        return (key >= span[b].lo) & (key < own_hi) & !((bad >> (i / 4)) & 1u);
      };
#pragma unroll
      for (int i = 0; i < 8; ++i) w[b][i] = S[b][i / 4][i % 4] * sc2;
      if (mixed) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[b][i] = visible(i) ? w[b][i] : -INFINITY;
        if (TREE && k + kTileKeys > R.every_hi) {
          const uint32_t bits = masked(b, k) >> (4 * g);
#pragma unroll
          for (int i = 0; i < 8; ++i) w[b][i] = (bits >> (16 * (i / 4) + i % 4)) & 1u ? w[b][i] : -INFINITY;
        }
      }
      float t = fmaxf(fmaxf(fmaxf(w[b][0], w[b][1]), fmaxf(w[b][2], w[b][3])),
                      fmaxf(fmaxf(w[b][4], w[b][5]), fmaxf(w[b][6], w[b][7])));
      t = max_xor16_32(t);
      if (__any(t > m[b])) {
        const float mn = fmaxf(m[b], t);
        const float a = mn == -INFINITY ? 1.0f : fast_exp2(m[b] - mn);
        m[b] = mn;
        z[b] *= a;
#pragma unroll
        for (int d = 0; d < 8; ++d) O[b][d] *= a;
      }
      const float mu = m[b] == -INFINITY ? 0.0f : m[b];  // nothing seen yet: every l is -inf
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        w[b][i] = fast_exp2(w[b][i] - mu);
        z[b] += w[b][i];
        hi[b][i] = (__bf16)w[b][i];
        lo[b][i] = (__bf16)(w[b][i] - (float)hi[b][i]);
      }
    }
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const bf16x8 A = values(d);
#pragma unroll
      for (int b = 0; b < NQ; ++b) {
        f32x4 &o = O[b][d];
        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, lo[b], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A, hi[b], o, 0, 0, 0);
      }
    }
    if (bad) {
#pragma unroll
      for (int i = 0; i < 2 * NQ; ++i) {
        const int at = k + 16 * (i / NQ);
        if constexpr (TREE) {
          const int row = 16 * (i % NQ) + c;
          if ((bad >> (i / NQ)) & 1u)
            gone |= __any(span[i % NQ].lo < span[i % NQ].hi &&
                          sees_any(L, sq, sq.t0 + token(row), span[i % NQ].lo, at, min(at + 16, span[i % NQ].hi)));
        } else if ((bad >> (i / NQ)) & 1u) {
          gone |= __any((span[i % NQ].lo < at + 16) & (span[i % NQ].hi > at));
        }
      }
    }
    bad = next_bad;
  }
  if (gone && lane == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);
  // Where every row sees all keys of a tile, values enter the products as they are.  A NaN stays one, but an infinity's
  // products with a weight's head and tail differ in sign, or are infinity times zero: the sum is NaN where it should be
  // infinite.  So if a sum is NaN over weights that are not, the wave looks through its values once more, and notes what
  // its rows got of them.
  bool nan = false;
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    z[b] = add_xor32(add_xor16(z[b]));
    f32x4 all = O[b][0];
#pragma unroll
    for (int d = 1; d < 8; ++d) all += O[b][d];
    const float sum = (all[0] + all[1]) + (all[2] + all[3]);
    nan |= (sum != sum) & (z[b] == z[b]);
  }
  if (__any(nan)) {
    start_notes();
#pragma unroll 1
    for (int k0 = k_beg + wave * kTileKeys; k0 < k_end; k0 += stride) {
      if (!any_not_finite(L, s, head, k0, k_end)) continue;
#pragma unroll 1
      for (int key = k0; key < min(k0 + kTileKeys, k_end); ++key) {
        const int64_t at = page_row(p.pages, L.shift, s, key);
        if (at >= 0) note(key, reinterpret_cast<const uint32_t *>(L.V + at + head)[lane]);
      }
    }
    wave_sync();
  }
  // (a NaN weight makes the row's total NaN, and with it what is noted)
  if (poisoned) {
#pragma unroll
    for (int b = 0; b < NQ; ++b) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const uint32_t got = *reinterpret_cast<const uint32_t *>(poison + (16 * b + c) * kHeadDim + 16 * d + 4 * g);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = (got >> (8 * i)) & 3u;
          if (x) O[b][d][i] = poison_value(x);
        }
      }
    }
  }

  // The waves' sums, combined in order; a row that sees nothing keeps none.
  __syncthreads();
  float *Ow = reinterpret_cast<float *>(my);            // [kRows][kMergeRow]
  float2 *mz = reinterpret_cast<float2 *>(Ow + kRows * kMergeRow);  // [kRows]
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    if (g == 0) mz[16 * b + c] = span[b].lo < span[b].hi ? make_float2(m[b], z[b]) : make_float2(-INFINITY, 0.0f);
#pragma unroll
    for (int d = 0; d < 8; ++d) *reinterpret_cast<f32x4 *>(Ow + (16 * b + c) * kMergeRow + 16 * d + 4 * g) = O[b][d];
  }
  __syncthreads();
  const int64_t slot = blockIdx.x;
#pragma unroll
  for (int b = 0; b < NQ; ++b) {
    const int r = 16 * b + (threadIdx.x >> 4), e = (threadIdx.x & 15) * 8;
    float M = -INFINITY, Z = 0.0f, o[8] = {};
#pragma unroll
    for (int v = 0; v < kRowsWaves; ++v)
      M = fmaxf(M, reinterpret_cast<const float2 *>(lds + v * kWaveLds + kRows * kMergeRow * 4)[r].x);
#pragma unroll
    for (int v = 0; v < kRowsWaves; ++v) {
      const float *Ov = reinterpret_cast<const float *>(lds + v * kWaveLds);
      const float2 t = reinterpret_cast<const float2 *>(Ov + kRows * kMergeRow)[r];
      if (t.y == 0.0f) continue;  // this wave saw nothing of the row
      const float a = fast_exp2(t.x - M);
      Z += a * t.y;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] += a * Ov[r * kMergeRow + e + i];
    }
    if (r >= nrow) continue;
    if (L.nsplit > 1) {
      float *part = L.part + (slot * kRows + r) * kHeadDim + e;
      if (e == 0) L.stats[slot * kRows + r] = make_float2(M, Z);
      if (Z == 0.0f) continue;
      *reinterpret_cast<f32x4 *>(part) = f32x4{o[0], o[1], o[2], o[3]};
      *reinterpret_cast<f32x4 *>(part + 4) = f32x4{o[4], o[5], o[6], o[7]};
    } else {
      const int j = token(r);
      store_row(L, sq.t0 + j, h * G + r - j * G, e, M, Z, o);
    }
  }
}

// A wave per query row: each quarter of it takes every fourth split, eight elements a lane, eight splits' loads
// in flight.  Short: what it takes is the latency of one load after another, so the splits' statistics and
// sums are asked for together, before the sequence is known (they lie in the workspace either way), and the weights
// follow (32 splits of a row: 8.4 us one by one, 4.2 by fours behind the sequence, 3.6 so).
__global__ __launch_bounds__(256) void attend_join_kernel(AttendPagedLaunch L) {
  const ebd_attend_paged_params &p = L.p;
  const int H = p.pages.kv_heads, G = p.group;
  const int shift = __builtin_ctz(L.rows) - 2, sub = blockIdx.x & ((1 << shift) - 1), uh = blockIdx.x >> shift;
  const int u = L.by_heads.quotient(uh), h = uh - u * H;
  const int64_t slot0 = (int64_t)uh * L.nsplit;
  const int r = 4 * sub + (threadIdx.x >> 6), lane = threadIdx.x & 63, g = lane >> 4, e = (lane & 15) * 8;
  const float2 *stats = L.stats + slot0 * L.rows + r;
  const float *part = L.part + (slot0 * L.rows + r) * kHeadDim + e;
  const int64_t step = (int64_t)L.rows * kHeadDim;
  constexpr int kMany = 8;
  float2 t[kMany];
  f32x4 x[kMany][2];
  auto load = [&](int v0) {
#pragma unroll
    for (int i = 0; i < kMany; ++i) {
      const int v = v0 + 4 * i + g;
      t[i] = make_float2(-INFINITY, 0.0f);
      if (v >= L.nsplit) continue;
      t[i] = stats[(int64_t)v * L.rows];
      x[i][0] = *reinterpret_cast<const f32x4 *>(part + v * step);
      x[i][1] = *reinterpret_cast<const f32x4 *>(part + v * step + 4);
    }
  };
  load(0);
  const Place at = place_of(L, u);
  if (at.s < 0) return;
  const Seq sq = sequence(p, at.s);
  const int row = at.rb * L.rows + r;
  if (row >= sq.tokens * G || !takes(L, (int64_t)sq.tokens * G)) return;
  float M = -INFINITY, Z = 0.0f, o[8] = {};
  for (int v0 = 0;;) {
    float mn = M;
#pragma unroll
    for (int i = 0; i < kMany; ++i) mn = fmaxf(mn, t[i].x);
    const float a = M == -INFINITY ? 0.0f : fast_exp2(M - mn);
    Z *= a;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= a;
    M = mn;
#pragma unroll
    for (int i = 0; i < kMany; ++i) {
      if (t[i].y == 0.0f) continue;  // nothing seen: its sums were not written
      const float w = fast_exp2(t[i].x - M);
      Z += w * t[i].y;
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] += w * x[i][j / 4][j % 4];
    }
    v0 += 4 * kMany;
    if (v0 >= L.nsplit) break;
    load(v0);
  }
  // the quarters, in a fixed order
  const float all = max_xor16_32(M);
  const float a = M == -INFINITY ? 0.0f : fast_exp2(M - all);
  const bool seen = Z != 0.0f;
  Z = add_xor32(add_xor16(Z * a));
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = add_xor32(add_xor16(seen ? o[j] * a : 0.0f));
  const int j = L.by_group.quotient(row);
  if (g == 0) store_row(L, sq.t0 + j, h * G + row - j * G, e, all, Z, o);
}

size_t attend_paged_part_bytes(const AttendPagedLaunch &L) {
  return L.nsplit > 1 ? (size_t)attend_paged_groups(L) * L.rows * (kHeadDim * sizeof(float) + sizeof(float2)) : 0;
}

int64_t attend_paged_groups(const AttendPagedLaunch &L) {
  return L.units * L.p.pages.kv_heads * L.nsplit;
}

int64_t attend_paged_join_groups(const AttendPagedLaunch &L) {
  return L.nsplit > 1 ? L.units * L.p.pages.kv_heads * (L.rows / 4) : 0;
}

namespace {
template <bool TREE>
hipError_t launch_rows(const AttendPagedLaunch &L, hipStream_t s) {
  const dim3 grid((unsigned)attend_paged_groups(L)), block(64 * kRowsWaves);
  if (L.rows == 16 && L.once) hipLaunchKernelGGL((attend_rows_kernel<1, true, TREE>), grid, block, 0, s, L);
  else if (L.rows == 16) hipLaunchKernelGGL((attend_rows_kernel<1, false, TREE>), grid, block, 0, s, L);
  else if (L.once) hipLaunchKernelGGL((attend_rows_kernel<2, true, TREE>), grid, block, 0, s, L);
  else hipLaunchKernelGGL((attend_rows_kernel<2, false, TREE>), grid, block, 0, s, L);
  return hipGetLastError();
}
}  // namespace

hipError_t launch_attend_paged(const AttendPagedLaunch &L, hipStream_t s) {
  if (L.rows > kRowsKernelMax) return launch_attend_tiles(L, s);
  return L.mask ? launch_rows<true>(L, s) : launch_rows<false>(L, s);
}

hipError_t launch_attend_paged_join(const AttendPagedLaunch &L, hipStream_t s) {
  hipLaunchKernelGGL(attend_join_kernel, dim3((unsigned)attend_paged_join_groups(L)), dim3(256), 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
