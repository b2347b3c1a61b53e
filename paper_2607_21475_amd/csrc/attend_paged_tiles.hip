// attend_paged_tiles.hip -- attention of many query rows over a paged cache on gfx950 (prompts, long chunks).
//
// attend_tiles: one work-group per (sequence, KV head, block of 256 query rows, split of the rows they see), eight
//   waves of 32 query rows each.  Tiles of 64 keys and values pass through LDS, the next one on its way (loads
//   that write LDS directly) while the waves compute the present one; one barrier a tile.
//   S^T = K Q^T on MFMA 32x32x16 bf16 (exact products, fp32 sums): a lane holds half of the 64 scores of
//   one query row, so maxima and sums are register operations and one swap of the wave's halves, and the
//   weights, rounded to bf16, are the B operand of O^T = V^T W^T as they stand, with the keys of a k block in
//   the order 4h .. 4h+3, 8+4h .. 8+4h+3 of half h.  V^T comes from the row-major tile by transposing LDS reads.
//   The 16-byte chunks of a tile's row r are stored at chunk ^ turn(r): rows that are read together (eight by
//   the transposing reads, 32 by the key reads) then spread over all banks.
//   The matrix products bound it: 4 x 128 operations per (query row, key), against which the weights' bf16
//   rounding (half a step, 2^-8, and averaged over a row's keys) saves a second product with their tails.
//   The running maximum moves only when a score exceeds it by 2^8 (weights stay below that; fp32 and
//   bf16 keep their relative precision), so that most tiles scale nothing.
#include "attend_paged.hpp"

namespace ebd {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kKeys = 64;                    // keys per tile
constexpr int kTile = kKeys * kRowBytes;     // bytes of its K, or of its V
constexpr int kStage = 2 * kTile;
constexpr int kWaves = 8;
constexpr float kLazy = 8.0f;

__device__ __forceinline__ int chunk_turn(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }

__device__ __forceinline__ float max_halves(float x) {
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace

__global__ __launch_bounds__(64 * kWaves, 2) void attend_tiles_kernel(AttendPagedLaunch L) {
  __shared__ __align__(1024) uint8_t tiles[2 * kStage];
  __shared__ float weights[kWaves][kKeys][32];  // of a tile that is summed key by key (below)
  __shared__ Range ranges[kWaves];
  __shared__ int bad_pages;
  const ebd_attend_paged_params &p = L.p;
  const int H = p.pages.kv_heads, G = p.group;
  // heads vary fastest (work-groups go round the XCDs: a head's stay together for 8, 4, 2 heads and
  // share its keys through the XCD's L2), then query blocks, the last (which see most) first
  int bid = blockIdx.x;
  const int h = bid % H;
  bid /= H;
  const int rb = L.blocks - 1 - bid % L.blocks;
  bid /= L.blocks;
  const int sp = bid % L.nsplit, s = bid / L.nsplit;
  const int lane = threadIdx.x & 63, half = lane >> 5, c = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  const Seq sq = sequence(p, s);
  const int row0 = rb * 32 * kWaves, nrow = min(32 * kWaves, sq.tokens * G - row0);
  if (threadIdx.x == 0 && rb == 0 && sp == 0 && h == 0 && L.status && sq.status) atomicOr(&L.status[s], sq.status);
  if (nrow <= 0) return;

  // what this wave's rows see, and the work-group's
  const int row = row0 + 32 * wave + c;
  Span span[1] = {span_of(p, sq, row)};
  const bool sees = span[0].lo < span[0].hi;
  const Range R = range_of<1>(span);
  if (threadIdx.x == 0) bad_pages = 0;
  if (lane == 0) ranges[wave] = R;
  __syncthreads();
  int lo = INT32_MAX, hi = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    lo = min(lo, ranges[w].lo);
    hi = max(hi, ranges[w].hi);
  }
  const int64_t start = (lo & -kKeys) + (int64_t)sp * L.split_rows;
  const int k_end = start < hi ? (int)min((int64_t)hi, start + L.split_rows) : 0;
  const int k_beg = start < hi ? (int)start : 0;

  const const_i32 *table = (const const_i32 *)(p.pages.page_table + (int64_t)s * p.pages.max_pages);
  const int slots = p.pages.page_size - 1;
  {
    bool bad = false;
    if (k_end > k_beg)
      for (int e = (k_beg >> L.shift) + (int)threadIdx.x; e <= (k_end - 1) >> L.shift; e += 64 * kWaves)
        bad |= (uint32_t)table[e] >= (uint32_t)p.pages.num_pages;
    if (bad) bad_pages = 1;
  }

  bf16x8 Q[8];  // B operand: column c is this lane's query row, dims 16 kb + 8 half .. + 7
  {
    const int j = sees ? row / G : 0, hq = h * G + (sees ? row % G : 0);
    const uint16_t *q = L.q + (sq.t0 + j) * p.q_rows.token_stride + hq * p.q_rows.head_stride;
#pragma unroll
    for (int kb = 0; kb < 8; ++kb)
      Q[kb] = __builtin_bit_cast(bf16x8, sees ? reinterpret_cast<const uint4 *>(q)[2 * kb + half] : make_uint4(0u, 0u, 0u, 0u));
  }
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) asm volatile("" : "+v"(Q[kb]));
  __syncthreads();
  const bool any_bad = __builtin_amdgcn_readfirstlane(bad_pages) != 0;
  if (any_bad && threadIdx.x == 0 && L.status) atomicOr(&L.status[s], EBD_ST_BAD_PAGE);

  // this wave's part of a tile: rows 8 wave .. + 7, four rows a load, of K and of V
  const uint32_t rs = (uint32_t)p.pages.row_stride * 2u;
  uint32_t off[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 8 * wave + 4 * i + (lane >> 4);
    off[i] = (uint32_t)(lane >> 4) * rs + (uint32_t)((lane & 15) ^ chunk_turn(r)) * 16u;
  }
  const int64_t head = (int64_t)h * p.pages.head_stride;
  auto page_of = [&](int k) -> int { return k < k_end ? table[k >> L.shift] : 0; };
  auto issue = [&](int k, int pg, int stage) {
    if ((uint32_t)pg >= (uint32_t)p.pages.num_pages) pg = 0;  // its rows are masked
    const int slot = (k + 8 * wave) & slots;
    const int64_t at = 2 * ((int64_t)pg * p.pages.page_stride + head) + (int64_t)slot * rs;
    const uint8_t *pk = reinterpret_cast<const uint8_t *>(L.K) + at, *pv = reinterpret_cast<const uint8_t *>(L.V) + at;
    const uint32_t to = lds_at(tiles + stage * kStage + 8 * wave * kRowBytes);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      load_lds16(to + i * 4 * kRowBytes, pk + (int64_t)(4 * i) * rs, off[i]);
      load_lds16(to + kTile + i * 4 * kRowBytes, pv + (int64_t)(4 * i) * rs, off[i]);
    }
  };

  // LDS offsets: K operand rows c, dims 16 kb + 8 half; V operand rows 4 half + c16 / 4 (+ 8)
  uint32_t ka[8], va[4][2];
#pragma unroll
  for (int kb = 0; kb < 8; ++kb) ka[kb] = c * kRowBytes + ((2 * kb + half) ^ chunk_turn(c)) * 16;
  const int c16 = lane & 15, q16 = (lane >> 4) & 1;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int r = 4 * half + (c16 >> 2) + 8 * u;
      va[d][u] = kTile + r * kRowBytes + ((4 * d + 2 * q16 + ((c16 & 3) >> 1)) ^ chunk_turn(r)) * 16 + 8 * (c16 & 1);
    }
  }

  f32x16 O[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) O[d] = f32x16{};
  float m = -INFINITY, z = 0.0f;
  const float sc2 = L.scale * kLog2e;

  auto step = [&](int k, const uint8_t *T, uint32_t bad) {
    const bool mixed = bad || k < R.every_lo || k + kKeys > min(R.every_hi, k_end);
    f32x16 S[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      S[b] = f32x16{};
#pragma unroll
      for (int kb = 0; kb < 8; ++kb)
        S[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(T + ka[kb] + b * 32 * kRowBytes), Q[kb], S[b], 0, 0, 0);
    }
    const int own_hi = min(span[0].hi, k_end);
    auto visible = [&](int b, int i) {
      const int key = k + 32 * b + 8 * (i / 4) + 4 * half + i % 4;
      return (key >= span[0].lo) & (key < own_hi) & !((bad >> (2 * b + i / 8)) & 1u);
    };
    if (mixed) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) S[b][i] = visible(b, i) ? S[b][i] : -INFINITY;
      }
    }
    float t = fmaxf(S[0][0], S[1][0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) t = fmaxf(t, fmaxf(S[0][i], S[1][i]));
    t = max_halves(t) * sc2;
    if (__any(t > m + kLazy)) {
      const float mn = fmaxf(m, t);
      const float a = mn == -INFINITY ? 1.0f : fast_exp2(m - mn);
      m = mn;
      z *= a;
#pragma unroll
      for (int d = 0; d < 4; ++d) O[d] *= a;
    }
    const float mu = m == -INFINITY ? 0.0f : m;  // nothing seen yet: every score is -inf
    bf16x8 W[4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        S[b][i] = fast_exp2(__builtin_fmaf(S[b][i], sc2, -mu));
        z += S[b][i];
        W[2 * b + i / 8][i % 8] = (__bf16)S[b][i];
      }
    }
    auto values = [&](int d, int ks) {
      return join8(read_transposed(T + va[d][0] + ks * 16 * kRowBytes), read_transposed(T + va[d][1] + ks * 16 * kRowBytes));
    };
    bool special = false;
    if (mixed) {
      // some row may not see a key that another sees: an infinity or NaN there must not reach it
      bool top = false;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const u32x4 v = *reinterpret_cast<const u32x4 *>(T + kTile + lane * 16 + i * 1024);
#pragma unroll
        for (int e = 0; e < 4; ++e) top |= ((v[e] & 0x7f80u) == 0x7f80u) | ((v[e] & 0x7f800000u) == 0x7f800000u);
      }
      special = __any(top);
    }
    if (!special) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
#pragma unroll
        for (int d = 0; d < 4; ++d) O[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(values(d, ks), W[ks], O[d], 0, 0, 0);
      }
    } else {
      // the same sums key by key, those that a row does not see left out
      float(*w)[32] = weights[wave];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[32 * b + 8 * (i / 4) + 4 * half + i % 4][c] = visible(b, i) ? S[b][i] : -1.0f;
      }
      wave_sync();
#pragma unroll 1
      for (int r = 0; r < kKeys; ++r) {
        const float wk = w[r][c];
        const bool ok = !(wk < 0.0f);  // a NaN weight counts
#pragma unroll
        for (int d = 0; d < 4; ++d) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const u32x2 v = *reinterpret_cast<const u32x2 *>(T + kTile + r * kRowBytes + ((4 * d + j) ^ chunk_turn(r)) * 16 + 8 * half);
            O[d][4 * j + 0] += ok ? wk * bf16_lo(v[0]) : 0.0f;
            O[d][4 * j + 1] += ok ? wk * bf16_hi(v[0]) : 0.0f;
            O[d][4 * j + 2] += ok ? wk * bf16_lo(v[1]) : 0.0f;
            O[d][4 * j + 3] += ok ? wk * bf16_hi(v[1]) : 0.0f;
          }
        }
      }
      wave_sync();
    }
  };

  int k = k_beg, stage = 0, pg = 0;
  if (k < k_end) {
    issue(k, page_of(k + 8 * wave), 0);
    pg = page_of(k + kKeys + 8 * wave);
  }
  for (; k < k_end; k += kKeys, stage ^= 1) {
    wait_loads<0>();
    __syncthreads();  // the tile is here, and the other one has been read
    if (k + kKeys < k_end) {
      issue(k + kKeys, pg, stage ^ 1);
      pg = page_of(k + 2 * kKeys + 8 * wave);
    }
    uint32_t bad = 0;
    if (any_bad) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
        bad |= (uint32_t)((uint32_t)page_of(k + 16 * b) >= (uint32_t)p.pages.num_pages) << b;
    }
    uint8_t *T = tiles + stage * kStage;
    if (k + kKeys > k_end || bad) {
      // values of rows that no query row may see must not reach a product: 0 x NaN
      const int r = 8 * wave + (lane >> 4);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int rr = r + 4 * i;
        if (k + rr >= k_end || ((bad >> (rr / 16)) & 1u))
          *reinterpret_cast<uint4 *>(T + kTile + rr * kRowBytes + (lane & 15) * 16) = make_uint4(0u, 0u, 0u, 0u);
      }
      __syncthreads();
    }
    if (k < R.hi && k + kKeys > R.lo) step(k, T, bad);
  }

  z += __shfl_xor(z, 32);
  if (32 * wave + c >= nrow) return;
  const int64_t slot = ((((int64_t)s * H + h) * L.blocks + rb) * L.nsplit + sp) * (32 * kWaves) + 32 * wave + c;
  if (L.nsplit > 1) {
    if (half == 0) L.stats[slot] = sees ? make_float2(m, z) : make_float2(-INFINITY, 0.0f);
    if (!sees || m == -INFINITY) return;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4 *>(L.part + slot * kHeadDim + 32 * d + 8 * j + 4 * half) =
            f32x4{O[d][4 * j], O[d][4 * j + 1], O[d][4 * j + 2], O[d][4 * j + 3]};
    }
    return;
  }
  const bool any = sees && m != -INFINITY;
  const float a = any ? 1.0f / z : 0.0f;
  const int64_t t = sq.t0 + row / G;
  const int hq = h * G + row % G;
  uint16_t *y = L.y + t * p.y_rows.token_stride + hq * p.y_rows.head_stride + 4 * half;
#pragma unroll
  for (int d = 0; d < 4; ++d) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u32x2 v;
      v[0] = any ? pack_bf16(O[d][4 * j] * a, O[d][4 * j + 1] * a) : 0u;
      v[1] = any ? pack_bf16(O[d][4 * j + 2] * a, O[d][4 * j + 3] * a) : 0u;
      *reinterpret_cast<u32x2 *>(y + 32 * d + 8 * j) = v;
    }
  }
  if (half == 0 && L.lse) L.lse[t * ((int64_t)H * G) + hq] = any ? (m + fast_log2(z)) * kLn2 : -INFINITY;
}

hipError_t launch_attend_tiles(const AttendPagedLaunch &L, hipStream_t s) {
  hipLaunchKernelGGL(attend_tiles_kernel, dim3((unsigned)attend_paged_groups(L)), dim3(64 * kWaves), 0, s, L);
  return hipGetLastError();
}

}  // namespace ebd
