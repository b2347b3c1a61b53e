// paged_api.cpp -- the C ABI of the paged cache: argument validation and launch planning.
#include "ebd.h"

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>

#include "ebd_internal.hpp"

namespace {

using namespace ebd;

constexpr int64_t kStrideMax = (int64_t)1 << 40;
constexpr int64_t kRowStrideMax = (int64_t)1 << 26;  // a lane's offset inside 16 rows stays below 32 bits
constexpr int64_t kGridMax = ((int64_t)1 << 24) - 1;  // tokens of a call, query rows of a sequence; groups of 256 threads
constexpr int64_t kRowsMax = (int64_t)1 << 30;         // rows of a sequence
constexpr int32_t kHeadsMax = 65536;

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

bool valid_rows(const ebd_rows &r) {
  return r.token_stride >= 0 && r.head_stride >= 0 && r.token_stride % 8 == 0 && r.head_stride % 8 == 0 &&
         r.token_stride < kStrideMax && r.head_stride < kStrideMax;
}

bool valid_pages(const ebd_pages &P) {
  if (P.num_seqs < 0 || P.kv_heads < 1 || P.num_pages < 1 || P.max_pages < 1 || P.page_size < 1) return false;
  if (P.num_seqs > 0 && !P.page_table) return false;
  if (P.page_stride < 8 || P.head_stride < 8 || P.row_stride < 8) return false;
  if (P.page_stride % 8 || P.head_stride % 8 || P.row_stride % 8) return false;
  return true;
}

bool supported_pages(const ebd_pages &P) {
  return P.head_dim == kHeadDim && P.kv_heads <= kHeadsMax && P.page_size >= 16 && P.page_size <= 65536 &&
         (P.page_size & (P.page_size - 1)) == 0 && P.page_stride < kStrideMax && P.head_stride < kStrideMax &&
         P.row_stride < kRowStrideMax;
}

int32_t log2_of(int32_t n) {
  int32_t s = 0;
  while ((1 << s) < n) ++s;
  return s;
}

bool valid_rotary(const ebd_rotary &R) {
  if (R.rot_dim < 2 || R.rot_dim > kHeadDim || R.rot_dim % 2) return false;
  if (R.layout != EBD_ROPE_HALF && R.layout != EBD_ROPE_PAIRS) return false;
  if ((R.flags & ~EBD_ROPE_INVERSE) != 0u || !std::isfinite(R.amplitude)) return false;
  return ((uintptr_t)R.freq & 7) == 0;
}

float amplitude_of(const ebd_rotary &R) { return R.amplitude != 0.0f ? R.amplitude : 1.0f; }

bool valid_attend_paged(const ebd_attend_paged_params *p) {
  if (!p || !valid_pages(p->pages)) return false;
  if (p->group < 1 || p->max_new < 0 || p->num_tokens < 0 || p->max_rows < 0) return false;
  if (p->window < 0 || p->scale < 0.0f || !std::isfinite(p->scale)) return false;
  return valid_rows(p->q_rows) && valid_rows(p->y_rows);
}

bool supported_attend_paged(const ebd_attend_paged_params *p) {
  return supported_pages(p->pages) && (int64_t)p->group * p->pages.kv_heads <= kHeadsMax &&
         p->num_tokens <= kGridMax && p->max_rows <= kRowsMax && (int64_t)p->max_new * p->group <= kGridMax;
}

// How a launch is cut.  Units (sequence, KV head, block of query rows) are split over the rows they see where that
// ends the launch sooner.  A work-group takes its split's rows and what a start and an end cost, about as long as
// kStartRows more; as many run at once as the chip holds (one a CU, or two of attend_tiles with 128 query rows).  Up
// to two rounds of them the launch ends with its last round, however full; past that the work-groups are out of step
// and end about half of one after each other.  Splits also cost the join: its launch, and the partial sums.  us, 8 KV
// heads of 4 query heads, without the join's cost / with it: 1024 tokens over 1024 rows 44.8 / 33.0, 4 of 256 over
// 1024 51.2 / 34.5, 512 over 512 28.1 / 20.9, one token over 300 rows 13.4 / 11.5; without splits beyond 256
// work-groups / by this rule: 33 sequences of up to 15000 rows (264 units) 218 / 193; by rounds alone / by this rule:
// 32 chunks of up to 512 tokens over up to 8192 rows 939 / 770.  Units that fill the first round, 384, 512, 768 or
// 1024 work-groups / 256: 8 sequences of 16384 rows 95, 94, 93, 97 / 90, 16 of up to 6144 rows 40, 36, 38, 40 / 32.
constexpr int64_t kCus = 256;
constexpr int64_t kRowsLeast = 128;  // fewest rows of a split: a tile for each wave, or eight tiles
// us by 512 / 256 / 128: 64 tokens over 1024 rows 24.5 / 21.1 / 21.0, 128 over 2048 28.4 / 24.7 / 27.6
constexpr int64_t kTilesLeast = 256;
constexpr int64_t kStartRows = 320;
constexpr int64_t kTilesStartRows = 640;
constexpr double kTilesJoin = 250.0;  // (and a row for each 128 query rows' sums, 135 KB written and read)
constexpr double kRowsJoin = 300.0;
constexpr int64_t kSplitsMost = 256;
constexpr int64_t kCacheBytes = (int64_t)64 << 20;

int64_t splits(int64_t units, int64_t span, int64_t slots, int64_t least, int64_t start, double join, double join_each) {
  const int64_t most = std::min<int64_t>(kSplitsMost, std::max<int64_t>(1, span / least));
  int64_t best = 1;
  double cost = 0.0;
  for (int i = 0; i < 16; ++i) {  // one to eight splits, and as many as fill one to eight rounds
    const int64_t ns = std::min(most, i < 8 ? i + 1 : std::max<int64_t>(1, (i - 7) * slots / units));
    const int64_t rows = ((span + ns - 1) / ns + 127) / 128 * 128;
    const int64_t groups = units * ((span + rows - 1) / rows);  // (rounded up, the size may leave fewer splits)
    const double rounds = groups <= 2 * slots ? (double)((groups + slots - 1) / slots) : (double)groups / (double)slots + 0.5;
    const double c = rounds * (double)(rows + start) + (ns > 1 ? join + join_each * (double)groups : 0.0);
    if (i == 0 || c < cost) best = ns, cost = c;
  }
  return best;
}

// A launch for blocks of `rows` query rows; `sum` query rows in all, the sequences' most `rows_max` each, and each of those
// that it takes more than `more_than`.
AttendPagedLaunch attend_paged_part(const ebd_attend_paged_params *p, int32_t rows, int64_t rows_max, int64_t sum,
                                    int64_t more_than = 0) {
  AttendPagedLaunch L{};
  L.p = *p;
  L.rows = rows;
  L.more_than = more_than;
  L.at_most = INT64_MAX;
  const bool tiles = rows >= kTileRows;
  const int64_t S = p->pages.num_seqs, H = p->pages.kv_heads;
  // Every sequence that the launch takes has at most a block that is not full, and some new tokens: a thousand without
  // any, beside a chunk of 64 tokens over 10000 rows, are no blocks (17 with the chunk's: 0.3 GB of partial sums;
  // were they, 17 GB).  Blocks set aside for the longest sequence cost an empty work-group each where there are none (64
  // sequences, one of 2048 tokens: 32768 of them, about 130 us).
  const int64_t aside = std::max<int64_t>(1, (rows_max + rows - 1) / rows);
  const int64_t counted = sum / rows + std::min<int64_t>(S, sum / std::max<int64_t>(p->group, more_than + 1));
  L.blocks = aside > 1 && S * aside > counted + counted / 2 ? 0 : (int32_t)aside;
  L.units = L.blocks ? S * aside : counted;
  // the most rows a block of query rows sees, under a window from a tile's border on
  int64_t span = p->max_rows;
  if (p->window > 0 && !p->qpos) span = std::min<int64_t>(span, (int64_t)p->window + rows / p->group + 1);
  span = std::max<int64_t>(span, 1) + (p->window > 0 ? 63 : 0);
  const int64_t full = std::max<int64_t>(1, L.blocks ? L.units : sum / rows);  // blocks that have work to do
  L.least = (int32_t)(tiles ? kTilesLeast : kRowsLeast);
  if (tiles) {
    L.nsplit = (int32_t)splits(full * H, span, rows == kTileRows ? 2 * kCus : kCus, kTilesLeast, kTilesStartRows,
                               kTilesJoin, (double)rows / kTileRows);
  } else {
    L.nsplit = (int32_t)splits(full * H, span, kCus, kRowsLeast, kStartRows, kRowsJoin, 0.0);
  }
  // keys and values that one work-group alone reads, and too many to stay in the last-level cache until the next call
  // on the same layer (us without / with the hint; groups of 4, 8 KV heads): 32 sequences of 16384 rows 356 / 318, 64 of up
  // to 4096 rows 124 / 111, 16 of up to 6144 rows, 8 tokens, eight layers in turn, 46.1 / 42.9; one of 4096 rows,
  // found in the cache, 14.4 / 15.3
  L.once = aside == 1 && S * H * span * 4 * kHeadDim > kCacheBytes;
  L.by_group.set(p->group);
  L.by_heads.set(H);
  L.by_blocks.set(std::max<int32_t>(L.blocks, 1));
  L.by_nsplit.set(L.nsplit);
  L.shift = log2_of(p->pages.page_size);
  L.scale = p->scale > 0.0f ? p->scale : 1.0f / std::sqrt((float)kHeadDim);
  return L;
}

// The launches of a call.  One serves every sequence, in blocks that fit the longest chunk.  Where most sequences must
// have far fewer new tokens than that (a prompt's chunk beside decode steps), those of up to 16 query rows (32 with
// more query heads than that) get a launch of their own: us with one launch / with two, 8 KV heads of 4 query heads:
// 2048 tokens over 4096 rows and 63 single ones over 8192: 857 / 507; 512 over 131072 and 31 over 4096: 2540 / 1155.
struct AttendPagedPlan {
  AttendPagedLaunch part[2];
  int parts;
};
// Whether blocks of 256 query rows, one work-group a CU, serve a call: they load every tile half as often, and have
// nothing to run under a start, an end or another's shorter block.  So only where the work-groups fill the chip once,
// the blocks are full and see about the same rows, which a call knows of one sequence.  us by 128 rows / by 256, 8 KV
// heads of 4 query heads, taken: 1024 tokens over 131072 rows 2197 / 2053, 32768 558 / 540, under a window of 2048 71 / 68,
// 2048 over 16384 513 / 504, 512 over 4096 61 / 60; not taken: 8192 over 8192 571 / 567, 2048 over 8192 257 / 265, 1500
// over 6000 167 / 180, 256 over 1024 30 / 35, 160 (a block half empty) over 32768 122 / 130; 8 ragged sequences of up to
// 256 over up to 16384 320 / 420.
bool long_blocks(const ebd_attend_paged_params *p, int64_t most) {
  if (p->pages.num_seqs != 1 || most < kLongRows || (int64_t)p->max_new * 8 > p->max_rows) return false;
  const AttendPagedLaunch L = attend_paged_part(p, kLongRows, most, std::min<int64_t>(p->num_tokens * p->group, most));
  const int64_t groups = attend_paged_groups(L), rows = (most + kLongRows - 1) / kLongRows * kLongRows;
  return groups <= kCus && 8 * groups >= 7 * kCus && 8 * most >= 7 * rows;
}
AttendPagedPlan attend_paged_plan(const ebd_attend_paged_params *p) {
  const int64_t S = p->pages.num_seqs, G = p->group, most = (int64_t)p->max_new * G;
  const int64_t sum = std::min<int64_t>(p->num_tokens * G, S * most);
  const int32_t rows = most <= 16 ? 16 : most <= kRowsKernelMax ? 32 : most <= kFewRows ? kFewRows : kTileRows;
  AttendPagedPlan plan;
  plan.parts = 1;
  if (rows == kTileRows && S > 1 && G <= kRowsKernelMax && 4 * (sum - most) <= (S - 1) * most) {
    const int32_t small = G <= 16 ? 16 : kRowsKernelMax;
    plan.parts = 2;
    plan.part[1] = attend_paged_part(p, small, small, S * small);
    plan.part[1].at_most = small;
    plan.part[0] = attend_paged_part(p, rows, most, sum, small);
  } else if (long_blocks(p, most)) {
    plan.part[0] = attend_paged_part(p, kLongRows, most, sum);
  } else {
    plan.part[0] = attend_paged_part(p, rows, most, sum);
  }
  return plan;
}

size_t part_bytes(const AttendPagedLaunch &L) { return (attend_paged_part_bytes(L) + 255) / 256 * 256; }
size_t plan_bytes(const AttendPagedPlan &plan) {
  size_t bytes = 256;
  for (int i = 0; i < plan.parts; ++i) bytes += part_bytes(plan.part[i]);
  return bytes;
}

}  // namespace

namespace ebd {

size_t attend_paged_workspace(const ebd_attend_paged_params *p) {
  if (!valid_attend_paged(p) || !supported_attend_paged(p)) return 0;
  return plan_bytes(attend_paged_plan(p));
}

}  // namespace ebd

extern "C" {

ebd_status ebd_rope(const ebd_rope_params *p, const uint16_t *x, uint16_t *y, void *stream) {
  if (!p || p->num_tokens < 0 || p->num_heads < 0 || p->reserved != 0) return EBD_ERR_INVALID_ARG;
  if (!valid_rotary(p->rot) || !valid_rows(p->x) || !valid_rows(p->y)) return EBD_ERR_INVALID_ARG;
  if (p->head_dim != kHeadDim || p->num_tokens > kGridMax || p->num_heads > kHeadsMax) return EBD_ERR_UNSUPPORTED;
  if (p->num_tokens == 0 || p->num_heads == 0) return EBD_OK;
  if (!x || !y || !p->pos || !p->rot.freq || !aligned16(x) || !aligned16(y)) return EBD_ERR_INVALID_ARG;
  const ebd_status ds = device_ok();
  if (ds != EBD_OK) return ds;
  RopeLaunch L{};
  L.p = *p;
  L.p.rot.amplitude = amplitude_of(p->rot);
  L.x = x;
  L.y = y;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return timed_launch("rope", s, [&] { return launch_rope(L, s); }) == hipSuccess ? EBD_OK : EBD_ERR_HIP;
}

ebd_status ebd_append_paged(const ebd_append_paged_params *p, const uint16_t *k_new,
                            const uint16_t *v_new, uint16_t *K, uint16_t *V, const uint16_t *q,
                            uint16_t *q_out, uint32_t *status, void *stream) {
  if (!p || !valid_pages(p->pages) || p->num_tokens < 0 || p->q_heads < 0 || p->reserved != 0)
    return EBD_ERR_INVALID_ARG;
  if (p->rot.freq && !valid_rotary(p->rot)) return EBD_ERR_INVALID_ARG;
  if (!valid_rows(p->k_rows) || !valid_rows(p->v_rows) || !valid_rows(p->q_rows) || !valid_rows(p->q_out_rows))
    return EBD_ERR_INVALID_ARG;
  if (!supported_pages(p->pages) || p->num_tokens > kGridMax || p->q_heads > kHeadsMax) return EBD_ERR_UNSUPPORTED;
  if (p->num_tokens == 0 || p->pages.num_seqs == 0) return EBD_OK;
  if (!k_new || !v_new || !K || !V || !p->new_off || !p->len) return EBD_ERR_INVALID_ARG;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(K) || !aligned16(V)) return EBD_ERR_INVALID_ARG;
  if ((p->q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr)) return EBD_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(q_out)) return EBD_ERR_INVALID_ARG;
  const ebd_status ds = device_ok();
  if (ds != EBD_OK) return ds;
  AppendPagedLaunch L{};
  L.p = *p;
  L.p.rot.amplitude = amplitude_of(p->rot);
  L.k_new = k_new;
  L.v_new = v_new;
  L.q = q;
  L.K = K;
  L.V = V;
  L.q_out = q_out;
  L.status = status;
  L.shift = log2_of(p->pages.page_size);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return timed_launch("append_paged", s, [&] { return launch_append_paged(L, s); }) == hipSuccess ? EBD_OK
                                                                                                   : EBD_ERR_HIP;
}

ebd_status ebd_attend_paged(const ebd_attend_paged_params *p, const uint16_t *q, const uint16_t *K,
                            const uint16_t *V, uint16_t *y, float *lse, uint32_t *status,
                            void *workspace, size_t ws_bytes, void *stream) {
  if (!valid_attend_paged(p)) return EBD_ERR_INVALID_ARG;
  if (!supported_attend_paged(p)) return EBD_ERR_UNSUPPORTED;
  if (p->num_tokens == 0 || p->pages.num_seqs == 0) return EBD_OK;
  if (p->max_new == 0 || !q || !K || !V || !y || !p->new_off || !p->len) return EBD_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(K) || !aligned16(V) || !aligned16(y) || ((uintptr_t)lse & 3))
    return EBD_ERR_INVALID_ARG;
  AttendPagedPlan plan = attend_paged_plan(p);
  for (int i = 0; i < plan.parts; ++i)
    if (attend_paged_groups(plan.part[i]) > kGridMax / 2 || attend_paged_join_groups(plan.part[i]) > kGridMax)
      return EBD_ERR_UNSUPPORTED;
  if (!workspace || ws_bytes < plan_bytes(plan) || ((uintptr_t)workspace & 255)) return EBD_ERR_WORKSPACE;
  const ebd_status ds = device_ok();
  if (ds != EBD_OK) return ds;
  hipStream_t s = static_cast<hipStream_t>(stream);
  char *ws = static_cast<char *>(workspace);
  for (int i = 0; i < plan.parts; ++i) {
    AttendPagedLaunch &L = plan.part[i];
    L.q = q;
    L.K = K;
    L.V = V;
    L.y = y;
    L.lse = lse;
    L.status = status;
    L.part = reinterpret_cast<float *>(ws);
    L.stats = reinterpret_cast<float2 *>(L.part + attend_paged_groups(L) * L.rows * kHeadDim);
    ws += part_bytes(L);
    if (timed_launch("attend_paged", s, [&] { return launch_attend_paged(L, s); }) != hipSuccess) return EBD_ERR_HIP;
    if (L.nsplit > 1 &&
        timed_launch("attend_paged_join", s, [&] { return launch_attend_paged_join(L, s); }) != hipSuccess)
      return EBD_ERR_HIP;
  }
  return EBD_OK;
}

ebd_status ebd_gather_paged(const ebd_gather_paged_params *p, const uint16_t *K, const uint16_t *V,
                            uint16_t *Ku, uint16_t *Vu, uint32_t *status, void *stream) {
  if (!p || !valid_pages(p->pages) || p->max_rows < 0 || p->num_rows < 0) return EBD_ERR_INVALID_ARG;
  if (!supported_pages(p->pages) || p->max_rows > kRowsMax || gather_paged_groups(*p) > kGridMax) return EBD_ERR_UNSUPPORTED;
  if (p->pages.num_seqs == 0 || p->max_rows == 0) return EBD_OK;
  if (!K || !V || !Ku || !Vu || !p->seq_off) return EBD_ERR_INVALID_ARG;
  if (!aligned16(K) || !aligned16(V) || !aligned16(Ku) || !aligned16(Vu)) return EBD_ERR_INVALID_ARG;
  const ebd_status ds = device_ok();
  if (ds != EBD_OK) return ds;
  GatherPagedLaunch L{};
  L.p = *p;
  L.K = K;
  L.V = V;
  L.Ku = Ku;
  L.Vu = Vu;
  L.status = status;
  L.shift = log2_of(p->pages.page_size);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return timed_launch("gather_paged", s, [&] { return launch_gather_paged(L, s); }) == hipSuccess ? EBD_OK
                                                                                                   : EBD_ERR_HIP;
}

}  // extern "C"
