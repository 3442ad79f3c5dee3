// C ABI of attention of chunks of new tokens over a paged cache: argument
// validation, room for the plan and the partial outputs, launches.  Declarations
// and contracts: include/bdlm_attn.h.
#include "bdlm_attn.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "cache_check.hpp"
#include "chunk.hpp"
#include "split_plan.hpp"

using namespace bdlm;

namespace {

constexpr int64_t kMaxLen = (int64_t)1 << 28;     // blocks, windows, sinks
constexpr int64_t kMaxStride = (int64_t)1 << 30;
static_assert(BDLM_CHUNK_STARTS == kChunkHead * sizeof(int32_t), "the plan's layout is the header's");

// Workgroups that run at once, of which the planner fills up to two rounds by cutting, and keys of a chunk at least.
// Where no walk can have more than twice as many, none is cut, and no merge is launched (one request of 400 keys, 32/8
// heads, d 128, cut in two 11.0 us and 6.4 for the merge, whole 13.7; 8/2 heads fp32 14.5 and 6.4, 20.0; chunks of 512 at least
// everywhere: one request of 1,000 keys 11.5 -> 14.0 us, 64 rows behind 1,000 15.8 -> 20.4).
constexpr int64_t kSlots = 2 * kCus, kSlotsF32 = kCus, kLeast = 256;
static_assert((kSlots & (kSlots - 1)) == 0 && (kSlotsF32 & (kSlotsF32 - 1)) == 0, "the planner shifts by them");

// What a plan and a call's partial outputs need, whatever the lengths are
// (chunk_plan.hip says why it is enough).
struct Room {
  int64_t items, joins, part_rows;
  int32_t limit, least;
  size_t plan_bytes, part_bytes, lse_bytes;
  uint64_t key;  // of the sizes that a plan is made for, not 0
};

// Keys of a chunk at least, with walks of up to `longest` keys.
int64_t least_keys(int64_t longest, int64_t limit) { return longest <= 2 * kLeast ? 2 * kLeast : std::min(kLeast, limit - 64); }

// Items, units of the merge and partial rows, with walks of up to `longest` keys.
struct Bounds {
  int64_t items, joins, part_rows;
};
Bounds bounds(const bdlm_cache* c, const bdlm_chunk* p, int64_t tiles, int64_t longest, int64_t limit) {
  const bool f32 = c->dtype == BDLM_F32;
  const int64_t all = p->rows * (p->heads / c->kv_heads);  // query rows of a KV head
  // chunks beyond the first of each tile: by the share, or by the limit (n_cut of a tile at most); n_least of a tile
  // where every chunk is as short as it may be
  const int64_t by_share = 2 * (f32 ? kSlotsF32 : kSlots) / c->kv_heads + 1;
  const int64_t n_cut = longest / (limit - 64), by_limit = tiles * n_cut;
  const int64_t n_least = std::max<int64_t>(longest - 1, 0) / least_keys(longest, limit), by_least = tiles * n_least;
  const int64_t more = std::min(std::max(by_share, by_limit), by_least);
  Bounds b{};
  if (tiles == 0) return b;
  b.items = tiles + more;
  // units of the merge, of cut tiles: of join_rows rows, or of one in those of more than kShortJoin chunks
  b.joins = std::min(tiles, more) * ((kPrefixSharedRows + join_rows(c->head_dim) - 1) / join_rows(c->head_dim)) +
            std::min(std::min(tiles, more / kShortJoin) * kPrefixSharedRows, all);
  // rows of cut tiles' chunks: at most a tile's of twice as many chunks, and as many as all rows have in that many chunks
  const int64_t tile = f32 ? kPrefixRowsF32 : all > 2 * kPrefixWaveRows ? kPrefixSharedRows : kPrefixWaveRows;
  const int64_t rows = std::max(std::min(2 * by_share * tile, all * (by_share + 1)), std::min(2 * by_limit * tile, all * (n_cut + 1)));
  b.part_rows = more == 0 ? 0 : std::min(rows, std::min(2 * by_least * tile, all * (n_least + 1)));
  return b;
}

// One number for some (each is mixed in by steps that lose nothing of those before).
uint64_t key_of(std::initializer_list<int64_t> xs) {
  uint64_t h = 0;
  for (const int64_t x : xs) {
    h = (h ^ (uint64_t)x) * 0x9e3779b97f4a7c15ull;
    h ^= h >> 29;
  }
  return h ? h : 1;
}

bdlm_status check_chunk(const bdlm_cache* c, const bdlm_chunk* p, Room& room) {
  const bdlm_status st = check_cache(c);
  if (st != BDLM_OK) return st;
  if (!p) return fail(BDLM_ERR_INVALID, "chunk is null");
  if (p->heads < 1 || p->heads % c->kv_heads != 0)
    return fail(BDLM_ERR_INVALID, "heads (%d) must be a positive multiple of kv_heads (%d)", p->heads, c->kv_heads);
  if (p->requests < 0 || p->requests > kMaxSeqs)
    return fail(BDLM_ERR_INVALID, "requests %lld outside [0, 2^19]", (long long)p->requests);
  if (p->rows < 0) return fail(BDLM_ERR_INVALID, "rows %lld is negative", (long long)p->rows);
  if (p->rows > kMaxRows / p->heads)
    return fail(BDLM_ERR_UNSUPPORTED, "rows %lld x heads %d exceeds 2^25", (long long)p->rows, p->heads);
  if (p->block_size < 1 || p->block_size > kMaxLen)
    return fail(BDLM_ERR_INVALID, "block_size must be in [1, 2^28] (got %lld)", (long long)p->block_size);
  if (p->window < 0 || p->window > kMaxLen)
    return fail(BDLM_ERR_INVALID, "window must be in [0, 2^28] (got %lld)", (long long)p->window);
  if (p->sinks < 0 || p->sinks > kMaxLen) return fail(BDLM_ERR_INVALID, "sinks must be in [0, 2^28] (got %d)", p->sinks);
  if (p->reserved != 0) return fail(BDLM_ERR_INVALID, "reserved field must be 0");
  if (!std::isfinite(p->scale)) return fail(BDLM_ERR_INVALID, "scale is not finite");
  const bool f32 = c->dtype == BDLM_F32;
  // (groups of 16 tokens are numbered in 31 bits)
  if (c->page_size > ((int64_t)1 << 34) / c->pages)
    return fail(BDLM_ERR_UNSUPPORTED, "pages %lld x page_size %lld exceeds 2^34", (long long)c->pages, (long long)c->page_size);
  const int64_t group = p->heads / c->kv_heads, all = p->rows * group;  // query rows of a KV head
  const int64_t some = std::min(p->requests, p->rows);                  // requests with rows
  // tiles: of 16 rows; or of 32 in requests of up to 64, else of 128
  const int64_t tiles = f32 ? some + all / kPrefixRowsF32
                            : std::min(some + all / kPrefixWaveRows, 2 * some + all / kPrefixSharedRows);
  // keys whose pages (or groups) a workgroup can hold, in two runs
  room.limit = (int32_t)std::min<int64_t>(!f32 && c->page_size % 16 == 0 ? (kChunkGroups - 2) * 16
                                                                         : (kPrefixTableEntries - 4) * c->page_size,
                                          (int64_t)1 << 29);
  // keys of a walk: what a table holds; with a window its own, the sinks, and those between the windows of a tile's rows
  const int64_t top = c->max_pages * c->page_size;
  const int64_t seen = p->window > 0 ? p->sinks + p->window + p->block_size + kPrefixSharedRows + 32 : top;
  const int64_t longest = std::min(top, seen);
  const Bounds most = bounds(c, p, tiles, top, room.limit), here = bounds(c, p, tiles, longest, room.limit);
  room.least = (int32_t)least_keys(longest, room.limit);
  room.items = here.items;
  room.joins = here.joins;
  room.part_rows = here.part_rows;
  if (room.items * c->kv_heads > kMaxWgs || room.part_rows >= kSharedTile)
    return fail(BDLM_ERR_UNSUPPORTED, "attention over the cache may need %lld workgroups (limit 2^22)",
                (long long)(room.items * c->kv_heads));
  // (the same for every window: a plan may be made anew with another one)
  room.plan_bytes = (size_t)(kChunkHead + 2 * p->requests + 1) * sizeof(int32_t) + most.items * sizeof(ChunkItemRec) +
                    most.joins * sizeof(ChunkJoin);
  const size_t parts = (size_t)room.part_rows * c->kv_heads;
  room.part_bytes = align256(parts * c->head_dim * sizeof(float));
  room.lse_bytes = align256(parts * (f32 ? sizeof(PartLse<false>) : sizeof(PartLse<true>)));
  room.key = key_of({c->dtype, c->kv_heads, c->head_dim, c->page_size, c->max_pages, c->seqs, p->requests, p->rows, p->heads,
                     p->block_size, p->window, p->window > 0 ? p->sinks : 0});
  return BDLM_OK;
}

bdlm_status check_rows(const bdlm_rows& r, const char* what, int64_t row_elems, int elem) {
  if (!r.ptr || !aligned16(r.ptr)) return fail(BDLM_ERR_INVALID, "%s is null or not 16-byte aligned", what);
  if (r.stride < row_elems || r.stride > kMaxStride || r.stride * elem % 16 != 0)
    return fail(BDLM_ERR_INVALID, "%s row stride %lld outside [%lld, 2^30] or not a multiple of 16 bytes", what,
                (long long)r.stride, (long long)row_elems);
  return BDLM_OK;
}

bdlm_status check_plan(const void* plan, size_t bytes, const Room& room) {
  if (!plan || (reinterpret_cast<uintptr_t>(plan) & 15u) || bytes < room.plan_bytes)
    return fail(BDLM_ERR_INVALID, "plan needs %zu bytes, 16-byte aligned (got %zu at %p)", room.plan_bytes, bytes, plan);
  return BDLM_OK;
}

}  // namespace

extern "C" {

size_t bdlm_chunk_plan_bytes(const bdlm_cache* c, const bdlm_chunk* p) {
  Room room;
  return check_chunk(c, p, room) == BDLM_OK ? room.plan_bytes : 0;
}

size_t bdlm_chunk_workspace_bytes(const bdlm_cache* c, const bdlm_chunk* p) {
  Room room;
  return check_chunk(c, p, room) == BDLM_OK ? room.part_bytes + room.lse_bytes : 0;
}

bdlm_status bdlm_chunk_plan(const bdlm_cache* c, const bdlm_chunk* p, const int32_t* seqs, const int32_t* counts,
                            void* plan, size_t plan_bytes, hipStream_t stream) {
  bdlm_status st;
  Room room;
  if ((st = check_chunk(c, p, room)) != BDLM_OK || (st = check_plan(plan, plan_bytes, room)) != BDLM_OK) return st;
  if (p->requests > 0 && (!seqs || !aligned4(seqs) || !counts || !aligned4(counts)))
    return fail(BDLM_ERR_INVALID, "sequences or counts are null or not 4-byte aligned");
  ChunkPlanArgs a{};
  a.lens = c->lens;
  a.seqs = seqs;
  a.counts = counts;
  a.plan = static_cast<int32_t*>(plan);
  a.top = c->max_pages * c->page_size;
  a.requests = (int32_t)p->requests;
  a.rows = (int32_t)p->rows;
  a.seqs_in_cache = (int32_t)c->seqs;
  a.group = p->heads / c->kv_heads;
  a.kv_heads = c->kv_heads;
  a.M = (int32_t)p->block_size;
  a.window = (int32_t)p->window;
  a.sinks = p->window > 0 ? p->sinks : 0;  // (without a window every earlier key is visible)
  a.f32 = c->dtype == BDLM_F32;
  a.limit = room.limit;
  a.least = room.least;
  a.slots = (int32_t)(a.f32 ? kSlotsF32 : kSlots);
  a.join_rows = join_rows(c->head_dim);
  a.max_items = (int32_t)room.items;
  a.max_joins = (int32_t)room.joins;
  a.max_part_rows = room.part_rows;
  a.key = room.key;
  const hipError_t e = timed(kKChunkPlan, stream, [&] { return launch_chunk_plan(a, stream); });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "chunk plan launch");
}

bdlm_status bdlm_chunk_attn(const bdlm_cache* c, const bdlm_chunk* p, int64_t layer, const void* plan, size_t plan_bytes,
                            bdlm_rows q, bdlm_rows o, float* lse, int64_t lse_pitch, int32_t fill, void* workspace,
                            size_t workspace_bytes, hipStream_t stream) {
  bdlm_status st;
  Room room;
  if ((st = check_chunk(c, p, room)) != BDLM_OK || (st = check_plan(plan, plan_bytes, room)) != BDLM_OK) return st;
  if (layer < 0 || layer >= c->layers)
    return fail(BDLM_ERR_INVALID, "layer %lld outside [0, %lld)", (long long)layer, (long long)c->layers);
  if (fill != 0 && fill != 1) return fail(BDLM_ERR_INVALID, "fill must be 0 or 1");
  if (lse_pitch < p->rows || lse_pitch > kMaxLen)
    return fail(BDLM_ERR_INVALID, "lse pitch %lld outside [%lld, 2^28]", (long long)lse_pitch, (long long)p->rows);
  if (p->rows == 0) return BDLM_OK;
  const int elem = c->dtype == BDLM_F32 ? 4 : 2;
  const int64_t width = (int64_t)p->heads * c->head_dim;
  if ((st = check_rows(q, "q", width, elem)) != BDLM_OK || (st = check_rows(o, "o", width, elem)) != BDLM_OK) return st;
  if (!lse || !aligned4(lse)) return fail(BDLM_ERR_INVALID, "lse is null or not 4-byte aligned");
  const size_t need = room.part_bytes + room.lse_bytes;
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)))
    return fail(BDLM_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu at %p)", need, workspace_bytes,
                workspace);
  const CacheArg ca = cache_arg(c);
  ChunkArgs a{};
  a.k = ca.k + layer * ca.layer_bytes;
  a.v = ca.v + layer * ca.layer_bytes;
  a.table = ca.table;
  a.q = q.ptr;
  a.qs = q.stride;
  a.o = o.ptr;
  a.os = o.stride;
  a.lse = lse;
  a.pitch = lse_pitch;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = need ? static_cast<char*>(workspace) + room.part_bytes : nullptr;
  a.plan = static_cast<const int32_t*>(plan);
  a.items = reinterpret_cast<const ChunkItemRec*>(a.plan + kChunkHead + 2 * p->requests + 1);
  a.joins = reinterpret_cast<const ChunkJoin*>(a.items + room.items);
  a.part_rows = room.part_rows;
  a.pages = ca.pages;
  a.page_size = ca.page_size;
  a.max_pages = ca.max_pages;
  if (ca.page_size > 1) {
    while (((int64_t)2 << a.page_shift) < ca.page_size) ++a.page_shift;
    a.page_mul = (uint32_t)(((uint64_t)1 << (32 + a.page_shift)) / (uint64_t)ca.page_size + 1);
  }
  a.heads = p->heads;
  a.kv_heads = c->kv_heads;
  a.group = p->heads / c->kv_heads;
  a.M = (int32_t)p->block_size;
  a.window = (int32_t)p->window;
  a.sinks = p->window > 0 ? p->sinks : 0;
  a.rows = (int32_t)p->rows;
  a.fill = fill;
  a.max_items = (int32_t)room.items;
  a.max_joins = (int32_t)room.joins;
  a.key = room.key;
  a.scale = p->scale > 0.f ? p->scale : 1.0f / std::sqrt((float)c->head_dim);
  a.scale_log2 = a.scale * 1.44269504088896340736f;
  const int bf16 = c->dtype == BDLM_BF16;
  hipError_t e = timed(kKChunkAttn, stream, [&] {
    return bf16 ? launch_chunk_bf16(a, c->head_dim, stream) : launch_chunk_f32(a, c->head_dim, stream);
  });
  if (e == hipSuccess && room.joins > 0)
    e = timed(kKChunkMerge, stream, [&] { return launch_chunk_merge(a, c->head_dim, bf16, stream); });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "attention of chunks over the cache");
}

}  // extern "C"
