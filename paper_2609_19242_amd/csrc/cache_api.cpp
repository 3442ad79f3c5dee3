// C ABI of the paged cache: argument validation, how attention over it is cut
// up, launches.  Declarations and contracts: include/bdlm_attn.h.
#include "bdlm_attn.h"

#include <algorithm>
#include <cmath>

#include "api_util.hpp"
#include "cache.hpp"
#include "split_plan.hpp"

using namespace bdlm;

namespace {

constexpr int64_t kMaxSeqs = (int64_t)1 << 19;  // a bit each in the bookkeeping's LDS
constexpr int64_t kMaxPages = ((int64_t)1 << 30) - 1;
constexpr int64_t kMaxRows = (int64_t)1 << 25;  // query rows x heads of one attention call (a grid dimension of the merge)
constexpr int64_t kMaxWgs = (int64_t)1 << 22;
constexpr int kMaxKeyChunks = 1 << 20;  // chunks of keys of one attention call

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

bdlm_status check_cache(const bdlm_cache* c) {
  if (!c) return fail(BDLM_ERR_INVALID, "cache is null");
  if (c->reserved != 0) return fail(BDLM_ERR_INVALID, "reserved field must be 0");
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(BDLM_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", c->head_dim);
  if (c->dtype != BDLM_BF16 && c->dtype != BDLM_F32) return fail(BDLM_ERR_UNSUPPORTED, "dtype %d not supported", c->dtype);
  if (c->kv_heads < 1 || c->kv_heads > 4096) return fail(BDLM_ERR_INVALID, "kv_heads %d outside [1, 4096]", c->kv_heads);
  if (c->layers < 1 || c->layers > 65536) return fail(BDLM_ERR_INVALID, "layers %lld outside [1, 65536]", (long long)c->layers);
  if (c->pages < 1 || c->pages > kMaxPages)
    return fail(BDLM_ERR_INVALID, "pages %lld outside [1, 2^30)", (long long)c->pages);
  if (c->page_size < 1 || c->page_size > ((int64_t)1 << 20))
    return fail(BDLM_ERR_INVALID, "page_size %lld outside [1, 2^20]", (long long)c->page_size);
  if (c->seqs < 1 || c->seqs > kMaxSeqs) return fail(BDLM_ERR_INVALID, "seqs %lld outside [1, 2^19]", (long long)c->seqs);
  if (c->max_pages < 1 || c->max_pages * c->page_size >= kMaxPos || c->max_pages >= kMaxPos)
    return fail(BDLM_ERR_INVALID, "max_pages %lld: a table must hold between one page and 2^30 tokens",
                (long long)c->max_pages);
  if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v))
    return fail(BDLM_ERR_INVALID, "cache k or v is null or not 16-byte aligned");
  const void* ints[] = {c->table, c->lens, c->refs, c->status, c->work};
  for (const void* p : ints)
    if (!p || !aligned4(p)) return fail(BDLM_ERR_INVALID, "a cache table is null or not 4-byte aligned");
  return BDLM_OK;
}

CacheArg cache_arg(const bdlm_cache* c) {
  CacheArg a{};
  a.k = static_cast<char*>(c->k);
  a.v = static_cast<char*>(c->v);
  a.table = c->table;
  a.lens = c->lens;
  a.refs = c->refs;
  a.status = c->status;
  a.layers = (int32_t)c->layers;
  a.pages = (int32_t)c->pages;
  a.page_size = (int32_t)c->page_size;
  a.seqs = (int32_t)c->seqs;
  a.max_pages = (int32_t)c->max_pages;
  a.row_bytes = c->kv_heads * c->head_dim * (c->dtype == BDLM_F32 ? 4 : 2);
  a.page_bytes = (int64_t)a.row_bytes * c->page_size;
  a.layer_bytes = a.page_bytes * c->pages;
  return a;
}

bdlm_status check_list(const bdlm_cache* c, int64_t n, const int32_t* a, const char* what) {
  if (n < 0 || n > c->seqs)
    return fail(BDLM_ERR_INVALID, "%lld %s for a cache of %lld sequences", (long long)n, what, (long long)c->seqs);
  if (n > 0 && (!a || !aligned4(a))) return fail(BDLM_ERR_INVALID, "%s are null or not 4-byte aligned", what);
  return BDLM_OK;
}

bdlm_status done(hipError_t e, const char* what) { return e == hipSuccess ? BDLM_OK : hip_fail(e, what); }

// How the keys of an attention call are cut into chunks and its rows into tiles.
//
// Chunks trade balance against partial sums, whose cost grows with the query rows
// (all heads of all requests), so few rows take shorter chunks.  Times below with
// keys that no cache holds yet, 32 heads on 8 KV heads, where not said otherwise.
//
// The prefix: long enough that its tiles of rows give one item to every workgroup
// slot that the requests' own items leave (items that tables of fewer than 512 keys
// beside the prefix hold count for less), half of them at least (16 requests, 16,000
// tokens: one for every slot 40 us, so 35; 40 requests 44, 41; 16,384 rows, 16K
// tokens, 4 KV heads: 4,096 keys, one item per slot, 173 us, 2,048 185, 8,192 197);
// and so few chunks, up to 1,024 keys each, that their sums take the short way
// (kShortJoin) where that leaves half the slots an item (24 requests, 16/16 heads,
// 16,000 tokens: 512 keys 43 us, 1,024 38).
// Below that, half a key per query row up to 1,024 keys, but no more than leave
// kFewItems items, and a 24th of the prefix within [256, 512] at least (one request,
// 16,000 tokens: chunks of 256 keys 25 us, 512 23, 1,024 29; 16 requests, 12/2 heads,
// 2,000 tokens: 256 16.5 us, 512 20; 64 requests, 4,000 tokens: 512 27 us, 1,024 33;
// 8,192 tokens and up to 1,500 of their own: 1,024 54.5, 512 59).
//
// A request's own keys: as many keys per query row, at least kOwnPerBase per
// (KV head, request, tile), within [512, 1024] (one request of 32,000 keys: chunks of
// 256 43 us, 512 35, 768 39; 8 of 300 to 6,000: 33, 28, 30; 16 of 100 to 2,000 take
// 384 sooner, 22 us, than 512, 24; 16 of 32 rows and up to 2,000 keys, 32/4 heads:
// 1,024 39 us, 1,536 47; 64 of 4,000 keys: 196, 193), their number limited by the
// workgroups that find nothing to do where a sequence is shorter than its table
// (kMaxOwnItems).  Tables of up to kOwnWhole keys: one chunk, which needs no sums.
//
// A prefix that would save less than kFoldBytes of reading is not kept apart:
// the requests' own keys then start at 0, and short ones need no partial sums.
// Nor is one whose requests fill tiles of rows by themselves, since each tile
// reads the prefix anyway, if it is at least half of what a table holds and the
// tiles leave slots free: every sequence is cut into the same number of equal
// chunks, so that no short item of a request's own keys runs after the prefix's
// long ones.  Their number: the least of rounds of items times keys per chunk plus
// the partial sums (at 128 rows and head_dim 128, three quarters of a key's time
// per item).  4 requests of 64 rows behind 16K tokens, with up to 4,000 more: 111 ->
// 101 us; 20 of 32 rows behind 9,000 with 2,000: 145 -> 135; 10 of 24 (40/8 heads)
// behind 5,000 with 1,000: 51 -> 51.
constexpr int64_t kSlots = 2 * kCus, kFewItems = 128, kOwnPerBase = 3, kOwnWhole = 512, kMaxOwnItems = 4096;
constexpr int64_t kFoldBytes = 8 << 20;

bdlm_status plan_prefix(const bdlm_cache* c, int64_t requests, int64_t rows, int32_t heads, int64_t prefix,
                        PrefixArgs& a, size_t& part_bytes) {
  const bool f32 = c->dtype == BDLM_F32;
  const int64_t group = heads / c->kv_heads, per = rows * group, all = requests * per;
  const int64_t row_bytes = (int64_t)2 * c->kv_heads * c->head_dim * (f32 ? 4 : 2);
  const int64_t common = prefix;
  if ((requests - 1) * prefix * row_bytes <= kFoldBytes) prefix = 0;
  a.prefix_shared = !f32 && all > 2 * kPrefixWaveRows;
  a.own_shared = !f32 && per > 2 * kPrefixWaveRows;
  auto tile = [&](bool shared) { return f32 ? kPrefixRowsF32 : shared ? kPrefixSharedRows : kPrefixWaveRows; };
  const int64_t pt = (all + tile(a.prefix_shared) - 1) / tile(a.prefix_shared);
  const int64_t ot = (per + tile(a.own_shared) - 1) / tile(a.own_shared);
  const int64_t base = c->kv_heads * requests * ot;
  const bool full = a.own_shared && requests * ot * 8 <= pt * 9 && base <= kSlots &&
                    2 * common >= c->max_pages * c->page_size;
  if (full) prefix = 0;
  a.prefix = (int32_t)prefix;
  const int64_t own = c->max_pages * c->page_size - prefix;
  // keys whose pages (or groups) a workgroup can hold, with a chunk that starts inside one
  const int64_t limit = !f32 && c->page_size % 16 == 0 ? (kPrefixGroups - 2) * 16 : (kPrefixTableEntries - 2) * c->page_size;
  auto up64 = [](int64_t x) { return (x + 63) / 64 * 64; };
  auto within = [](int64_t x, int64_t lo, int64_t hi) { return std::min(std::max(x, lo), hi); };
  const int64_t row_min = requests * rows * heads / 2;
  const int64_t low = within(prefix / 24, 256, 512);
  const int64_t want = std::min(within(row_min, low, 1024), std::max(low, c->kv_heads * pt * prefix / kFewItems));
  const int64_t slots = std::max(kSlots - base * std::min<int64_t>(own, 512) / 512, kSlots / 2);
  const int64_t joins = c->kv_heads * pt * kShortJoin >= kSlots / 2 ? std::min<int64_t>(prefix / (kShortJoin - 2), 1024) : 0;
  const int64_t pc = std::min(up64(std::max({want, c->kv_heads * pt * prefix / slots, joins})),
                              std::min(limit, up64(prefix + 1)));
  a.prefix_chunk = (int32_t)pc;
  a.prefix_chunks = (int32_t)((prefix + pc - 1) / pc);
  int64_t own_min = own <= kOwnWhole ? kOwnWhole : within(std::max(kOwnPerBase * base, row_min), 512, 1024);
  int64_t whole = 0;  // chunks of every request where whole sequences are cut up
  if (full) {
    int64_t best = INT64_MAX;
    for (int64_t n = 1; n <= 2 * kSlots / base && (n == 1 || own / n >= 512); ++n) {
      const int64_t cost = (base * n + kSlots - 1) / kSlots * own / n + n * base * 3 / 4;
      if (own / n <= limit - 128 && cost < best) best = cost, whole = n;
    }
    if (whole > 0) own_min = 512;
  }
  int64_t oc = std::min((own + own_min - 1) / own_min, std::max<int64_t>(kMaxOwnItems / base, 1));
  if (whole > 0) oc = whole;
  oc = std::max(oc, (own + limit - 65) / (limit - 64));
  if (oc == 0 && a.prefix_chunks == 0) oc = 1;
  a.own_chunks = (int32_t)oc;
  a.own_min = (int32_t)std::min(own_min, limit - 64);
  a.prefix_tiles = (int32_t)pt;
  a.own_tiles = (int32_t)ot;
  const int64_t parts = a.prefix_chunks + oc, pi = c->kv_heads * pt * a.prefix_chunks, oi = base * oc;
  if (pi + oi > kMaxWgs || parts > kMaxKeyChunks)
    return fail(BDLM_ERR_UNSUPPORTED, "attention over the cache needs %lld workgroups and %lld chunks (limits 2^22, %d)",
                (long long)(pi + oi), (long long)parts, kMaxKeyChunks);
  a.prefix_items = (int32_t)pi;
  a.own_items = (int32_t)oi;
  part_bytes = parts == 1 ? 0 : (size_t)parts * requests * rows * heads * c->head_dim * sizeof(float);
  return BDLM_OK;
}

// Workspace: the partial outputs (`part` bytes), behind them their log2-sum-exp.
size_t prefix_workspace(const bdlm_cache* c, size_t part) {
  const size_t per = c->dtype == BDLM_F32 ? sizeof(PartLse<false>) : sizeof(PartLse<true>);
  return part ? align256(part) + align256(part / (c->head_dim * sizeof(float)) * per) : 0;
}

bdlm_status check_prefix(const bdlm_cache* c, int64_t requests, int64_t rows, int32_t heads, int64_t prefix) {
  if (heads < 1 || heads % c->kv_heads != 0)
    return fail(BDLM_ERR_INVALID, "heads (%d) must be a positive multiple of kv_heads (%d)", heads, c->kv_heads);
  if (requests < 0 || rows < 0) return fail(BDLM_ERR_INVALID, "requests %lld x rows %lld", (long long)requests, (long long)rows);
  if (requests > kMaxRows || rows > kMaxRows || (requests > 0 && rows > 0 && requests * rows > kMaxRows / heads))
    return fail(BDLM_ERR_UNSUPPORTED, "requests %lld x rows %lld x heads %d exceeds 2^25", (long long)requests,
                (long long)rows, heads);
  if (prefix < 0 || prefix > c->max_pages * c->page_size)
    return fail(BDLM_ERR_INVALID, "prefix %lld outside [0, %lld], what a table holds", (long long)prefix,
                (long long)(c->max_pages * c->page_size));
  return BDLM_OK;
}

}  // namespace

extern "C" {

size_t bdlm_cache_work_bytes(int64_t pages, int64_t seqs) {
  if (pages < 1 || pages > kMaxPages || seqs < 1 || seqs > kMaxSeqs) return 0;
  return (size_t)(kCacheHead + std::max(3 * pages, pages + seqs)) * sizeof(int32_t);
}

bdlm_status bdlm_cache_grow(const bdlm_cache* c, int64_t n, const int32_t* seqs, const int32_t* counts,
                            hipStream_t stream) {
  bdlm_status st;
  if ((st = check_cache(c)) != BDLM_OK || (st = check_list(c, n, seqs, "sequences")) != BDLM_OK ||
      (st = check_list(c, n, counts, "counts")) != BDLM_OK)
    return st;
  return done(timed(kKCachePages, stream,
                    [&] { return launch_cache_grow(cache_arg(c), CacheList{(int32_t)n, seqs, counts}, c->work, stream); }),
              "cache grow launch");
}

bdlm_status bdlm_cache_fork(const bdlm_cache* c, int64_t n, const int32_t* parents, const int32_t* children,
                            hipStream_t stream) {
  bdlm_status st;
  if ((st = check_cache(c)) != BDLM_OK || (st = check_list(c, n, parents, "parents")) != BDLM_OK ||
      (st = check_list(c, n, children, "children")) != BDLM_OK)
    return st;
  return done(timed(kKCachePages, stream,
                    [&] {
                      return launch_cache_fork(cache_arg(c), CacheList{(int32_t)n, parents, children}, c->work, stream);
                    }),
              "cache fork launch");
}

bdlm_status bdlm_cache_free(const bdlm_cache* c, int64_t n, const int32_t* seqs, hipStream_t stream) {
  bdlm_status st;
  if ((st = check_cache(c)) != BDLM_OK || (st = check_list(c, n, seqs, "sequences")) != BDLM_OK) return st;
  return done(timed(kKCachePages, stream,
                    [&] { return launch_cache_free(cache_arg(c), CacheList{(int32_t)n, seqs, nullptr}, stream); }),
              "cache free launch");
}

bdlm_status bdlm_cache_compact(const bdlm_cache* c, hipStream_t stream) {
  const bdlm_status st = check_cache(c);
  if (st != BDLM_OK) return st;
  return done(timed(kKCachePages, stream, [&] { return launch_cache_compact(cache_arg(c), c->work, stream); }),
              "cache compact launch");
}

bdlm_status bdlm_cache_write(const bdlm_cache* c, int64_t layer, int64_t n, const int32_t* seqs, const int32_t* counts,
                             const int32_t* starts, int64_t rows, bdlm_rows k, bdlm_rows v, hipStream_t stream) {
  bdlm_status st;
  if ((st = check_cache(c)) != BDLM_OK || (st = check_list(c, n, seqs, "sequences")) != BDLM_OK ||
      (st = check_list(c, n, counts, "counts")) != BDLM_OK)
    return st;
  if (layer < 0 || layer >= c->layers)
    return fail(BDLM_ERR_INVALID, "layer %lld outside [0, %lld)", (long long)layer, (long long)c->layers);
  if (rows < 0 || rows >= kMaxPos) return fail(BDLM_ERR_INVALID, "rows %lld outside [0, 2^30)", (long long)rows);
  if (starts && !aligned4(starts)) return fail(BDLM_ERR_INVALID, "starts are not 4-byte aligned");
  if (!starts && n > 0 && rows % n != 0)
    return fail(BDLM_ERR_INVALID, "%lld rows for %lld sequences: without starts each has the same number",
                (long long)rows, (long long)n);
  const int elem = c->dtype == BDLM_F32 ? 4 : 2;
  const int64_t width = (int64_t)c->kv_heads * c->head_dim;
  const bdlm_rows t[2] = {k, v};
  for (int i = 0; i < 2 && rows > 0 && n > 0; ++i) {
    if (!t[i].ptr || !aligned16(t[i].ptr))
      return fail(BDLM_ERR_INVALID, "new %s is null or not 16-byte aligned", i ? "v" : "k");
    if (t[i].stride < width || t[i].stride > ((int64_t)1 << 30) || t[i].stride * elem % 16 != 0)
      return fail(BDLM_ERR_INVALID, "new %s: row stride %lld below %lld or not a multiple of 16 bytes", i ? "v" : "k",
                  (long long)t[i].stride, (long long)width);
  }
  CacheRows r{};
  r.n = (int32_t)n;
  r.rows = (int32_t)rows;
  r.seqs = seqs;
  r.counts = counts;
  r.starts = starts;
  r.k = static_cast<const char*>(k.ptr);
  r.v = static_cast<const char*>(v.ptr);
  r.k_stride = k.stride * elem;
  r.v_stride = v.stride * elem;
  r.layer = layer;
  return done(timed(kKCacheWrite, stream, [&] { return launch_cache_write(cache_arg(c), r, stream); }),
              "cache write launch");
}

size_t bdlm_prefix_attn_workspace_bytes(const bdlm_cache* c, int64_t requests, int64_t rows, int32_t heads,
                                        int64_t prefix) {
  PrefixArgs a{};
  size_t part = 0;
  if (check_cache(c) != BDLM_OK || check_prefix(c, requests, rows, heads, prefix) != BDLM_OK) return 0;
  if (requests == 0 || rows == 0 || plan_prefix(c, requests, rows, heads, prefix, a, part) != BDLM_OK) return 0;
  return prefix_workspace(c, part);
}

bdlm_status bdlm_prefix_attn(const bdlm_cache* c, int64_t layer, int64_t requests, const int32_t* seqs, int64_t rows,
                             int32_t heads, int64_t prefix, int32_t block, float scale, const void* q, void* o,
                             float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  bdlm_status st;
  if ((st = check_cache(c)) != BDLM_OK || (st = check_prefix(c, requests, rows, heads, prefix)) != BDLM_OK) return st;
  if (layer < 0 || layer >= c->layers)
    return fail(BDLM_ERR_INVALID, "layer %lld outside [0, %lld)", (long long)layer, (long long)c->layers);
  if (block != 0 && block != 1) return fail(BDLM_ERR_INVALID, "block must be 0 or 1");
  if (!std::isfinite(scale)) return fail(BDLM_ERR_INVALID, "scale is not finite");
  if (requests == 0 || rows == 0) return BDLM_OK;
  if (!seqs || !aligned4(seqs)) return fail(BDLM_ERR_INVALID, "sequences are null or not 4-byte aligned");
  if (!q || !o || !lse || !aligned16(q) || !aligned16(o))
    return fail(BDLM_ERR_INVALID, "q, o or lse is null or not 16-byte aligned");
  PrefixArgs a{};
  size_t part = 0;
  if ((st = plan_prefix(c, requests, rows, heads, prefix, a, part)) != BDLM_OK) return st;
  const size_t need = prefix_workspace(c, part);
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)))
    return fail(BDLM_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu at %p)", need,
                workspace_bytes, workspace);
  const CacheArg ca = cache_arg(c);
  a.k = ca.k + layer * ca.layer_bytes;
  a.v = ca.v + layer * ca.layer_bytes;
  a.table = ca.table;
  a.lens = ca.lens;
  a.seqs = seqs;
  a.q = q;
  a.o = o;
  a.lse = lse;
  a.part_o = static_cast<float*>(workspace);
  a.part_lse = need ? static_cast<char*>(workspace) + align256(part) : nullptr;
  a.pages = ca.pages;
  a.page_size = ca.page_size;
  a.seqs_in_cache = ca.seqs;
  a.max_pages = ca.max_pages;
  a.requests = (int32_t)requests;
  a.rows = (int32_t)rows;
  a.heads = heads;
  a.kv_heads = c->kv_heads;
  a.group = heads / c->kv_heads;
  a.block = block;
  a.scale = scale > 0.f ? scale : 1.0f / std::sqrt((float)c->head_dim);
  a.scale_log2 = a.scale * 1.44269504088896340736f;
  const int bf16 = c->dtype == BDLM_BF16;
  hipError_t e = timed(kKPrefixAttn, stream, [&] {
    return bf16 ? launch_prefix_bf16(a, c->head_dim, stream) : launch_prefix_f32(a, c->head_dim, stream);
  });
  if (e == hipSuccess && need > 0)
    e = timed(kKPrefixMerge, stream, [&] { return launch_prefix_merge(a, c->head_dim, bf16, stream); });
  return done(e, "attention over the cache");
}

}  // extern "C"
