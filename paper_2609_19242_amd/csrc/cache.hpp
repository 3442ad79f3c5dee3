// The paged cache as the kernels see it: attention of decoding requests over
// it (prefix_*.hip) and the operations on its pages (cache_pages.hip).
#pragma once

#include "common.hpp"

namespace bdlm {

struct CacheArg {
  char *k, *v;     // [layers][pages][page_size][kv_heads][head_dim]
  int32_t* table;  // [seqs][max_pages] page numbers, -1 behind a sequence's last page
  int32_t* lens;   // [seqs] tokens
  int32_t* refs;   // [pages] tables that hold the page, 0: free
  int32_t* status; // [2] outcome of the last page operation, pages it lacked
  int64_t page_bytes, layer_bytes;  // of K (and V)
  int32_t layers, pages, page_size, seqs, max_pages;
  int32_t row_bytes;  // kv_heads * head_dim elements
};

// ---- page operations (cache_pages.hip)
struct CacheList {
  int32_t n;
  const int32_t *a, *b;  // fork: parents, children; grow: sequences, counts; free: sequences
};
struct CacheRows {
  int32_t n, rows;        // sequences, rows of the new tensors
  const int32_t *seqs, *counts, *starts;
  const char *k, *v;
  int64_t k_stride, v_stride;  // bytes between rows
  int64_t layer;
};
// Words of the page operations' workspace (bdlm_cache_work_bytes): a header, then
//   grow: the new pages (at most `pages`);
//   fork: each child's page for its last rows (n <= seqs), then the new pages (at most `pages`);
//   compact: the free pages to fill, the pages that move there, and each page's new number (`pages` words each).
constexpr int kCacheHead = 16;
hipError_t launch_cache_grow(const CacheArg& c, const CacheList& l, int32_t* work, hipStream_t s);
hipError_t launch_cache_fork(const CacheArg& c, const CacheList& l, int32_t* work, hipStream_t s);
hipError_t launch_cache_free(const CacheArg& c, const CacheList& l, hipStream_t s);
hipError_t launch_cache_compact(const CacheArg& c, int32_t* work, hipStream_t s);
hipError_t launch_cache_write(const CacheArg& c, const CacheRows& r, hipStream_t s);

// ---- attention of decoding requests (prefix_bf16.hip, prefix_f32.hip, prefix_merge.hip)
//
// Rows.  The query rows of a KV head are numbered token * group + g over the
// tokens [request][row] and the query heads of its group.  They meet the
// prefix's keys [0, prefix) all together, and their own request's keys
// [prefix, len) by request; keys are cut into chunks, and every (chunk, row)
// leaves a normalised partial output (fp32) and its log2-sum-exp (fp32 in bf16
// calls, fp64 in fp32 ones: partials.hpp) in `part_o`, `part_lse`
// ([chunk][token][head]), which prefix_merge adds up.  With one chunk in all,
// the kernels write O and LSE themselves.
template <bool BF16> struct PartLseOf { typedef float type; };
template <> struct PartLseOf<false> { typedef double type; };
template <bool BF16> using PartLse = typename PartLseOf<BF16>::type;
struct PrefixArgs {
  const char *k, *v;  // this layer's
  const int32_t *table, *lens, *seqs;
  const void* q;
  void* o;
  float *lse, *part_o;
  void* part_lse;
  int32_t pages, page_size, seqs_in_cache, max_pages;
  int32_t requests, rows, heads, kv_heads, group;
  int32_t prefix, block;      // block: every row sees all len keys
  float scale, scale_log2;    // (scale: for the fp32 kernels, which multiply by log2(e) in 64 bits)
  int32_t prefix_chunks, prefix_chunk;  // chunks of the prefix, keys per chunk
  int32_t own_chunks, own_min;          // chunks of a request's own keys at most, keys per chunk at least
  int32_t prefix_tiles, own_tiles;      // tiles of query rows
  int32_t prefix_items, own_items;
  int32_t prefix_shared, own_shared;    // bf16: tiles of rows share a chunk's keys (else waves share out its keys)
};
constexpr int kPrefixTableEntries = 2048;  // pages of a chunk at most
constexpr int kPrefixGroups = 1024;        // bf16, pages of whole groups of 16 tokens: groups of a chunk at most
constexpr int kShortJoin = 16;             // parts whose outputs are joined the short way (kFewParts)
constexpr int kPrefixSharedRows = 128, kPrefixWaveRows = 32, kPrefixRowsF32 = 16;

hipError_t launch_prefix_bf16(const PrefixArgs& a, int head_dim, hipStream_t s);
hipError_t launch_prefix_f32(const PrefixArgs& a, int head_dim, hipStream_t s);
hipError_t launch_prefix_merge(const PrefixArgs& a, int head_dim, int bf16, hipStream_t s);

// A work item of the attention kernels: query rows [row0, row0 + nrows) of a
// KV head against the keys [k0, k1) in the pages of one sequence.
struct PrefixItem {
  int kvh, row0, nrows, part;
  int seq;      // -1: no such sequence
  int k0, k1;
  bool shared;
};

__device__ inline int cache_len(const PrefixArgs& a, int seq) {
  if ((unsigned)seq >= (unsigned)a.seqs_in_cache) return 0;
  const int64_t top = (int64_t)a.max_pages * a.page_size;
  const int n = a.lens[seq];
  return n < 0 ? 0 : (int64_t)n > top ? (int)top : n;
}

// Item `wg`: the prefix's items first, [chunk][tile of rows][KV head], then the
// requests' own, [chunk][request][tile][KV head]: workgroups that run together
// read the same keys, and with 8 KV heads each XCD serves one.
__device__ inline bool prefix_item(const PrefixArgs& a, int wg, int tile_rows_prefix, int tile_rows_own,
                                   PrefixItem& it) {
  if (wg >= a.prefix_items + a.own_items) return false;
  const int per = a.rows * a.group;  // rows of a request
  if (wg < a.prefix_items) {
    it.kvh = wg % a.kv_heads;
    int rest = wg / a.kv_heads;
    const int tile = rest % a.prefix_tiles;
    it.part = rest / a.prefix_tiles;
    it.row0 = tile * tile_rows_prefix;
    it.nrows = imin(tile_rows_prefix, a.requests * per - it.row0);
    it.seq = a.seqs[0];
    it.k0 = it.part * a.prefix_chunk;
    it.k1 = imin(it.k0 + a.prefix_chunk, a.prefix);
    it.shared = a.prefix_shared;
  } else {
    wg -= a.prefix_items;
    it.kvh = wg % a.kv_heads;
    int rest = wg / a.kv_heads;
    const int tile = rest % a.own_tiles;
    rest /= a.own_tiles;
    const int r = rest % a.requests, c = rest / a.requests;
    it.part = a.prefix_chunks + c;
    it.row0 = r * per + tile * tile_rows_own;
    it.nrows = imin(tile_rows_own, per - tile * tile_rows_own);
    it.seq = a.seqs[r];
    const int n = imax(cache_len(a, it.seq) - a.prefix, 0);
    // this request's chunks: as few as own_min allows, of a multiple of 64 keys
    const int chunks = imin(imax((n + a.own_min - 1) / a.own_min, 1), a.own_chunks);
    const int size = (n / chunks / 64 + 1) * 64;  // (chunks * size >= n)
    it.k0 = a.prefix + imin(c * size, n);
    it.k1 = a.prefix + imin((c + 1) * size, n);
    it.shared = a.own_shared;
  }
  if ((unsigned)it.seq >= (unsigned)a.seqs_in_cache) it.k1 = it.k0, it.seq = -1;
  return true;
}

// A query row: its element in Q and O is (token * heads + head) * D; it sees the keys below `end`.
struct PrefixRow {
  int token, head, end;
};
__device__ inline PrefixRow prefix_row(const PrefixArgs& a, int kvh, int row) {
  PrefixRow x;
  x.token = row / a.group;
  x.head = kvh * a.group + (row - x.token * a.group);
  const int r = x.token / a.rows, i = x.token - r * a.rows;
  const int n = cache_len(a, a.seqs[r]);
  x.end = a.block ? n : imax(n - a.rows + i + 1, 0);
  return x;
}
// Where the row's LSE goes: [request][heads][rows].
__device__ inline int64_t prefix_lse_at(const PrefixArgs& a, const PrefixRow& x) {
  const int r = x.token / a.rows;
  return ((int64_t)r * a.heads + x.head) * a.rows + (x.token - r * a.rows);
}

}  // namespace bdlm
