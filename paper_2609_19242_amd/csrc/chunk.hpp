// Attention of chunks of new tokens over a paged cache: requests with different
// numbers of rows (one for a decoding request, hundreds for a piece of a prompt),
// causal by blocks of M tokens, optionally within a window of which the first S
// tokens stay visible; the rules of packed calls over pages.
//
// A small kernel (chunk_plan.hip) lays out the work of a step on the device, where
// the lengths are, once for all layers; the tile kernels of prefix_bf16.hip and
// prefix_f32.hip run its items (ChunkArgs in place of PrefixArgs), and
// chunk_merge.hip joins the outputs of tiles whose keys were cut into chunks.
//
// Rows.  The query rows of a request and a KV head are numbered row * group + g over
// its new tokens and the query heads of the group, in tiles of 128 (requests of more
// than 64 of them), 32, or in fp32 16.
//
// Keys.  A tile's rows see the keys [0, S) and [w0, end) of their sequence, w0 the first row's
// window's start, end the last row's end.  They are walked as [0, n) with the gap
// between taken out: v < gap_at is key v, the others are key v + gap.  gap_at and gap
// are multiples of 16, so that groups of 16 keys stay together; keys that no row of
// the tile sees (at most 15 before w0, and behind S) read as zeros.
#pragma once

#include "cache.hpp"

namespace bdlm {

// Words of a plan in device memory: a header, the requests' first rows, their first
// tiles (with the total behind), the items, the merge's units.
constexpr int kChunkHead = 16;
enum : int { kPlanItems = 0, kPlanJoins = 1, kPlanRows = 2, kPlanRoom = 3, kPlanKey = 4 };  // of the header (room: for items, in front of the units; key: 8 bytes)

struct ChunkItemRec {
  int32_t seq, token0, pos0, len;  // (-1: none) the request's first row, its position, the sequence's tokens
  int32_t row0, nrows;             // rows of the tile, within the request's
  int32_t k0, k1;                  // of the walk
  int32_t gap_at, gap, w0;         // (w0: in the walk)
  int32_t part;                    // first row of its partial outputs, -1: it writes the outputs; bit 30: a tile of 128
};
constexpr int32_t kSharedTile = 1 << 30;
constexpr int kChunkGroups = kPrefixTableEntries;  // bf16, pages of whole groups of 16 tokens: groups of a chunk at most
constexpr int kFillWgs = 32;  // workgroups beside the items', for rows of no request
// Rows of a cut tile whose parts a workgroup of the merge joins: `nrows` rows from
// row0 on, their first parts from partial row `part` on, n parts `step` rows apart.
struct ChunkJoin {
  int32_t token0, row0, nrows, part, n, step, pad0, pad1;
};
constexpr int join_rows(int head_dim) { return 1024 / head_dim; }  // of a unit; one where there are many parts

struct ChunkPlanArgs {
  const int32_t *lens, *seqs, *counts;
  int32_t* plan;
  int64_t top;  // tokens that a table holds
  int32_t requests, rows, seqs_in_cache, group, kv_heads, M, window, sinks;
  int32_t f32, limit, least, slots;   // keys of a chunk at most, at least; workgroups that run at once
  int32_t join_rows, max_items, max_joins;
  int64_t max_part_rows;
  uint64_t key;
};

// The header of a plan of (longer items << 32 | others) items, (units << 32 | partial rows) and the requests' rows.  Where
// not all of them were written, for want of room, it is a plan of nothing that fits no call.
__host__ __device__ inline void put_chunk_head(const ChunkPlanArgs& a, int64_t items, int64_t parts, int64_t rows, bool written) {
  a.plan[kPlanItems] = written ? (int32_t)((items >> 32) + (items & 0xffffffff)) : 0;
  a.plan[kPlanJoins] = written ? (int32_t)(parts >> 32) : 0;
  a.plan[kPlanRows] = (int32_t)(rows < a.rows ? rows : a.rows);
  a.plan[kPlanRoom] = a.max_items;
  *(uint64_t*)(a.plan + kPlanKey) = written ? a.key : 0;  // (no call's key is 0)
}

struct ChunkArgs {
  const char *k, *v;  // this layer's
  const int32_t* table;
  const void* q;
  void* o;
  float *lse, *part_o;
  void* part_lse;
  const int32_t* plan;
  const ChunkItemRec* items;
  const ChunkJoin* joins;
  int64_t qs, os, pitch;  // elements between rows; rows of the LSE
  int64_t part_rows;      // partial rows of a KV head
  int32_t pages, page_size, max_pages;
  uint32_t page_mul;      // for page_of
  int32_t page_shift;
  int32_t heads, kv_heads, group, M, window, sinks;
  int32_t rows, fill;     // rows behind the last request's become 0 (LSE -inf)
  int32_t max_items, max_joins;
  float scale, scale_log2;
  uint64_t key;  // the plan's must be the same
};

hipError_t launch_chunk_plan(const ChunkPlanArgs& a, hipStream_t s);
hipError_t launch_chunk_bf16(const ChunkArgs& a, int head_dim, hipStream_t s);
hipError_t launch_chunk_f32(const ChunkArgs& a, int head_dim, hipStream_t s);
hipError_t launch_chunk_merge(const ChunkArgs& a, int head_dim, int bf16, hipStream_t s);

// ---- what the tile kernels ask of a call
struct ChunkItem : PrefixItem {
  int token0, pos0, len, gap_at, gap, w0;
};
template <class A> struct ItemOf { typedef PrefixItem type; };
template <> struct ItemOf<ChunkArgs> { typedef ChunkItem type; };
template <class A> struct GroupOf { typedef int64_t type; };
template <> struct GroupOf<ChunkArgs> { typedef int32_t type; };
template <class A> constexpr bool kIsChunk = false;
template <> constexpr inline bool kIsChunk<ChunkArgs> = true;

// Whether the plan is one of this call's sizes: those that its layout, its items' places and its keys come
// from (a number that the host forms from them lies in both).  Another one's items could lead anywhere.
__device__ inline bool plan_fits(const ChunkArgs& a) { return *(const uint64_t*)(a.plan + kPlanKey) == a.key; }
__device__ inline int plan_items(const ChunkArgs& a) { return plan_fits(a) ? imin(a.plan[kPlanItems], a.max_items) : 0; }
__device__ inline int plan_joins(const ChunkArgs& a) { return plan_fits(a) ? imin(a.plan[kPlanJoins], a.max_joins) : 0; }

template <bool BF16>
__device__ inline bool attn_item(const PrefixArgs& a, int wg, PrefixItem& it) {
  if constexpr (!BF16) return prefix_item(a, wg, kPrefixRowsF32, kPrefixRowsF32, it);
  return prefix_item(a, wg, a.prefix_shared ? kPrefixSharedRows : kPrefixWaveRows,
                     a.own_shared ? kPrefixSharedRows : kPrefixWaveRows, it);
}
// Items by number, the KV heads of one together (with 8 of them each XCD serves one).
template <bool BF16>
__device__ inline bool attn_item(const ChunkArgs& a, int wg, ChunkItem& it) {
  const int n = wg / a.kv_heads;
  if (n >= plan_items(a)) return false;
  const ChunkItemRec& r = a.items[n];
  it.kvh = wg - n * a.kv_heads;
  it.row0 = r.row0;
  it.nrows = r.nrows;
  it.shared = r.part >= 0 ? (r.part & kSharedTile) != 0 : (~r.part & kSharedTile) != 0;
  it.part = r.part >= 0 ? r.part & ~kSharedTile : -1;
  it.seq = r.seq;
  it.k0 = r.k0;
  it.k1 = r.k1;
  it.token0 = r.token0;
  it.pos0 = r.pos0;
  it.len = r.len;
  it.gap_at = r.gap_at;
  it.gap = r.gap;
  it.w0 = r.w0;
  return true;
}

__device__ inline bool writes_outputs(const PrefixArgs& a, const PrefixItem&) { return a.prefix_chunks + a.own_chunks == 1; }
__device__ inline bool writes_outputs(const ChunkArgs&, const ChunkItem& it) { return it.part < 0; }

// A row of an item.
__device__ inline PrefixRow item_row(const PrefixArgs& a, const PrefixItem& it, int row) {
  return prefix_row(a, it.kvh, it.row0 + row);
}
struct ChunkRow : PrefixRow {
  int lo;  // it sees [0, sinks) and [lo, end) of the walk
};
__device__ inline ChunkRow item_row(const ChunkArgs& a, const ChunkItem& it, int row) {
  ChunkRow x;
  const int n = it.row0 + row, i = n / a.group;
  x.token = it.token0 + i;
  x.head = it.kvh * a.group + (n - i * a.group);
  const int at = it.pos0 + i;
  const int e = at < 0 ? 0 : a.M * (at / a.M + 1), end = imin(e, it.len);
  x.lo = (a.window > 0 ? imax(e - a.window, 0) : 0) - it.gap;
  x.end = end <= it.gap_at ? end : imax(end - it.gap, it.gap_at);
  return x;
}
template <int D> __device__ inline int64_t q_elem(const PrefixArgs& a, const PrefixRow& x) {
  return ((int64_t)x.token * a.heads + x.head) * D;
}
template <int D> __device__ inline int64_t o_elem(const PrefixArgs& a, const PrefixRow& x) { return q_elem<D>(a, x); }
template <int D> __device__ inline int64_t q_elem(const ChunkArgs& a, const PrefixRow& x) {
  return x.token * a.qs + (int64_t)x.head * D;
}
template <int D> __device__ inline int64_t o_elem(const ChunkArgs& a, const PrefixRow& x) {
  return x.token * a.os + (int64_t)x.head * D;
}
__device__ inline int64_t lse_elem(const PrefixArgs& a, const PrefixRow& x) { return prefix_lse_at(a, x); }
__device__ inline int64_t lse_elem(const ChunkArgs& a, const PrefixRow& x) { return x.head * a.pitch + x.token; }
// The partial row of the item's row `row`.
__device__ inline int64_t part_row(const PrefixArgs& a, const PrefixItem& it, const PrefixRow& x, int) {
  return (int64_t)it.part * a.requests * a.rows * a.heads + ((int64_t)x.token * a.heads + x.head);
}
__device__ inline int64_t part_row(const ChunkArgs& a, const ChunkItem& it, const PrefixRow&, int row) {
  return it.kvh * a.part_rows + it.part + row;
}

// key / page_size.  Chunks: (key page_mul >> 32) >> page_shift, with page_mul = 1 + floor(2^(32 + page_shift) /
// page_size), 2^page_shift < page_size <= 2^(page_shift + 1), which is that for key < 2^31 (page_size 1: page_mul 0).
__device__ inline int page_of(const PrefixArgs& a, int key) { return key / a.page_size; }
__device__ inline int page_of(const ChunkArgs& a, int key) {
  return a.page_mul ? (int)(__umulhi((uint32_t)key, a.page_mul) >> a.page_shift) : key;
}

// Key v of the walk.
__device__ inline int walk_key(const PrefixItem&, int v) { return v; }
__device__ inline int walk_key(const ChunkItem& it, int v) { return v < it.gap_at ? v : v + it.gap; }

// The pages of an item's keys, one table entry after the other: entries of the keys
// below the gap, then of those above.
struct WalkPages {
  int p0, n0, p1, n;  // first page and entries below the gap, first page above, entries in all
  __device__ inline int page(int e) const { return e < n0 ? p0 + e : p1 + (e - n0); }
};
__device__ inline WalkPages walk_pages(const ChunkArgs& a, const ChunkItem& it) {
  WalkPages w{0, 0, 0, 0};
  if (it.k1 <= it.k0) return w;
  const int below = imin(it.k1, it.gap_at);
  if (it.k0 < below) {
    w.p0 = it.k0 / a.page_size;
    w.n0 = (below - 1) / a.page_size - w.p0 + 1;
  }
  w.n = w.n0;
  if (it.k1 > it.gap_at) {
    w.p1 = (imax(it.k0, it.gap_at) + it.gap) / a.page_size;
    w.n += (it.k1 - 1 + it.gap) / a.page_size - w.p1 + 1;
  }
  return w;
}

// Rows behind the last request's: the workgroups without an item write zeros (LSE -inf).  With a plan that does not fit,
// all rows become NaN.
template <class T, int D>
__device__ inline void fill_rest(const PrefixArgs&, int, int) {}
template <class T, int D>
__device__ inline void fill_rest(const ChunkArgs& a, int wg, int wgs) {
  const bool fits = plan_fits(a);
  if (fits && !a.fill) return;
  const int used = plan_items(a) * a.kv_heads, first = fits ? a.plan[kPlanRows] : 0;
  typedef int quad __attribute__((ext_vector_type(4)));
  const int x = fits ? 0 : sizeof(T) == 2 ? 0x7fc07fc0 : 0x7fc00000;  // (NaN)
  const float z = fits ? -INFINITY : __builtin_nanf("");
  constexpr int PR = D * (int)sizeof(T) / 16;  // 16-byte pieces of a head's row
  const int64_t n = (int64_t)(a.rows - first) * a.heads * PR, step = (int64_t)(wgs - used) * blockDim.x;
  for (int64_t i = (int64_t)(wg - used) * blockDim.x + threadIdx.x; i < n; i += step) {
    const int64_t hr = i / PR, row = hr / a.heads + first, h = hr % a.heads;
    *(quad*)((T*)a.o + row * a.os + h * D + (i % PR) * (16 / (int)sizeof(T))) = quad{x, x, x, x};
    if (i % PR == 0) a.lse[h * a.pitch + row] = z;
  }
}

}  // namespace bdlm
