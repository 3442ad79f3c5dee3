// Key-major work items shared by the dK/dV kernels: key tiles whose walks may
// be cut into chunks (SplitArgs in common.hpp), and the sums over the chunks.
#pragma once

#include "common.hpp"
#include "packed.hpp"

namespace bdlm {

// The key tile of a workgroup of the dK/dV kernel: tiles of a (batch, KV head)
// pair in visiting order (heaviest range first), the first chunks of all tiles
// of a range, then the second ones, and so on: the workgroups that run side by
// side then read the same query rows (the walks of the scheduled kernel start
// at the last query row whatever the tile).
struct KeyTileItem {
  int b, kvh, r, t, chunk;
  int tile;  // index among the tiles of the chunked ranges of all pairs (of the tile's count)
  int item;  // packed calls: the plan's item
};
__device__ inline bool key_tile_item(const AttnArgs& a, int wg, KeyTileItem& it) {
  int bk, rank;
  if (!xcd_pair_item(wg, a.kv_heads * a.batch, a.split.wgs_per_pair, true, bk, rank)) return false;
  it.b = bk / a.kv_heads;
  it.kvh = bk - it.b * a.kv_heads;
  it.r = a.order[0];
  it.tile = bk * a.split.tiles_per_pair;
  for (int n = 0; n < a.n_k; ++n) {
    const int r = a.order[n], ch = a.split.chunks[r], nw = a.kr[r].ntiles * ch;
    it.r = r;
    if (rank < nw) break;
    rank -= nw;
    if (ch > 1) it.tile += a.kr[r].ntiles;
  }
  const int nt = imax(a.kr[it.r].ntiles, 1);
  it.chunk = rank / nt;
  it.t = rank - it.chunk * nt;
  it.tile += it.t;
  return true;
}

// The same of a packed call: a chunk of a key tile's walk, as the plan cut it.
__device__ inline bool key_tile_item(const PackedArgs& a, int wg, KeyTileItem& it) {
  if (!xcd_pair_item(wg, a.kv_heads, a.n_items, true, it.kvh, it.item)) return false;
  it.b = it.r = it.chunk = it.tile = 0;
  it.t = a.items[it.item].tile;
  return true;
}

// With sinks: tile -1 - t is the t-th of the sinks (packed.hpp).
__device__ inline bool key_tile_item(const SinkKArgs& a, int wg, KeyTileItem& it) {
  if (!key_tile_item(static_cast<const PackedArgs&>(a), wg, it)) return false;
  if (it.t < 0) it.t = -1 - it.t;
  return true;
}

// A workgroup's chunk of its tile's walk: steps [n0, n1), and whether the walk is
// cut (then it leaves partial sums, else it writes the gradients).  False: no such chunk.
struct Chunk {
  int n0, n1;
  bool cut;
};
template <class View>
__device__ __forceinline__ bool chunk_of(const AttnArgs& a, const View&, const KeyTileItem& it, int nsteps, int tid,
                                         Chunk& c) {
  const int max_ch = a.split.chunks[it.r];
  const int nch = max_ch > 1 ? chunks_of(nsteps, a.split.unit, max_ch) : 1;
  if (max_ch > 1 && it.chunk == 0 && tid == 0) a.split.counts[it.tile] = nch;
  if (it.chunk >= nch) return false;
  c.n0 = it.chunk * a.split.unit;
  c.n1 = it.chunk + 1 < nch ? c.n0 + a.split.unit : nsteps;
  c.cut = nch > 1;
  return true;
}
template <class View>
__device__ __forceinline__ bool chunk_of(const PackedArgs& a, const View&, const KeyTileItem& it, int nsteps, int,
                                         Chunk& c) {
  const PackedItem& p = a.items[it.item];
  c.n0 = p.n0;
  c.n1 = imin(p.n1, nsteps);
  c.cut = p.slot >= 0;
  return true;
}

// First row of the partial sums of a chunk of key tile t (of ROWS rows) of range r.
template <int ROWS>
__device__ inline int64_t partial_row(const AttnArgs& a, int b, int kvh, int r, int t, int chunk) {
  const KRangeArg& kr = a.kr[r];
  return (int64_t)(b * a.kv_heads + kvh) * a.split.rows_per_pair + kr.pos0 + t * ROWS + a.split.at[kr.stream][chunk];
}

// ... of this workgroup's chunk.
template <int ROWS>
__device__ inline int64_t partial_row(const AttnArgs& a, const KeyTileItem& it) {
  return partial_row<ROWS>(a, it.b, it.kvh, it.r, it.t, it.chunk);
}
template <int ROWS>
__device__ inline int64_t partial_row(const PackedArgs& a, const KeyTileItem& it) {
  return ((int64_t)a.items[it.item].slot * a.kv_heads + it.kvh) * ROWS;
}

// A tile of the chunked ranges, for the kernel that adds up its chunks: tile
// `n` of all pairs' chunked tiles.
struct SumItem {
  int b, kvh, r, t;
};
__device__ inline void sum_item(const AttnArgs& a, int n, SumItem& it) {
  const int bk = n / a.split.tiles_per_pair;
  int tile = n - bk * a.split.tiles_per_pair;
  it.b = bk / a.kv_heads;
  it.kvh = bk - it.b * a.kv_heads;
  it.r = a.order[0];
  for (int k = 0; k < a.n_k; ++k) {
    const int r = a.order[k];
    it.r = r;
    if (a.split.chunks[r] <= 1) continue;
    if (tile < a.kr[r].ntiles) break;
    tile -= a.kr[r].ntiles;
  }
  it.t = tile;
}

// What the summing kernel of tiles of ROWS keys reads and writes for tile `n`:
// chunks (1: nothing to add), keys of the tile, the partial rows of chunk ch,
// and the element of key `key` of the tile in dK and dV.
template <int ROWS>
struct SumTile {
  int n, nk, kvh;
  int64_t dk, dv, dks, dvs;  // first key's element and the elements between keys
  int64_t row0, step;        // packed calls: partial rows of chunk ch at row0 + ch * step
  SumItem it;
};
template <int ROWS, int D>
__device__ inline SumTile<ROWS> sum_tile(const AttnArgs& a, int n) {
  SumTile<ROWS> s;
  sum_item(a, n, s.it);
  const KRangeArg& kr = a.kr[s.it.r];
  s.n = a.split.counts[n];
  s.nk = imin(ROWS, kr.len - s.it.t * ROWS);
  s.kvh = s.it.kvh;
  s.dks = s.dvs = (int64_t)a.kv_heads * D;
  s.dk = s.dv = (((int64_t)s.it.b * kr.bstride + s.it.t * ROWS) * a.kv_heads + s.it.kvh) * D;
  return s;
}
template <int ROWS, int D>
__device__ inline SumTile<ROWS> sum_tile(const PackedArgs& a, int n) {
  SumTile<ROWS> s;
  const PackedSum& p = a.sums[n / a.kv_heads];
  s.kvh = n - n / a.kv_heads * a.kv_heads;
  s.n = p.n;
  s.nk = imin(ROWS, p.len - p.tile * ROWS);
  s.dks = a.dks;
  s.dvs = a.dvs;
  s.dk = ((int64_t)p.row0 + p.tile * ROWS) * a.dks + s.kvh * D;
  s.dv = ((int64_t)p.row0 + p.tile * ROWS) * a.dvs + s.kvh * D;
  s.row0 = ((int64_t)p.slot * a.kv_heads + s.kvh) * ROWS;
  s.step = (int64_t)a.kv_heads * ROWS;
  s.it = SumItem{};
  return s;
}
template <int ROWS>
__device__ inline int64_t partial_row(const AttnArgs& a, const SumTile<ROWS>& s, int ch) {
  return partial_row<ROWS>(a, s.it.b, s.it.kvh, s.it.r, s.it.t, ch);
}
template <int ROWS>
__device__ inline int64_t partial_row(const PackedArgs&, const SumTile<ROWS>& s, int ch) {
  return s.row0 + ch * s.step;
}
__device__ inline void* partials_of(const AttnArgs& a) { return a.split.partials; }
__device__ inline void* partials_of(const PackedArgs& a) { return a.partials; }
__device__ inline void* dk_of(const AttnArgs& a, const SumItem& it) { return a.kr[it.r].dk; }
__device__ inline void* dv_of(const AttnArgs& a, const SumItem& it) { return a.kr[it.r].dv; }
__device__ inline void* dk_of(const PackedArgs& a, const SumItem&) { return a.dk; }
__device__ inline void* dv_of(const PackedArgs& a, const SumItem&) { return a.dv; }

}  // namespace bdlm
