// Query-major tiling shared by the forward and the dQ kernel.
//
// A workgroup owns BM consecutive query rows of one query range and one query
// head and walks the key tiles (BN rows) of every key range that any of its
// rows can see.  The visible keys of a query row form one position interval
// (common.hpp), whose ends are non-decreasing in the query position, so for
// the tile's rows [pq0, pq1] the union of the intervals is [lo(pq0), hi(pq1))
// and the intersection is [lo(pq1), hi(pq0)): key tiles outside the union are
// never visited and key tiles inside the intersection need no mask test.
#pragma once

#include "common.hpp"
#include "device.hpp"
#include "packed.hpp"

namespace bdlm {

struct QTileItem {
  int b, h, r, t;  // batch, query head, query range, tile within the range
  int item;        // packed calls: the plan's item
};

// Hardware workgroup -> (batch, query head, query range, tile); false: no item.
// The items of a (batch, KV head) pair meet in one XCD group (xcd_pair_item);
// within a pair the query heads of the group are interleaved, and the tiles of
// each range run from the last (longest key prefix) to the first.
template <int HP = 1>
__device__ inline bool q_tile_item(const AttnArgs& a, int wg, QTileItem& it) {
  int bk, rank;
  if (!xcd_pair_item(wg, a.kv_heads * a.batch, a.group * a.total_tiles, false, bk, rank)) return false;
  it.b = bk / a.kv_heads;
  const int kvh = bk - it.b * a.kv_heads;
  const int order = rank / a.group;
  it.h = kvh * a.group + (rank - order * a.group);
  if (a.interleave) {
    it.r = order % a.n_q;
    it.t = a.qr[it.r].ntiles - 1 - order / a.n_q;
  } else {
    int r = 0;
    while (r + 1 < a.n_q && order >= a.qr[r + 1].tile0) ++r;
    it.r = r;
    it.t = a.qr[r].ntiles - 1 - (order - a.qr[r].tile0);
  }
  return true;
}

// The same of a packed call, whose items lie heaviest first in the plan; h is
// the first of the HP query heads that a tile's waves take.
template <int HP = 1>
__device__ inline bool q_tile_item(const PackedArgs& a, int wg, QTileItem& it) {
  int rank;
  const int per = a.group / HP;
  if (!xcd_pair_item(wg, a.kv_heads, per * a.n_items, false, it.b, rank)) return false;
  it.item = rank / per;
  it.h = it.b * a.group + (rank - it.item * per) * HP;
  it.b = it.r = 0;
  it.t = a.items[it.item].tile;
  return true;
}

// The key tiles [t, t1) of a packed item's chunk of its tile's walk [t, t1).
__device__ inline void cut_walk(const AttnArgs&, const QTileItem&, int&, int&, bool&) {}
__device__ inline void cut_walk(const PackedArgs& a, const QTileItem& it, int& t, int& t1, bool& have) {
  const PackedItem& p = a.items[it.item];
  t1 = imin(t1, t + p.n1);
  t += p.n0;
  have = have && t < t1;
}
__device__ inline bool first_chunk(const AttnArgs&, const QTileItem&) { return true; }
__device__ inline bool first_chunk(const PackedArgs& a, const QTileItem& it) { return a.items[it.item].n0 == 0; }
// The row of its partial sums, [slot][heads / HP][row of the waves], for row l32 of wave w.
template <int NW, int HP>
__device__ inline int64_t q_partial_row(const PackedArgs& a, const QTileItem& it, int w, int l32) {
  return ((int64_t)a.items[it.item].slot * (a.heads / HP) + it.h / HP) * (NW * 32) + w * 32 + l32;
}

// Key tiles [t0, t1) of key range j that any query position in [pq0, pq1]
// can see, and the sub-span [f0, f1) every one of them sees completely.
template <class A>
__device__ inline void key_tile_span(const A& a, int j, int qs, int pq0, int pq1, int BN,
                                     int& t0, int& t1, int& f0, int& f1) {
  const KRangeArg& kr = k_range(a, j);
  int lo0, hi0, lo1, hi1;
  key_interval(qs, pq0, kr.stream, rule_of(a), lo0, hi0);
  key_interval(qs, pq1, kr.stream, rule_of(a), lo1, hi1);
  const int u0 = imax(lo0 - kr.pos0, 0), u1 = imin(hi1 - kr.pos0, kr.len);
  t0 = t1 = f0 = f1 = 0;
  if (u1 <= u0) return;
  t0 = u0 / BN;
  t1 = (u1 + BN - 1) / BN;
  const int i0 = imax(lo1 - kr.pos0, 0), i1 = imin(hi0 - kr.pos0, kr.len);
  if (i1 > i0) {
    f0 = (i0 + BN - 1) / BN;
    f1 = i1 / BN;
  }
}

// With sinks: the walk's tiles (packed.hpp), those that all rows see among them.
struct NoSinks {};
template <class A>
__device__ inline NoSinks sink_walk_of(const A&, int, int) { return {}; }
__device__ inline SinkWalk sink_walk_of(const SinkView& a, int pq0, int pq1) {
  return sink_walk(a.rule, a.sinks, pq0, pq1, a.kr[0].pos0, a.kr[0].len);
}
__device__ inline void key_tile_span(const SinkView& a, int, int, int pq0, int pq1, int BN, int& t0, int& t1, int& f0,
                                     int& f1) {
  const SinkWalk w = sink_walk_of(a, pq0, pq1);
  int lo0, hi0, lo1, hi1;
  key_interval(kClean, pq0, kClean, a.rule, lo0, hi0);
  key_interval(kClean, pq1, kClean, a.rule, lo1, hi1);
  const int lo = imax(lo1 - a.kr[0].pos0, 0) - w.gap, hi = imin(hi0 - a.kr[0].pos0, a.kr[0].len) - w.gap;
  t0 = f0 = f1 = 0;
  t1 = (w.n + BN - 1) / BN;
  if (hi > 0) {
    f0 = lo <= a.sinks ? 0 : (lo + BN - 1) / BN;
    f1 = hi / BN;
  }
}
// This lane's part of it: its window at [lo, lo + w) (positions as if the walk were
// the sequence), and the end of its sinks.
__device__ inline void lane_walk(const SinkView& a, const SinkWalk& w, int pq, int& lo, int& wid, int& sinks) {
  const int pos0 = a.kr[0].pos0;
  int l, h;
  key_interval(kClean, pq, kClean, a.rule, l, h);
  l = imax(l - pos0, 0) - w.gap;
  h = imin(h - pos0, a.kr[0].len);
  h = h <= w.gap_at ? h : imax(h - w.gap, w.gap_at);
  lo = pos0 + l;
  wid = imax(h - l, 0);
  sinks = imin(a.sinks, h);
}
// The keys that it sees.
__device__ inline int row_keys(const SinkView& a, const SinkWalk& w, int pq) {
  int lo, wid, sinks;
  lane_walk(a, w, pq, lo, wid, sinks);
  lo -= a.kr[0].pos0;
  return imax(sinks, 0) + imax(lo + wid - imax(lo, sinks), 0);
}

// With sinks, fp32: the sinks, and the window's tiles among the other keys.
__device__ inline void key_tile_span(const SinkViewF32& a, int j, int, int pq0, int pq1, int BN, int& t0, int& t1, int& f0,
                                     int& f1) {
  const int pos0 = a.kr[0].pos0, n = a.kr[0].ntiles, S = a.sinks;
  int lo0, hi0, lo1, hi1;
  key_interval(kClean, pq0, kClean, a.rule, lo0, hi0);
  key_interval(kClean, pq1, kClean, a.rule, lo1, hi1);
  // (the window's ends from key S on; of the sinks a row sees those before its end)
  const int u0 = j == 0 ? 0 : imax(lo0 - pos0 - S, 0), i0 = j == 0 ? 0 : imax(lo1 - pos0 - S, 0);
  const int u1 = j == 0 ? imin(hi1 - pos0, S) : imin(hi1 - pos0, n) - S;
  const int i1 = j == 0 ? imin(hi0 - pos0, S) : imin(hi0 - pos0, n) - S;
  t0 = t1 = f0 = f1 = 0;
  if (u1 <= u0) return;
  t0 = u0 / BN;
  t1 = (u1 + BN - 1) / BN;
  if (i1 > i0) {
    f0 = (i0 + BN - 1) / BN;
    f1 = i1 / BN;
  }
}

// First key tile at or after key range jj that the query tile can see.
template <class A>
__device__ inline bool find_key_tile(const A& a, int jj, int qs, int pq0, int pq1, int BN,
                                     int& jo, int& to, int& t1o, int& f0o, int& f1o) {
  for (; jj < a.n_k; ++jj) {
    int a0, a1, b0, b1;
    key_tile_span(a, jj, qs, pq0, pq1, BN, a0, a1, b0, b1);
    if (a1 > a0) {
      jo = jj;
      to = a0;
      t1o = a1;
      f0o = b0;
      f1o = b1;
      return true;
    }
  }
  return false;
}

// Packed calls: the keys [u0, u1) of the sequence that some row of the query
// tile can see.  Only these are copied: what the others hold, an evicted or
// unwritten part of a window's past, say, must not meet a probability of zero
// as an infinity or NaN.
__device__ inline void seen_keys(const AttnArgs&, int, int, int& u0, int& u1) {
  u0 = 0;
  u1 = kBig;
}
__device__ inline void seen_keys(const PackedView& a, int pq0, int pq1, int& u0, int& u1) {
  const KRangeArg& kr = a.kr[0];
  int lo0, hi0, lo1, hi1;
  key_interval(kClean, pq0, kClean, rule_of(a), lo0, hi0);
  key_interval(kClean, pq1, kClean, rule_of(a), lo1, hi1);
  u0 = imax(lo0 - kr.pos0, 0);
  u1 = imin(hi1 - kr.pos0, kr.len);
}

// Key tiles of all ranges that the query tile can see.
template <class A>
__device__ inline int count_key_tiles(const A& a, int qs, int pq0, int pq1, int BN) {
  int n = 0;
  for (int j = 0; j < a.n_k; ++j) {
    int a0, a1, b0, b1;
    key_tile_span(a, j, qs, pq0, pq1, BN, a0, a1, b0, b1);
    n += a1 - a0;
  }
  return n;
}

// This lane's visible key interval [lo, lo + w) inside key range j (w may be 0).
template <class A>
__device__ inline void lane_key_interval(const A& a, int j, int qs, int pq, int& lo, int& w) {
  const KRangeArg& kr = k_range(a, j);
  int l, h;
  key_interval(qs, pq, kr.stream, rule_of(a), l, h);
  l = imax(l, kr.pos0);
  h = imin(h, kr.pos0 + kr.len);
  lo = l;
  w = imax(h - l, 0);
}

__device__ inline void lane_key_interval(const SinkViewF32& a, int j, int, int pq, int& lo, int& w) {
  const int pos0 = a.kr[0].pos0;
  int l, h;
  key_interval(kClean, pq, kClean, a.rule, l, h);
  lo = j == 0 ? pos0 : imax(l, pos0 + a.sinks);
  w = imax(imin(h, pos0 + (j == 0 ? a.sinks : a.kr[0].ntiles)) - lo, 0);
}

}  // namespace bdlm
