// The plan of a packed call (packed.hpp): its work items, from the sequences'
// lengths.  Host code, no HIP calls.
#pragma once

#include "bdlm_attn.h"

#include <algorithm>
#include <cmath>
#include <functional>
#include <vector>

#include "packed.hpp"
#include "split_plan.hpp"

namespace bdlm {

struct PackedPlanItems {
  std::vector<PackedItem> q, k;
  std::vector<PackedSum> sums;
  int32_t slots = 0;
  struct Chunks {  // in place of q, if some of its walks are cut
    std::vector<PackedItem> items;
    std::vector<PackedSum> sums;
    int32_t slots = 0;
  } fwd, dq;
  int32_t teams = 1;
};

inline int packed_step_rows(bool f32, int group) { return f32 ? kRowsF32 : group % 2 ? 64 : 32; }

// Partial sums of cut walks at most (per call); longer chunks where they would come to more.
constexpr size_t kMaxPackedPartials = (size_t)256 << 20;

// Key tiles of a query tile's chunks at least; what partial sums cost, in key tiles.
constexpr int64_t kMinFwdUnit = 8, kFwdSumTiles = 10, kFwdSumTiles64 = 18, kDqSumTiles = 8;
// What a workgroup's start-up costs, in key tiles.
constexpr int64_t kStartTiles = 3;

// Work items, heaviest first: a workgroup that starts late should be short.
//
// Query tiles: 128 rows (16 in fp32) of one sequence, or as many fewer as a
// tile has heads (packed_tile_heads), by the keys they walk.
//
// Forward and dQ, bf16: where few tiles have long walks (a piece of a long prompt,
// few heads), the busiest CU's walks, not the card, set the time.  If they are longer
// than the average load of a CU by more than partial outputs cost, walks are cut
// into equal chunks of at most that load, a chunk per CU, whose outputs
// packed_q_sums.hip joins (the factor is what a chunk's tiles take longer without a
// second team; dQ has none in any case, and is cut sooner and, with more tiles than
// CUs, into shorter chunks).  d 128, without and with cuts, 32/8 heads: 1 row behind
// 2,048 keys 33 and 19 us, behind 8,192 109 and 22, behind 32,768 444 and 40; 256 rows
// 37 and 30, 119 and 59, 438 and 184; 512 rows behind 2,048 are left whole (42, 47
// cut), 1,024 behind 8,192 too (155, 193); 3,000 rows of 4/2 heads 45 and 32, dQ 74
// and 39; dQ of 2,667, 200 and 15, 12/2 heads, 68 and 56, of 2,213, 600 and 152, 16/16,
// 68 and 60.  (Chunks that fill two workgroups a CU write twice the partial outputs:
// 256 rows behind 8,192 65 us.)
//
// Two teams per workgroup (fwd_bf16.hip): up to a workgroup per CU, as in joint
// calls, and up to two where a CU that takes them one after the other, as it gets
// free, ends before one that holds two at once: with uneven walks (prompts of 1,355
// rows, 24/8 heads, 288 workgroups 35 -> 27 us; 2,213, 600 and 152, 16/16 heads, 54
// -> 41; 3,000, 16/4 heads, 69 -> 53; 2,048, 32/8 heads 51 -> 46), not with even or
// short ones (8 of 500, 16/4 heads 20, 23; 1,000 and 800 behind 4,000 140, 149).
//
// Key tiles: 128 keys (16), by the steps of their walks.  The longest walk,
// the first keys' of the longest sequence, sets the time when there are few;
// walks longer than the average load of a CU's workgroups are cut into chunks of
// that load as in split_plan.hpp, whose reasons and limits hold here too (fp32:
// the whole load, not a quarter of it: 5 texts of 33 to 407 rows, 8/2 heads, d 64
// 46 -> 43 us, of which the sums 10 -> 5; bf16, 8K of documents: 0.5, 0.75, 1 and
// 1.5 loads 263, 252, 245 and 261 us).
//
// Sinks (packed.hpp): a query tile's walk is that of its sinks and its window; a
// sequence's key tiles are those of its sinks, numbered -1 - t, which all rows from
// theirs on walk, and those of its other keys.
inline PackedPlanItems packed_items(const bdlm_packed& p, int64_t n, const bdlm_packed_seq* seqs) {
  PackedPlanItems out;
  const bool f32 = p.dtype == BDLM_F32;
  const int M = (int)p.block_size, group = p.heads / p.kv_heads;
  const int tile_heads = f32 ? 1 : packed_tile_heads(group);
  const int q_tile = f32 ? kRowsF32 : kQRowsShortBf16 / tile_heads, k_tile = f32 ? kRowsF32 : kBwdKeysBf16;
  const int step = packed_step_rows(f32, group);
  const int64_t per_block = f32 || group % 2 ? group : group / 2;
  const MaskRule rule{M, kIntraBlock, (int)p.window, 1, kBig, nullptr}, always{M, kIntraBlock, 0, 1, kBig, nullptr};

  struct Cost {
    int64_t cost;
    PackedItem it;
  };
  std::vector<Cost> q, k, walks;  // walks: the query tiles by 64-key tiles
  int64_t total = 0, fwd_total = 0;
  for (int64_t i = 0; i < n; ++i) {
    const bdlm_packed_seq& s = seqs[i];
    const int ql = (int)s.q_len, kl = (int)s.k_len;
    const int shift = packed_shift(ql, kl, M), qp = shift + kl - ql;
    PackedItem it{(int32_t)s.q_start, ql, (int32_t)s.k_start, kl, 0, 0, kBig, -1};
    for (int t = 0; t * (int64_t)q_tile < ql; ++t) {
      const int first = t * q_tile, last = std::min(ql, first + q_tile) - 1;
      int lo, hi, lo1, hi1;
      key_interval(kClean, qp + first, kClean, rule, lo, hi);
      key_interval(kClean, qp + last, kClean, rule, lo1, hi1);
      it.tile = t;
      const int u0 = std::max(lo - shift, 0), u1 = std::min(hi1 - shift, kl);
      if (p.sinks == 0) {
        q.push_back({std::max(0, u1 - u0), it});
        walks.push_back({u1 > u0 ? (u1 + 63) / 64 - u0 / 64 : 0, it});
      } else {
        const int n = sink_walk(rule, std::min(p.sinks, kl), qp + first, qp + last, shift, kl).n;
        q.push_back({n, it});
        walks.push_back({(n + 63) / 64, it});
      }
      fwd_total += walks.back().cost;
    }
    const int sinks = std::min(p.sinks, kl);
    auto key_tiles = [&](int from, int to, const MaskRule& seen, bool sink) {  // keys [from, to) of the sequence
      for (int t = 0; from + t * (int64_t)k_tile < to; ++t) {
        const int first = from + t * k_tile, last = std::min(to, first + k_tile) - 1;
        int lo, hi, lo1, hi1;
        query_interval(kClean, kClean, shift + first, seen, lo, hi);
        query_interval(kClean, kClean, shift + last, seen, lo1, hi1);
        const int u0 = std::max(lo - qp, 0), u1 = std::min(hi1 - qp, ql);
        const int64_t steps = u1 > u0 ? ((u1 + step - 1) / step - u0 / step) * per_block : 0;
        it.tile = sink ? -1 - t : t;
        k.push_back({steps, it});
        total += steps * p.kv_heads;
      }
    };
    key_tiles(0, sinks, always, true);
    key_tiles(sinks, kl, rule, false);
  }
  auto heavier = [](const Cost& a, const Cost& b) { return a.cost > b.cost; };
  std::stable_sort(q.begin(), q.end(), heavier);
  std::stable_sort(k.begin(), k.end(), heavier);
  for (const Cost& c : q) out.q.push_back(c.it);
  const int64_t per = p.heads / tile_heads;  // workgroups of a query tile

  // Chunks of the query tiles' walks (bf16).
  std::stable_sort(walks.begin(), walks.end(), heavier);
  const int64_t fwd_longest = walks.empty() ? 0 : walks[0].cost;
  const int64_t wgs = (int64_t)walks.size() * per, fwd_average = (fwd_total * per + kCus - 1) / kCus;
  const int64_t unit_q = std::max(kMinFwdUnit, fwd_average);
  // what the busiest CU walks without cuts: all workgroups resident, or dealt out as others end
  int64_t busiest = 0;
  if (wgs <= kCus * (p.head_dim == 64 ? 3 : 2))
    for (int64_t i = 0; i < wgs; i += kCus) busiest += walks[i / per].cost;
  else
    busiest = std::max(fwd_longest, fwd_average);
  const int64_t busiest_dq = busiest;
  bool teams = !f32 && wgs <= kTeamWgs;
  if (!f32 && wgs > kTeamWgs && wgs <= 2 * kTeamWgs) {  // one workgroup of two teams per CU, the next when it ends
    std::vector<int64_t> load(kCus, 0);  // (a heap, the least loaded CU first)
    int64_t most = 0;
    for (int64_t i = 0; i < wgs; ++i) {
      std::pop_heap(load.begin(), load.end(), std::greater<int64_t>());
      int64_t& cu = load.back();
      cu += walks[i / per].cost + (cu > 0 ? kStartTiles : 0);
      most = std::max(most, cu);
      std::push_heap(load.begin(), load.end(), std::greater<int64_t>());
    }
    teams = most * 13 <= busiest * 12;
    if (teams) busiest = most;
  }
  auto cut = [&](int64_t unit, PackedPlanItems::Chunks& to) {
    const int64_t most = (int64_t)(kMaxPackedPartials / (per * kQRowsShortBf16 * p.head_dim * sizeof(float)));
    for (;; unit *= 2) {
      int64_t slots = 0;
      for (const Cost& c : walks)
        if (c.cost > unit) slots += (c.cost + unit - 1) / unit;
      if (slots <= most) break;
    }
    std::vector<Cost> chunks;
    for (const Cost& c : walks) {
      const int64_t nch = std::max<int64_t>((c.cost + unit - 1) / unit, 1), size = (c.cost + nch - 1) / nch;
      PackedItem it = c.it;
      if (nch > 1) to.sums.push_back({it.q0, it.q_len, it.tile, to.slots, (int32_t)nch, 0, 0, 0});
      for (int64_t j = 0; j < nch; ++j) {
        it.n0 = (int32_t)(j * size);
        it.n1 = j + 1 < nch ? (int32_t)((j + 1) * size) : kBig;
        it.slot = nch > 1 ? to.slots++ : -1;
        chunks.push_back({std::max<int64_t>(0, std::min(c.cost, (j + 1) * size) - j * size), it});
      }
    }
    if (to.slots == 0) return;
    std::stable_sort(chunks.begin(), chunks.end(), heavier);
    for (const Cost& c : chunks) to.items.push_back(c.it);
  };
  const int64_t sum_tiles = p.head_dim == 64 ? kFwdSumTiles64 : kFwdSumTiles;
  if (!f32 && busiest > unit_q * 8 / 5 + sum_tiles) cut(unit_q, out.fwd);
  if (!f32 && busiest_dq > unit_q * 23 / 20 + kDqSumTiles)
    cut(wgs > kCus ? std::max(kMinFwdUnit, unit_q * 3 / 4) : unit_q, out.dq);
  if (teams && out.fwd.items.empty()) out.teams = 2;

  // Chunks of the key tiles' walks.
  const int64_t longest = k.empty() ? 0 : k[0].cost;
  const int64_t average = total / (f32 ? kCus : kCus * dkdv_wgs_per_cu(p.head_dim, 0, group));
  int64_t unit = std::max<int64_t>(f32 ? kMinUnitF32 : kMinUnitBf16, average);
  if (!f32 && average < kMinUnitBf16) {  // a nearly idle card: as split_plan
    const int64_t u = std::max<int64_t>(kMinUnitBf16Idle, average);
    int64_t wgs = 0;
    for (const Cost& c : k) wgs += std::max<int64_t>((c.cost + u - 1) / u, 1);
    if (wgs * p.kv_heads <= kCus) unit = u;
  }
  const int64_t margin = f32 ? 0 : std::min<int64_t>(kCutSteps, average / 3);
  const size_t slot_bytes = (size_t)p.kv_heads * k_tile * 2 * p.head_dim * (f32 ? sizeof(double) : sizeof(float));
  if (longest <= average + margin) unit = longest;
  for (; longest > unit; unit *= 2) {
    int64_t slots = 0;
    for (const Cost& c : k)
      if (c.cost > unit) slots += (c.cost + unit - 1) / unit;
    if (slots <= (int64_t)(kMaxPackedPartials / slot_bytes)) break;
  }
  std::vector<Cost> chunks;
  for (const Cost& c : k) {
    const int64_t nch = c.cost > unit ? (c.cost + unit - 1) / unit : 1;
    PackedItem it = c.it;
    if (nch > 1) {
      const int sinks = std::min(p.sinks, it.k_len);
      out.sums.push_back(it.tile < 0 ? PackedSum{it.k0, sinks, -1 - it.tile, out.slots, (int32_t)nch, 0, 0, 0}
                                     : PackedSum{it.k0 + sinks, it.k_len - sinks, it.tile, out.slots, (int32_t)nch, 0, 0, 0});
    }
    for (int64_t j = 0; j < nch; ++j) {
      it.n0 = (int32_t)(j * unit);
      it.n1 = j + 1 < nch ? (int32_t)((j + 1) * unit) : kBig;
      it.slot = nch > 1 ? out.slots++ : -1;
      chunks.push_back({j + 1 < nch ? unit : c.cost - j * unit, it});
    }
  }
  std::stable_sort(chunks.begin(), chunks.end(), heavier);
  for (const Cost& c : chunks) out.k.push_back(c.it);
  return out;
}

}  // namespace bdlm
