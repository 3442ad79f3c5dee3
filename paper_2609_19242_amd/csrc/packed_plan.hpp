// The plan of a packed call (packed.hpp): its work items, from the sequences'
// lengths.  Host code, no HIP calls.
#pragma once

#include "bdlm_attn.h"

#include <algorithm>
#include <cmath>
#include <vector>

#include "packed.hpp"
#include "split_plan.hpp"

namespace bdlm {

struct PackedPlanItems {
  std::vector<PackedItem> q, k;
  std::vector<PackedSum> sums;
  int32_t slots = 0;
  int32_t teams = 1;
};

inline int packed_step_rows(bool f32, int group) { return f32 ? kRowsF32 : group % 2 ? 64 : 32; }

// Partial sums of cut walks at most (per call); longer chunks where they would come to more.
constexpr size_t kMaxPackedPartials = (size_t)256 << 20;

// Work items, heaviest first: a workgroup that starts late should be short.
//
// Query tiles: 128 rows (16 in fp32) of one sequence, or as many fewer as a
// tile has heads (packed_tile_heads), by the keys they walk.
//
// Key tiles: 128 keys (16), by the steps of their walks.  The longest walk,
// the first keys' of the longest sequence, sets the time when there are few;
// walks longer than the average load of a CU's workgroups are cut into chunks of
// that load as in split_plan.hpp, whose reasons and limits hold here too (fp32:
// the whole load, not a quarter of it: 5 texts of 33 to 407 rows, 8/2 heads, d 64
// 46 -> 43 us, of which the sums 10 -> 5; bf16, 8K of documents: 0.5, 0.75, 1 and
// 1.5 loads 263, 252, 245 and 261 us).
inline PackedPlanItems packed_items(const bdlm_packed& p, int64_t n, const bdlm_packed_seq* seqs) {
  PackedPlanItems out;
  const bool f32 = p.dtype == BDLM_F32;
  const int M = (int)p.block_size, group = p.heads / p.kv_heads;
  const int tile_heads = f32 ? 1 : packed_tile_heads(group);
  const int q_tile = f32 ? kRowsF32 : kQRowsShortBf16 / tile_heads, k_tile = f32 ? kRowsF32 : kBwdKeysBf16;
  const int step = packed_step_rows(f32, group);
  const int64_t per_block = f32 || group % 2 ? group : group / 2;
  const MaskRule rule{M, kIntraBlock, (int)p.window, 1, kBig, nullptr};

  struct Cost {
    int64_t cost;
    PackedItem it;
  };
  std::vector<Cost> q, k;
  int64_t total = 0;
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
      q.push_back({std::max(0, std::min(hi1, shift + kl) - std::max(lo, shift)), it});
    }
    for (int t = 0; t * (int64_t)k_tile < kl; ++t) {
      const int first = t * k_tile, last = std::min(kl, first + k_tile) - 1;
      int lo, hi, lo1, hi1;
      query_interval(kClean, kClean, shift + first, rule, lo, hi);
      query_interval(kClean, kClean, shift + last, rule, lo1, hi1);
      const int u0 = std::max(lo - qp, 0), u1 = std::min(hi1 - qp, ql);
      const int64_t steps = u1 > u0 ? ((u1 + step - 1) / step - u0 / step) * per_block : 0;
      it.tile = t;
      k.push_back({steps, it});
      total += steps * p.kv_heads;
    }
  }
  auto heavier = [](const Cost& a, const Cost& b) { return a.cost > b.cost; };
  std::stable_sort(q.begin(), q.end(), heavier);
  std::stable_sort(k.begin(), k.end(), heavier);
  for (const Cost& c : q) out.q.push_back(c.it);
  if (!f32 && (int64_t)out.q.size() * (p.heads / tile_heads) <= kTeamWgs) out.teams = 2;

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
    if (nch > 1) out.sums.push_back({it.k0, it.k_len, it.tile, out.slots, (int32_t)nch, 0, 0, 0});
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
