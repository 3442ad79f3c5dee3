// Packed attention: sequences of different lengths in one call, each causal by
// blocks of M tokens (M = 1: by token), optionally within a window.
//
// The tile kernels (fwd_*, bwd_dq, bwd_dkdv, bwd_f32) take their call as a
// template parameter.  For packed calls that is PackedArgs: a workgroup reads
// its work item from the plan that the host laid out once for the lengths, and
// runs the item's sequence as a problem of one query and one key range
// (PackedView), with the clean-to-clean rules of common.hpp.
//
// What bounds them is what bounds the joint calls.  Measured, 32/8 heads: 30K
// rows of prompts with up to 9K earlier keys, d 128, forward 4.29 ms (1,115
// TFLOP/s); 11 documents of 130 to 2,500 rows, forward 133 us (860), dQ 187 (920
// with what it forms again), dK/dV 240 (955) and 5 for the sums; 48 prompts of up to
// 2,013 rows at d 64 139 us (the vector units 88% busy).
#pragma once

#include "common.hpp"

namespace bdlm {

// A work item: a tile of query rows, or a chunk of its walk (bf16; key tiles
// [n0, n1) of those it sees), or a chunk of the walk of a tile of keys (dK/dV;
// steps [n0, n1)).  slot >= 0: where its partial sums go.
// Sequence: rows [q0, q0 + q_len) of the queries, [k0, k0 + k_len) of the keys.
struct PackedItem {
  int32_t q0, q_len, k0, k_len, tile, n0, n1, slot;
};
// A tile whose walk was cut (row0, len: its sequence's rows):
// its partial sums in slots [slot, slot + n).
struct PackedSum {
  int32_t row0, len, tile, slot, n, pad0, pad1, pad2;
};

struct PackedArgs {
  const PackedItem* items;
  const PackedSum* sums;
  int32_t n_items, n_sums;
  int32_t heads, kv_heads, group, M, window;
  float scale, scale_log2;
  int32_t q_rows;      // rows of the query tensors: the pitch of the LSE and of the row statistics
  int32_t stats_form;  // as AttnArgs::stats_form
  int32_t qs, ks, vs, os, dos, dqs, dks, dvs;  // elements between rows
  const void *q, *k, *v, *dO;
  void *o, *dq, *dk, *dv;
  float *lse, *l2, *delta;
  void* partials;
  float* part_lse;     // forward: log2-sum-exp of each partial row
  int32_t sinks;       // with a window: first keys that stay visible (0: none, and without a window)
};

// Positions start at a multiple of M that leaves room for query rows before
// the first key (q_len > k_len), which see nothing.
__host__ __device__ inline int packed_shift(int q_len, int k_len, int M) {
  const int d = q_len - k_len;
  return d <= 0 ? 0 : (d + M - 1) / M * M;
}

// Query heads of a KV head that the four waves of a bf16 forward or dQ tile
// take side by side: the tile is then 128 / heads rows of each.  They read the
// same keys as 128 rows of one head would, but the rows' causal ends lie closer
// together, so fewer pairs are computed in vain and the waves end together.
inline int packed_tile_heads(int group) { return group % 4 == 0 ? 4 : group % 2 == 0 ? 2 : 1; }

// One sequence of a packed call, with the members of AttnArgs that the kernels read.
struct PackedView {
  static constexpr int n_q = 1, n_k = 1, batch = 1, out_f32 = 0, hilo = 0;
  static constexpr float hilo_tau = 0.f;
  int32_t heads, kv_heads, group, stats_form;
  MaskRule rule;
  float scale, scale_log2;
  int64_t qs, ks, vs, os, dos, dqs, dks, dvs;
  QRangeArg qr[1];
  KRangeArg kr[1];
};

__device__ __forceinline__ PackedView packed_view(const PackedArgs& p, const PackedItem& it, int elem) {
  PackedView a;
  a.heads = p.heads;
  a.kv_heads = p.kv_heads;
  a.group = p.group;
  a.stats_form = p.stats_form;
  a.rule = MaskRule{p.M, kIntraBlock, p.window, 1, kBig, nullptr};
  a.scale = p.scale;
  a.scale_log2 = p.scale_log2;
  a.qs = p.qs;
  a.ks = p.ks;
  a.vs = p.vs;
  a.os = p.os;
  a.dos = p.dos;
  a.dqs = p.dqs;
  a.dks = p.dks;
  a.dvs = p.dvs;
  const int shift = packed_shift(it.q_len, it.k_len, p.M);
  const int64_t q0 = it.q0, k0 = it.k0;
  auto at = [&](const void* base, int64_t row, int32_t stride) {
    return (void*)((char*)const_cast<void*>(base) + row * stride * elem);
  };
  QRangeArg& qr = a.qr[0];
  qr = QRangeArg{};
  qr.stream = kClean;
  qr.pos0 = shift + it.k_len - it.q_len;
  qr.len = it.q_len;
  qr.bstride = p.q_rows;  // (batch element 0 only: the pitch of the LSE's heads)
  qr.q = at(p.q, q0, p.qs);
  qr.o = at(p.o, q0, p.os);
  qr.dO = at(p.dO, q0, p.dos);
  qr.dq = at(p.dq, q0, p.dqs);
  qr.lse = p.lse + q0;
  qr.l2 = p.l2 + q0 * p.heads;  // row statistics: [sequence][heads][rows]
  qr.delta = p.delta + q0 * p.heads;
  KRangeArg& kr = a.kr[0];
  kr = KRangeArg{};
  kr.stream = kClean;
  kr.pos0 = shift;
  kr.len = it.k_len;
  kr.k = at(p.k, k0, p.ks);
  kr.v = at(p.v, k0, p.vs);
  kr.dk = at(p.dk, k0, p.dks);
  kr.dv = at(p.dv, k0, p.dvs);
  return a;
}

__host__ __device__ inline MaskRule rule_of(const PackedView& a) { return a.rule; }

// ---- the two kinds of call, for the tile kernels.
// Elements between rows of each tensor, and the element of row `row` of batch
// element b of a range and its head h.
template <int D> __device__ __forceinline__ int64_t q_stride(const AttnArgs& a) { return (int64_t)a.heads * D; }
template <int D> __device__ __forceinline__ int64_t o_stride(const AttnArgs& a) { return (int64_t)a.heads * D; }
template <int D> __device__ __forceinline__ int64_t do_stride(const AttnArgs& a) { return (int64_t)a.heads * D; }
template <int D> __device__ __forceinline__ int64_t dq_stride(const AttnArgs& a) { return (int64_t)a.heads * D; }
template <int D> __device__ __forceinline__ int64_t k_stride(const AttnArgs& a) { return (int64_t)a.kv_heads * D; }
template <int D> __device__ __forceinline__ int64_t v_stride(const AttnArgs& a) { return (int64_t)a.kv_heads * D; }
template <int D> __device__ __forceinline__ int64_t dk_stride(const AttnArgs& a) { return (int64_t)a.kv_heads * D; }
template <int D> __device__ __forceinline__ int64_t dv_stride(const AttnArgs& a) { return (int64_t)a.kv_heads * D; }
template <int D> __device__ __forceinline__ int64_t q_stride(const PackedView& a) { return a.qs; }
template <int D> __device__ __forceinline__ int64_t o_stride(const PackedView& a) { return a.os; }
template <int D> __device__ __forceinline__ int64_t do_stride(const PackedView& a) { return a.dos; }
template <int D> __device__ __forceinline__ int64_t dq_stride(const PackedView& a) { return a.dqs; }
template <int D> __device__ __forceinline__ int64_t k_stride(const PackedView& a) { return a.ks; }
template <int D> __device__ __forceinline__ int64_t v_stride(const PackedView& a) { return a.vs; }
template <int D> __device__ __forceinline__ int64_t dk_stride(const PackedView& a) { return a.dks; }
template <int D> __device__ __forceinline__ int64_t dv_stride(const PackedView& a) { return a.dvs; }
template <int D>
__device__ __forceinline__ int64_t row_elem(const AttnArgs&, int b, int64_t bstride, int64_t row, int64_t heads, int h,
                                            int64_t) {
  return (((int64_t)b * bstride + row) * heads + h) * D;
}
template <int D>
__device__ __forceinline__ int64_t row_elem(const PackedView&, int, int64_t, int64_t row, int64_t, int h,
                                            int64_t stride) {
  return row * stride + h * D;
}

// ---- sinks: a window, and the first S keys of a sequence stay visible.
//
// A row sees the keys [0, min(S, e)) and [e - W, e).  A call with sinks is the same
// kernels over another view of the sequence (SinkQArgs, SinkQArgsF32, SinkKArgs):
//  * forward and dQ, bf16: a query tile's rows see [0, S) and [w0, end), w0 the first row's
//    window's start.  They are walked as [0, n) with the gap between taken out, in multiples
//    of 16 keys, so that a few sinks share the first tile with the window's first keys: v
//    < gap_at is key v, the others are key v + gap.  Keys that no row of the tile sees (at
//    most 15 before w0, and behind S) read as zeros.  (8 texts of 2,048, 32/8 heads, d 128,
//    window 128: without sinks forward 96 us, dQ 149, with 4 of them 97 and 157, and 115 and
//    170 with the sinks in a tile of their own.)
//  * the same, fp32: two key ranges, the sinks and the others.
//  * dK/dV: the sinks, which all rows from theirs on see, are keys of a call without a
//    window, the others of one without sinks: items of two kinds, tile -1 - t the
//    t-th of the sinks.  A tile of 4 keys costs as much as one of 128 (the same texts:
//    169 us without, 225 with them; 16K tokens of 3 documents, window 1,024: 633, 671).
struct SinkQArgs : PackedArgs {};
struct SinkDArgs : SinkQArgs {};  // D of rows of few keys alone (bwd_dq.hip)
struct SinkQArgsF32 : PackedArgs {};
struct SinkKArgs : PackedArgs {};

struct SinkWalk {
  int n, gap_at, gap, w0;
};
// The walk of the rows at positions [pq0, pq1] over len keys from position pos0 on.
__host__ __device__ inline SinkWalk sink_walk(const MaskRule& rule, int sinks, int pq0, int pq1, int pos0, int len) {
  int lo0, hi0, lo1, hi1;
  key_interval(kClean, pq0, kClean, rule, lo0, hi0);
  key_interval(kClean, pq1, kClean, rule, lo1, hi1);
  const int end = imin(hi1 - pos0, len);
  SinkWalk w{imax(end, 0), kBig, 0, imax(lo0 - pos0, 0)};
  const int below = (imin(sinks, w.n) + 15) & ~15, first = w.w0 & ~15;
  if (first > below) {
    w.gap_at = below;
    w.gap = first - below;
    w.w0 -= w.gap;
    w.n = end > first ? below + end - first : imin(below, w.n);  // (a block may end behind its window's start)
  }
  return w;
}

// Whether a row whose window lies apart from the sinks may see no more than n keys: all of the sinks, and of its window
// what is left of it where its block of M tokens ends behind the sequence.
__host__ __device__ inline bool may_see_few(int sinks, int window, int M, int n) {
  return window > 0 && (int64_t)sinks + (window > M - 1 ? window - (M - 1) : 0) <= n;
}

struct SinkView : PackedView {
  int32_t sinks;
};
__device__ __forceinline__ SinkView call_view(const SinkQArgs& p, int item, int elem) {
  const PackedItem& it = p.items[item];
  SinkView a;
  static_cast<PackedView&>(a) = packed_view(p, it, elem);
  a.sinks = imin(p.sinks, it.k_len);
  return a;
}

struct SinkViewF32 : PackedView {
  static constexpr int n_k = 2;
  int32_t sinks;             // the first range's keys
  int64_t k_ahead, v_ahead;  // bytes from a sequence's first key to the second range
};
__device__ __forceinline__ SinkViewF32 call_view(const SinkQArgsF32& p, int item, int elem) {
  const PackedItem& it = p.items[item];
  SinkViewF32 a;
  static_cast<PackedView&>(a) = packed_view(p, it, elem);
  a.sinks = imin(p.sinks, it.k_len);
  a.k_ahead = (int64_t)a.sinks * p.ks * elem;
  a.v_ahead = (int64_t)a.sinks * p.vs * elem;
  a.kr[0].len = a.sinks;
  a.kr[0].ntiles = it.k_len;
  return a;
}
__device__ __forceinline__ KRangeArg k_range(const SinkViewF32& a, int j) {
  KRangeArg r = a.kr[0];
  if (j > 0) {
    r.pos0 += a.sinks;
    r.len = r.ntiles - a.sinks;
    r.k = (const char*)r.k + a.k_ahead;
    r.v = (const char*)r.v + a.v_ahead;
  }
  return r;
}

__device__ __forceinline__ PackedView call_view(const SinkKArgs& p, int item, int elem) {
  const PackedItem& it = p.items[item];
  PackedView a = packed_view(p, it, elem);
  const int S = imin(p.sinks, it.k_len);
  KRangeArg& kr = a.kr[0];
  if (it.tile < 0) {
    a.rule.window = 0;
    kr.len = S;
  } else {
    kr.pos0 += S;
    kr.len -= S;
    auto on = [&](const void* x, int32_t stride) { return (void*)((char*)const_cast<void*>(x) + (int64_t)S * stride * elem); };
    kr.k = on(kr.k, p.ks);
    kr.v = on(kr.v, p.vs);
    kr.dk = on(kr.dk, p.dks);
    kr.dv = on(kr.dv, p.dvs);
  }
  return a;
}

// Query and key ranges by number; a packed sequence has one of each (indexed by
// a variable, its copy would live in scratch memory).
__device__ __forceinline__ const QRangeArg& q_range(const AttnArgs& a, int i) { return a.qr[i]; }
__device__ __forceinline__ const KRangeArg& k_range(const AttnArgs& a, int j) { return a.kr[j]; }
__device__ __forceinline__ const QRangeArg& q_range(const PackedView& a, int) { return a.qr[0]; }
__device__ __forceinline__ const KRangeArg& k_range(const PackedView& a, int) { return a.kr[0]; }

// What a kernel reads its call through: the arguments themselves, or the sequence of a packed item.
__device__ __forceinline__ const AttnArgs& call_view(const AttnArgs& a, int, int) { return a; }
__device__ __forceinline__ PackedView call_view(const PackedArgs& a, int item, int elem) {
  return packed_view(a, a.items[item], elem);
}
template <class A> constexpr bool kIsPacked = false;
template <> constexpr inline bool kIsPacked<PackedArgs> = true;
template <> constexpr inline bool kIsPacked<PackedView> = true;
template <> constexpr inline bool kIsPacked<SinkQArgs> = true;
template <> constexpr inline bool kIsPacked<SinkDArgs> = true;
template <> constexpr inline bool kIsPacked<SinkQArgsF32> = true;
template <> constexpr inline bool kIsPacked<SinkKArgs> = true;
template <class A> constexpr bool kHasSinks = false;
template <> constexpr inline bool kHasSinks<SinkQArgs> = true;
template <> constexpr inline bool kHasSinks<SinkDArgs> = true;
template <class A> constexpr bool kFormsD = false;
template <> constexpr inline bool kFormsD<SinkDArgs> = true;

hipError_t launch_fwd_bf16(const PackedArgs& a, int head_dim, int teams, hipStream_t s);
hipError_t launch_packed_fwd_sum(const PackedArgs& a, int head_dim, int slots, hipStream_t s);
hipError_t launch_packed_dq_sum(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_fwd_f32(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dq_bf16(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dkdv(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dkdv_sum(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dq_f32(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dkv_f32(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_sum_f32(const PackedArgs& a, int head_dim, hipStream_t s);
hipError_t launch_fwd_bf16(const SinkQArgs& a, int head_dim, int teams, hipStream_t s);
hipError_t launch_fwd_f32(const SinkQArgsF32& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dq_bf16(const SinkQArgs& a, int head_dim, hipStream_t s);  // (two kernels where rows may see few keys)
hipError_t launch_bwd_dkdv(const SinkKArgs& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dq_f32(const SinkQArgsF32& a, int head_dim, hipStream_t s);
hipError_t launch_bwd_dkv_f32(const SinkKArgs& a, int head_dim, hipStream_t s);

}  // namespace bdlm
