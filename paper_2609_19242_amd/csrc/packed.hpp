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

}  // namespace bdlm
