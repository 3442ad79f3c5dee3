// The chunks' partial sums of query tiles whose walks were cut (packed_plan.hpp
// says which), gfx950: the forward's outputs joined (partials.hpp), a wave per
// row and head; dQ's shares added in the chunks' order, D / 4 lanes per row and
// head.  Bound by the launch and by reading, 64 KB per chunk of 128 rows at d 128.
#include "packed.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

// Row r of the 128 that the four waves of a cut tile hold, of its heads side by side.
struct CutRow {
  int row, head, n;     // in the sequence (past its last: nothing to do); parts
  int64_t token;        // in the call's tensors
  int64_t first, step;  // partial rows: first + j step
};
__device__ __forceinline__ CutRow cut_row(const PackedArgs& a, int tile_heads, int item, int r) {
  const int per = a.heads / tile_heads, n = item / per, hg = item - n * per, w = r >> 5;
  const PackedSum& s = a.sums[n];
  CutRow x;
  x.row = s.tile * (kQRowsShortBf16 / tile_heads) + w / tile_heads * 32 + (r & 31);
  if (x.row >= s.len) x.row = -1;
  x.head = hg * tile_heads + w % tile_heads;
  x.n = s.n;
  x.token = (int64_t)s.row0 + x.row;
  x.first = ((int64_t)s.slot * per + hg) * kQRowsShortBf16 + r;
  x.step = (int64_t)per * kQRowsShortBf16;
  return x;
}

template <int D>
__global__ __launch_bounds__(256) void packed_fwd_sum_kernel(const PackedArgs a, const int tile_heads) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const CutRow c = cut_row(a, tile_heads, blockIdx.x >> 5, (blockIdx.x & 31) * 4 + w);
  if (c.row < 0) return;
  const JoinedRow<D> x = join_partials<D>((const float*)a.partials, a.part_lse,
                                          [&](int j) { return c.first + j * c.step; }, c.n, lane);
  if (lane >= JoinedRow<D>::LPR) return;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = to_bf16(x.x[e]);
  *(bf16x4*)((bf16*)a.o + c.token * a.os + (int64_t)c.head * D + lane * 4) = y;
  if (lane == 0) a.lse[(int64_t)c.head * a.q_rows + c.token] = x.lse;
}

template <int D>
__global__ __launch_bounds__(256) void packed_dq_sum_kernel(const PackedArgs a, const int tile_heads) {
  constexpr int LPR = D / 4, ROWS = 256 / LPR, WGS = kQRowsShortBf16 / ROWS;  // lanes per row, rows and groups of them
  const int item = blockIdx.x / WGS, r = (blockIdx.x - item * WGS) * ROWS + threadIdx.x / LPR;
  const CutRow c = cut_row(a, tile_heads, item, r);
  if (c.row < 0) return;
  const int col = threadIdx.x % LPR * 4;
  const float* p = (const float*)a.partials + c.first * D + col;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < c.n; j0 += 4) {
    f32x4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = *(const f32x4*)(p + imin(j0 + k, c.n - 1) * c.step * D);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (j0 + k < c.n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += v[k][e];
      }
  }
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = to_bf16(x[e]);
  *(bf16x4*)((bf16*)a.dq + c.token * a.dqs + (int64_t)c.head * D + col) = y;
}

}  // namespace

hipError_t launch_packed_fwd_sum(const PackedArgs& a, int head_dim, hipStream_t s) {
  const int heads = packed_tile_heads(a.group);
  const dim3 grid((unsigned)(a.n_sums * (a.heads / heads) * 32)), threads(256);
  if (head_dim == 128) hipLaunchKernelGGL((packed_fwd_sum_kernel<128>), grid, threads, 0, s, a, heads);
  else hipLaunchKernelGGL((packed_fwd_sum_kernel<64>), grid, threads, 0, s, a, heads);
  return hipGetLastError();
}

hipError_t launch_packed_dq_sum(const PackedArgs& a, int head_dim, hipStream_t s) {
  const int heads = packed_tile_heads(a.group), n = a.n_sums * (a.heads / heads);
  const dim3 threads(256);
  if (head_dim == 128) hipLaunchKernelGGL((packed_dq_sum_kernel<128>), dim3(n * 16), threads, 0, s, a, heads);
  else hipLaunchKernelGGL((packed_dq_sum_kernel<64>), dim3(n * 8), threads, 0, s, a, heads);
  return hipGetLastError();
}

}  // namespace bdlm
