// The chunks' partial sums of query tiles whose walks were cut (packed_plan.hpp
// says which), gfx950: the forward's outputs joined (partials.hpp); dQ's shares added in the chunks' order, D / 4 lanes per row and
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

template <int D, bool FEW>
__global__ __launch_bounds__(256) void packed_fwd_sum_kernel(const PackedArgs a, const int tile_heads) {
  constexpr int LPR = JoinedRow<D>::LPR, ROWS = FEW ? 256 / LPR : 4, WGS = kQRowsShortBf16 / ROWS;
  const int lane = FEW ? threadIdx.x % LPR : threadIdx.x & 63;
  const int item = blockIdx.x / WGS, r = (blockIdx.x - item * WGS) * ROWS +
                                         (FEW ? (int)threadIdx.x / LPR : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
  const CutRow c = cut_row(a, tile_heads, item, r);
  if (c.row < 0) return;
  auto at = [&](int j) { return c.first + j * c.step; };
  const float* const o = (const float*)a.partials;
  const JoinedRow<D> x = FEW ? join_few<D>(o, a.part_lse, at, c.n, lane) : join_partials<D>(o, a.part_lse, at, c.n, lane);
  if (lane >= LPR) return;
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

template <int D>
void launch_fwd_sum(const PackedArgs& a, bool few, hipStream_t s) {
  const int heads = packed_tile_heads(a.group), n = a.n_sums * (a.heads / heads);
  const dim3 grid((unsigned)(n * (kQRowsShortBf16 / (few ? 256 / JoinedRow<D>::LPR : 4)))), threads(256);
  if (few) hipLaunchKernelGGL((packed_fwd_sum_kernel<D, true>), grid, threads, 0, s, a, heads);
  else hipLaunchKernelGGL((packed_fwd_sum_kernel<D, false>), grid, threads, 0, s, a, heads);
}

}  // namespace

// slots: of all cut tiles together
hipError_t launch_packed_fwd_sum(const PackedArgs& a, int head_dim, int slots, hipStream_t s) {
  const bool few = slots <= (int64_t)a.n_sums * kFewParts;
  head_dim == 128 ? launch_fwd_sum<128>(a, few, s) : launch_fwd_sum<64>(a, few, s);
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
