// The chunks' partial outputs of a packed bf16 forward (packed_plan.hpp says
// which walks are cut) joined (partials.hpp), gfx950: a wave per row of a cut
// tile and head.  Bound by its launch and by reading the partial outputs, 64 KB per
// chunk of 128 rows at d 128.
#include "packed.hpp"
#include "partials.hpp"

namespace bdlm {

namespace {

template <int D>
__global__ __launch_bounds__(256) void packed_fwd_sum_kernel(const PackedArgs a, const int tile_heads) {
  // workgroup: four rows of the 128 that a tile's waves hold, of its heads side by side
  const int per = a.heads / tile_heads;
  const int quad = blockIdx.x & 31, rest = blockIdx.x >> 5, n = rest / per, hg = rest - n * per;
  const int lane = threadIdx.x & 63, r = quad * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PackedSum& s = a.sums[n];
  const int w = r >> 5, row = s.tile * (kQRowsShortBf16 / tile_heads) + w / tile_heads * 32 + (r & 31);
  if (row >= s.len) return;
  const int head = hg * tile_heads + w % tile_heads;
  const int64_t first = ((int64_t)s.slot * per + hg) * kQRowsShortBf16 + r, step = (int64_t)per * kQRowsShortBf16;
  const JoinedRow<D> x =
      join_partials<D>((const float*)a.partials, a.part_lse, [&](int j) { return first + j * step; }, s.n, lane);
  if (lane >= JoinedRow<D>::LPR) return;
  bf16x4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = to_bf16(x.x[e]);
  *(bf16x4*)((bf16*)a.o + ((int64_t)s.row0 + row) * a.os + (int64_t)head * D + lane * 4) = y;
  if (lane == 0) a.lse[(int64_t)head * a.q_rows + s.row0 + row] = x.lse;
}

}  // namespace

hipError_t launch_packed_fwd_sum(const PackedArgs& a, int head_dim, hipStream_t s) {
  const int heads = packed_tile_heads(a.group);
  const dim3 grid((unsigned)(a.n_sums * (a.heads / heads) * 32)), threads(256);
  if (head_dim == 128) hipLaunchKernelGGL((packed_fwd_sum_kernel<128>), grid, threads, 0, s, a, heads);
  else hipLaunchKernelGGL((packed_fwd_sum_kernel<64>), grid, threads, 0, s, a, heads);
  return hipGetLastError();
}

}  // namespace bdlm
