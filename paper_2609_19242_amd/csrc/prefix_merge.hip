// The chunks' partial outputs of attention over a paged cache (cache.hpp)
// added up, gfx950: with z_j the log2-sum-exp of chunk j of a row,
//   m = max z_j,  w_j = 2^(z_j - m),  O = sum w_j O_j / sum w_j,
//   LSE = ln 2 (m + log2 sum w_j)
// in fp32, in an order that depends on the number of chunks only.  A wave per
// row: D / 4 lanes hold 16 bytes each of one chunk's output, the wave takes
// 256 / D chunks at a time, four such rounds in flight.  Chunks that a row does
// not see (z_j = -inf) have left no output; what lies there takes no part.
// Bound by reading the partials (16,384 rows of 128, 4 chunks: 10.7 us, 3.9 TB/s;
// 2,048 rows, up to 10 chunks: 4.8 us).
#include "cache.hpp"
#include "device.hpp"

namespace bdlm {

namespace {

constexpr float kLn2 = 0.69314718055994530942f;

template <int D, bool BF16>
__global__ __launch_bounds__(256) void prefix_merge_kernel(const PrefixArgs a) {
  constexpr int LPR = D / 4, PP = 64 / LPR;  // lanes per chunk, chunks at a time
  const int lane = threadIdx.x & 63, part = lane / LPR, col = lane % LPR;
  const int64_t total = (int64_t)a.requests * a.rows * a.heads;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= total) return;
  const int parts = a.prefix_chunks + a.own_chunks;
  float m = -INFINITY;
  for (int j = lane; j < parts; j += 64) m = fmaxf(m, a.part_lse[j * total + row]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float ref = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = part; j0 < parts; j0 += 4 * PP) {
    float z[4];
    f32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t at = imin(j0 + k * PP, parts - 1) * total + row;
      z[k] = a.part_lse[at];
      p[k] = *(const f32x4*)(a.part_o + at * D + col * 4);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool seen = j0 + k * PP < parts && z[k] > -INFINITY;
      const float w = seen ? exp2f_fast(z[k] - ref) : 0.f;
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = seen ? fmaf(w, p[k][e], x[e]) : x[e];
    }
  }
#pragma unroll
  for (int s = LPR; s < 64; s <<= 1) {
    sum += __shfl_xor(sum, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], s);
  }
  if (part != 0) return;
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  if constexpr (BF16) {
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = to_bf16(x[e] * inv);
    *(bf16x4*)((bf16*)a.o + row * D + col * 4) = y;
  } else {
    *(f32x4*)((float*)a.o + row * D + col * 4) = x * inv;
  }
  if (lane == 0) {
    PrefixRow pr;
    pr.token = (int)(row / a.heads);
    pr.head = (int)(row - (int64_t)pr.token * a.heads);
    pr.end = 0;
    a.lse[prefix_lse_at(a, pr)] = sum > 0.f ? (m + log2f(sum)) * kLn2 : -INFINITY;
  }
}

}  // namespace

hipError_t launch_prefix_merge(const PrefixArgs& a, int head_dim, int is_bf16, hipStream_t s) {
  const int64_t rows = (int64_t)a.requests * a.rows * a.heads;
  const dim3 grid((unsigned)((rows + 3) / 4)), threads(256);
  if (rows == 0) return hipSuccess;
  if (head_dim == 128) {
    if (is_bf16) hipLaunchKernelGGL((prefix_merge_kernel<128, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((prefix_merge_kernel<128, false>), grid, threads, 0, s, a);
  } else {
    if (is_bf16) hipLaunchKernelGGL((prefix_merge_kernel<64, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((prefix_merge_kernel<64, false>), grid, threads, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace bdlm
