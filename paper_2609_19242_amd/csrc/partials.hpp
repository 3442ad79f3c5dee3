// Partial outputs of attention over disjoint sets of keys, joined: with z_j the
// log2-sum-exp of part j of a row and O_j its normalised output,
//   m = max z_j,  w_j = 2^(z_j - m),  O = sum w_j O_j / sum w_j,
//   LSE = ln 2 (m + log2 sum w_j)
// in fp32, in an order that depends on the number of parts only.  A wave per
// row: D / 4 lanes hold 16 bytes each of one part's output, the wave takes
// 256 / D parts at a time, four such rounds in flight.  Parts that a row does
// not see (z_j = -inf) have left no output; what lies there takes no part.
#pragma once

#include "common.hpp"
#include "device.hpp"

namespace bdlm {

template <int D>
struct JoinedRow {
  static constexpr int LPR = D / 4;  // lanes per part
  f32x4 x;   // this lane's columns 4 (lane % LPR) .. + 3, in the lanes < LPR
  float lse;
};

// at(j): row of part j in `o` ([row][D]) and `z`.
template <int D, class At>
__device__ __forceinline__ JoinedRow<D> join_partials(const float* o, const float* z, At at, int parts, int lane) {
  constexpr int LPR = JoinedRow<D>::LPR, PP = 64 / LPR;  // lanes per part, parts at a time
  const int part = lane / LPR, col = lane % LPR;
  float m = -INFINITY;
  for (int j = lane; j < parts; j += 64) m = fmaxf(m, z[at(j)]);
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
  const float ref = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = part; j0 < parts; j0 += 4 * PP) {
    float zz[4];
    f32x4 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t row = at(imin(j0 + k * PP, parts - 1));
      zz[k] = z[row];
      p[k] = *(const f32x4*)(o + row * D + col * 4);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bool seen = j0 + k * PP < parts && zz[k] > -INFINITY;
      const float w = seen ? exp2f_fast(zz[k] - ref) : 0.f;
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
  JoinedRow<D> r;
  r.x = x * (sum > 0.f ? 1.f / sum : 0.f);
  r.lse = sum > 0.f ? (m + log2f(sum)) * 0.69314718055994530942f : -INFINITY;
  return r;
}

}  // namespace bdlm
