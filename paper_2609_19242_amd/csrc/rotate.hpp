// Norms of queries and keys for each head with the position rotation
// (rotate.hip), as the C ABI layer calls them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bdlm {

constexpr int kMaxPairs = 64, kMaxAxes = 4;
constexpr int kRotateWaves = 4;   // of a workgroup
constexpr int kRotateChain = 64;  // products to a weight's gradient that a lane adds up in fp32

struct RotateTensor {
  const void *x, *dy, *w;  // rows; the outputs' gradients; the weight, or null
  void *out;               // y, or dx
  int64_t xs, dys, outs;   // elements between rows
  int32_t heads, passes;   // heads; passes of a wave's heads over them
};

// A wave takes `rows_per` rows (a power of two) at a time, with 64 / (D / 16) /
// rows_per of their heads side by side, and those heads' passes dealt out to
// `split` waves.
struct RotateArgs {
  RotateTensor t[2];  // queries, keys
  const int32_t* pos;  // [axes][rows]
  int64_t rows;
  double eps;
  float* partials;     // backward: [workgroup][2][D] sums of the weights' gradients
  float* dw[2];
  int32_t axes, dim, rows_per, split, wgs;
  int64_t chain;       // passes over a tensor's heads that a wave makes, at most
  double quarters[kMaxPairs];  // quarter turns per position
  int8_t axis[kMaxPairs];      // (the launch's time grows with its arguments' size)
};

hipError_t launch_rotate_fwd(const RotateArgs& a, int head_dim, int bf16, int interleaved, hipStream_t s);
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, int bf16, int interleaved, hipStream_t s);

}  // namespace bdlm
