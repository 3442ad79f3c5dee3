// Norms of queries and keys for each head with the position rotation in the
// same pass, forward and backward, bf16 and fp32, gfx950.
//
// For a head's row x of D elements with weight w, at positions p_a, with pair i
// of the first `dim` elements on axis a(i) turning by t_i = p_a(i) f_i:
//   r = 1 / sqrt(mean x^2 + eps),  n = x r w  (no norm: n = x),
//   y = n, its pairs (n1, n2) turned to (n1 cos t - n2 sin t, n2 cos t + n1 sin t).
// Backward, with g = dy turned by -t and h = g w:
//   dw = sum over rows and heads of g x r,  dx = r (h - x r mean(h x r)).
// r is formed again from x, which backward reads in any case: nothing is saved.
//
// Bound by memory.  D / 16 lanes hold a head's row, 16 elements each in two runs
// of 8 (16 bytes in bf16): pair partners lie in the same lane (halves D / 2
// apart, or neighbours), so that the rotation needs no exchange, and a pass of a
// wave reads whole 128-byte lines.  A lane forms its 8 cosines and sines once per
// row, under the loads of its first pass, and keeps them for all passes over the
// row's heads; each pass's loads are issued before the pass in front is computed
// (backward, 16,384 rows of 32/8 heads, d 128: 141 -> 121 us).
// Measured, bf16: 30,011 rows of 32/8 heads, d 128, 115 us (5.3 TB/s, a copy's rate);
// 16,384 rows forward 60 us, backward 113 (4.5 TB/s; two waves per SIMD, for the 32
// sums of the weights' gradients that a lane keeps); 8,190 rows of 16/16 heads, d 64, 14
// and 24 us; 64 rows 5 us, the launch and one row's chain of loads.  fp32: 16,384 rows
// forward 130 us, backward with the weights' sums 196 (5.2 TB/s).
//
// Rounding.  An angle is position times frequency in 64 bits, in quarter turns,
// reduced there to half a quarter; sine and cosine of the rest in fp32 by their
// Taylor series to x^9 and x^10 (|x| <= pi / 4: the rest of the series is below
// 2^-28).  bf16: the sum of squares and all products are fp32 (so squares must stay
// below 2^127: |x|, |g w| < 2^60), the outputs are rounded once.  fp32: the sums over a row
// are fp64.  dw: a lane adds up to 64 products in fp32 and those sums in fp64 (in LDS, for which it
// has no registers; calls whose chains cannot be longer run without: 8,190 rows of 16/16 heads, d 64, with the weights'
// sums 28.3 us, with that LDS 28.9), a wave's and a workgroup's lanes are added in fp32 in a fixed order, the workgroups' in fp64; it is returned in fp32.
#include "device.hpp"
#include "rotate.hpp"

namespace bdlm {

namespace {

constexpr int kWaves = kRotateWaves;

// 8 consecutive elements, as they lie in memory.
template <class T> struct Raw8;
template <> struct Raw8<bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *(const bf16x8*)p; }
  __device__ __forceinline__ float operator[](int e) const { return (float)v[e]; }
};
template <> struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p, b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ float operator[](int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
};
__device__ __forceinline__ void store8(bf16* p, const float (&x)[8]) {
  bf16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = to_bf16(x[e]);
  *(bf16x8*)p = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// The type of sums over a head's row.
template <class T> struct SumOf { typedef float type; };
template <> struct SumOf<float> { typedef double type; };

__device__ __forceinline__ float shfl_x(float x, int m) { return __shfl_xor(x, m); }
__device__ __forceinline__ double shfl_x(double x, int m) { return __shfl_xor(x, m); }
template <int LPR, class S>
__device__ __forceinline__ S row_sum(S x) {
#pragma unroll
  for (int m = 1; m < LPR; m <<= 1) x += shfl_x(x, m);
  return x;
}

__device__ __forceinline__ float inverse_root(float x) { return __builtin_amdgcn_rsqf(x); }
__device__ __forceinline__ float inverse_root(double x) { return (float)(1.0 / sqrt(x)); }

// Cosine and sine of `u` quarter turns.
__device__ __forceinline__ void turn_of(double u, float& c, float& s) {
  const double n = __builtin_rint(u);
  const float x = (float)(u - n) * 1.57079632679489661923f, x2 = x * x;
  const float sn = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const int q = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const float a = q & 1 ? sn : cs, b = q & 1 ? cs : sn;
  c = (q + 1) & 2 ? -a : a;
  s = q & 2 ? -b : b;
}

// Where a lane's two runs of 8 elements lie in a head's row.
template <bool IL>
__device__ __forceinline__ void runs_of(int l, int dim, int& a, int& b) {
  const bool halves = !IL && 16 * l < dim;
  a = halves ? 8 * l : 16 * l;
  b = halves ? dim / 2 + 8 * l : 16 * l + 8;
}

// The lane's pairs turned (by -t: `back`).
template <bool IL>
__device__ __forceinline__ void turn(float (&a)[8], float (&b)[8], const float (&c)[8], const float (&s)[8], bool back) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float& x = IL ? (j < 4 ? a[2 * j] : b[2 * j - 8]) : a[j];
    float& y = IL ? (j < 4 ? a[2 * j + 1] : b[2 * j - 7]) : b[j];
    const float sn = back ? -s[j] : s[j], u = x, v = y;
    x = fmaf(u, c[j], -(v * sn));
    y = fmaf(v, c[j], u * sn);
  }
}

// What a lane knows of the wave's rows: its row's cosines and sines.
template <int D, bool IL>
struct Lane {
  static constexpr int LPR = D / 16, HPG = 64 / LPR;
  int l, ra, rb, sub, head, heads;  // lane of its head's row; runs; row of the wave's; first head, heads side by side
  int64_t row;
  bool ok;
  float c[8], s[8];
  __device__ __forceinline__ Lane(const RotateArgs& a, int lane) {
    l = lane % LPR;
    runs_of<IL>(l, a.dim, ra, rb);
    heads = HPG / a.rows_per;
    sub = lane / LPR / heads;
    head = lane / LPR % heads;
  }
  __device__ __forceinline__ void seek(const RotateArgs& a, int64_t set) {
    row = set * a.rows_per + sub;
    ok = row < a.rows;
    if (!ok) row = a.rows - 1;
  }
  __device__ __forceinline__ void angles(const RotateArgs& a) {
    if (16 * l < a.dim) {
      if (a.axes == 1) {
        const double p = (double)a.pos[row];
#pragma unroll
        for (int j = 0; j < 8; ++j) turn_of(p * a.quarters[8 * l + j], c[j], s[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          turn_of((double)a.pos[a.axis[8 * l + j] * a.rows + row] * a.quarters[8 * l + j], c[j], s[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 1.f, s[j] = 0.f;
    }
  }
};

// A lane's elements of a head's row.
template <class T>
struct Piece {
  Raw8<T> a, b;
  __device__ __forceinline__ void load(const void* base, int64_t at, int ra, int rb) {
    a.load((const T*)base + at + ra);
    b.load((const T*)base + at + rb);
  }
};
template <class T>
__device__ __forceinline__ void load_weight(Piece<T>& w, const RotateTensor& t, int ra, int rb) {
  if (t.w) {
    w.load(t.w, 0, ra, rb);
  } else {
    float one[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    T ones[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (T)one[e];
    w.a.load(ones);
    w.b.load(ones);
  }
}

// The passes of a wave over a row's heads, of both tensors: the keys' follow the queries' in the deal.
__device__ __forceinline__ int first_pass(const RotateArgs& a, int i, int part) {
  return i == 0 ? part : (part - a.t[0].passes % a.split + a.split) % a.split;
}

template <class T, int D, bool IL, bool NORM>
__global__ __launch_bounds__(kWaves * 64) void rotate_fwd_kernel(const RotateArgs a) {
  using S = typename SumOf<T>::type;
  const int lane = threadIdx.x & 63;
  Lane<D, IL> me(a, lane);
  const int64_t sets = (a.rows + a.rows_per - 1) / a.rows_per;
  const int64_t first = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t n = first; n < sets * a.split; n += (int64_t)gridDim.x * kWaves) {
    const int64_t set = n / a.split;
    const int part = (int)(n - set * a.split);
    me.seek(a, set);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const RotateTensor& t = a.t[i];
      auto head_of = [&](int p) __attribute__((always_inline)) {  // (a lane without one reads the first)
        const int h = p * me.heads + me.head;
        return (int64_t)(me.ok && h < t.heads ? h : 0) * D;
      };
      Piece<T> w, x, next;
      int p = first_pass(a, i, part);
      if (p < t.passes) x.load(t.x, me.row * t.xs + head_of(p), me.ra, me.rb);
      if constexpr (NORM) load_weight<T>(w, t, me.ra, me.rb);
      if (i == 0) me.angles(a);  // (under the first loads)
      for (; p < t.passes; p += a.split) {
        const int after = p + a.split;
        if (after < t.passes) next.load(t.x, me.row * t.xs + head_of(after), me.ra, me.rb);
        float u[8], v[8];
        float r = 1.f;
        if constexpr (NORM) {
          S ss = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) ss += (S)x.a[e] * (S)x.a[e] + (S)x.b[e] * (S)x.b[e];
          ss = row_sum<D / 16>(ss);
          r = inverse_root(ss * (S)(1.0 / D) + (S)a.eps);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = NORM ? x.a[e] * r * w.a[e] : x.a[e];
          v[e] = NORM ? x.b[e] * r * w.b[e] : x.b[e];
        }
        turn<IL>(u, v, me.c, me.s, false);
        if (me.ok && p * me.heads + me.head < t.heads) {
          T* o = (T*)t.out + me.row * t.outs + head_of(p);
          store8(o + me.ra, u);
          store8(o + me.rb, v);
        }
        x = next;
      }
    }
  }
}

// LONG: some lane may add up more than kRotateChain products to a weight's gradient.
template <class T, int D, bool IL, bool NORM, bool LONG>
__global__ __launch_bounds__(kWaves * 64) void rotate_bwd_kernel(const RotateArgs a) {
  using S = typename SumOf<T>::type;
  constexpr int LPR = D / 16;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Lane<D, IL> me(a, lane);
  const int64_t sets = (a.rows + a.rows_per - 1) / a.rows_per;
  float dw[2][16];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f;
  // this lane's longer sums, and whether there are some (of the wave's, as the chains' lengths)
  [[maybe_unused]] __shared__ double far[LONG ? kWaves : 1][32][64];
  [[maybe_unused]] int chain[2] = {0, 0};
  [[maybe_unused]] bool have_far[2] = {false, false};
  for (int64_t n = (int64_t)blockIdx.x * kWaves + w; n < sets * a.split; n += (int64_t)gridDim.x * kWaves) {
    const int64_t set = n / a.split;
    const int part = (int)(n - set * a.split);
    me.seek(a, set);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const RotateTensor& t = a.t[i];
      auto head_of = [&](int p) __attribute__((always_inline)) {
        const int h = p * me.heads + me.head;
        return (int64_t)(me.ok && h < t.heads ? h : 0) * D;
      };
      Piece<T> wt, x, d, next_x, next_d;
      auto load = [&](Piece<T>& px, Piece<T>& pd, int p) __attribute__((always_inline)) {
        pd.load(t.dy, me.row * t.dys + head_of(p), me.ra, me.rb);
        if constexpr (NORM) px.load(t.x, me.row * t.xs + head_of(p), me.ra, me.rb);
      };
      int p = first_pass(a, i, part);
      if (p < t.passes) load(x, d, p);
      if constexpr (NORM) load_weight<T>(wt, t, me.ra, me.rb);
      if (i == 0) me.angles(a);
      for (; p < t.passes; p += a.split) {
        const int after = p + a.split;
        if (after < t.passes) load(next_x, next_d, after);
        const bool mine = me.ok && p * me.heads + me.head < t.heads;
        float g[8], k[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = d.a[e], k[e] = d.b[e];
        turn<IL>(g, k, me.c, me.s, true);
        if constexpr (NORM) {
          S ss = 0, hx = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            ss += (S)x.a[e] * (S)x.a[e] + (S)x.b[e] * (S)x.b[e];
            hx += (S)(g[e] * wt.a[e]) * (S)x.a[e] + (S)(k[e] * wt.b[e]) * (S)x.b[e];
          }
          ss = row_sum<LPR>(ss);
          hx = row_sum<LPR>(hx);
          const float r = inverse_root(ss * (S)(1.0 / D) + (S)a.eps);
          const float m = (float)(hx * (S)(1.0 / D) * (S)r);  // mean(h x r)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (mine) {
              dw[i][e] = fmaf(g[e], x.a[e] * r, dw[i][e]);
              dw[i][8 + e] = fmaf(k[e], x.b[e] * r, dw[i][8 + e]);
            }
            g[e] = r * fmaf(-(x.a[e] * r), m, g[e] * wt.a[e]);
            k[e] = r * fmaf(-(x.b[e] * r), m, k[e] * wt.b[e]);
          }
          if constexpr (LONG) {
            if (++chain[i] == kRotateChain) {
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                double& sum = far[w][16 * i + e][lane];
                sum = (have_far[i] ? sum : 0.0) + (double)dw[i][e];
                dw[i][e] = 0.f;
              }
              chain[i] = 0;
              have_far[i] = true;
            }
          }
        }
        if (mine) {
          T* o = (T*)t.out + me.row * t.outs + head_of(p);
          store8(o + me.ra, g);
          store8(o + me.rb, k);
        }
        x = next_x;
        d = next_d;
      }
    }
  }
  if constexpr (NORM) {
    if (!a.partials) return;
    // the lanes that hold the same elements, then the waves, in a fixed order
    __shared__ float sums[kWaves][2][D];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (LONG && have_far[i]) dw[i][e] = (float)(far[w][16 * i + e][lane] + (double)dw[i][e]);
#pragma unroll
        for (int m = LPR; m < 64; m <<= 1) dw[i][e] += __shfl_xor(dw[i][e], m);
        if (lane < LPR) sums[w][i][(e < 8 ? me.ra : me.rb) + (e & 7)] = dw[i][e];
      }
    __syncthreads();
    for (int n = threadIdx.x; n < 2 * D; n += kWaves * 64) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) x += sums[k][n / D][n % D];
      a.partials[((int64_t)(n / 16) * a.wgs + blockIdx.x) * 16 + n % 16] = x;
    }
  }
}

// The workgroups' sums added up: 16 columns a workgroup, 4 of a workgroup's sums a lane.
template <int D>
__global__ __launch_bounds__(1024) void rotate_dw_kernel(const RotateArgs a) {
  __shared__ double sums[16][16];
  const int lane = threadIdx.x & 63, col = lane & 3, at = threadIdx.x >> 2;
  const float* const p = a.partials + (int64_t)blockIdx.x * a.wgs * 16 + col * 4;
  double x[4] = {0, 0, 0, 0};
  for (int r = at; r < a.wgs; r += 256) {
    const f32x4 v = *(const f32x4*)(p + (int64_t)r * 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += (double)v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int m = 4; m < 64; m <<= 1) x[e] += shfl_x(x[e], m);
    if (lane < 4) sums[threadIdx.x >> 6][col * 4 + e] = x[e];
  }
  __syncthreads();
  if (threadIdx.x < 16) {
    double y = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) y += sums[k][threadIdx.x];
    const int n = blockIdx.x * 16 + threadIdx.x;
    float* const dw = a.dw[n / D];
    if (dw) dw[n % D] = (float)y;
  }
}

template <class T, int D, bool IL>
void launch(const RotateArgs& a, bool bwd, hipStream_t s) {
  const dim3 grid(a.wgs), threads(kWaves * 64);
  const bool norm = a.eps > 0;
  if (!bwd) {
    if (norm) hipLaunchKernelGGL((rotate_fwd_kernel<T, D, IL, true>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((rotate_fwd_kernel<T, D, IL, false>), grid, threads, 0, s, a);
    return;
  }
  if (a.wgs == 0) {  // (no rows: zeros)
  } else if (norm && a.partials && a.chain > kRotateChain)
    hipLaunchKernelGGL((rotate_bwd_kernel<T, D, IL, true, true>), grid, threads, 0, s, a);
  else if (norm) hipLaunchKernelGGL((rotate_bwd_kernel<T, D, IL, true, false>), grid, threads, 0, s, a);
  else hipLaunchKernelGGL((rotate_bwd_kernel<T, D, IL, false, false>), grid, threads, 0, s, a);
  if (a.partials) hipLaunchKernelGGL((rotate_dw_kernel<D>), dim3(2 * D / 16), dim3(1024), 0, s, a);
}
template <class T, int D>
void launch(const RotateArgs& a, int il, bool bwd, hipStream_t s) {
  il ? launch<T, D, true>(a, bwd, s) : launch<T, D, false>(a, bwd, s);
}
hipError_t launch(const RotateArgs& a, int head_dim, int is_bf16, int il, bool bwd, hipStream_t s) {
  if (is_bf16) head_dim == 128 ? launch<bf16, 128>(a, il, bwd, s) : launch<bf16, 64>(a, il, bwd, s);
  else head_dim == 128 ? launch<float, 128>(a, il, bwd, s) : launch<float, 64>(a, il, bwd, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate_fwd(const RotateArgs& a, int head_dim, int is_bf16, int interleaved, hipStream_t s) {
  return launch(a, head_dim, is_bf16, interleaved, false, s);
}
hipError_t launch_rotate_bwd(const RotateArgs& a, int head_dim, int is_bf16, int interleaved, hipStream_t s) {
  return launch(a, head_dim, is_bf16, interleaved, true, s);
}

}  // namespace bdlm
