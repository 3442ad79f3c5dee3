// Attention of decoding requests over a paged cache, fp32, gfx950: as
// prefix_bf16.hip, with scores, exponentials and sums in fp64 on the fp64
// matrix cores (f64tile.hpp), like the fp32 forward (fwd_f32.hip).  A workgroup
// of eight waves owns 16 query rows of a KV head and a chunk of keys, whose
// 16-key tiles the waves take in turn; K and V rows go straight from global
// memory into registers, rows past the chunk from a row of zeros.  Bound by
// the fp64 matrix rate (16 rows share a tile's products however few they are)
// and, for few requests, by latency (4 requests of 290 keys, 8/2 heads, d 64: 13.5
// us for three tiles a wave, behind the chain sequence, length, page, key).
#include "chunk.hpp"
#include "f64tile.hpp"

namespace bdlm {

namespace {

constexpr int kWaves = 8;
constexpr double kRescale = 256.0;  // as in fwd_f32.hip

__device__ __attribute__((aligned(256))) const float zero_row_f32[128] = {};

template <int D, class Args>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefix_f32_kernel(
    const Args a) {
  constexpr int NC = D / 16;
  // Q as fp64 row operands during the walk, the waves' O^T sums after it
  __shared__ __attribute__((aligned(16))) double lds[kWaves * 16 * kRedRow<D>];
  __shared__ double red_m[kWaves][16], red_l[kWaves][16];
  __shared__ int pages[kPrefixTableEntries];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i = lane & 15, g = lane >> 4;
  typename ItemOf<Args>::type it;
  if (!attn_item<false>(a, blockIdx.x, it)) {
    fill_rest<float, D>(a, blockIdx.x, gridDim.x);
    return;
  }
  const bool single = writes_outputs(a, it);
  const int nkeys = it.k1 - it.k0, page0 = it.k0 / a.page_size;
  [[maybe_unused]] WalkPages wp;
  if constexpr (kIsChunk<Args>) wp = walk_pages(a, it);
  if (nkeys > 0) {
    int n = (it.k1 - 1) / a.page_size - page0 + 1;
    if constexpr (kIsChunk<Args>) n = wp.n;
    for (int e = tid; e < n; e += kWaves * 64) {
      int pe = page0 + e;
      if constexpr (kIsChunk<Args>) pe = wp.page(e);
      const int p = a.table[(int64_t)it.seq * a.max_pages + pe];
      pages[e] = (unsigned)p < (unsigned)a.pages ? p : -1;
    }
  }
  // (the rows of a tile lie apart: one at a time, in the order of stage_row_operands)
  for (int n = tid; n < 64 * NC; n += kWaves * 64) {
    const int ln = n & 63, c = n >> 6, r = imin(ln & 15, it.nrows - 1), gg = ln >> 4;
    const auto pr = item_row(a, it, r);
    const fl4 x = *(const fl4*)((const float*)a.q + q_elem<D>(a, pr) + 16 * c + 4 * gg);
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[((2 * c + (e >> 1)) * 64 + ln) * 2 + (e & 1)] = (double)x[e];
  }
  const auto mine_row = item_row(a, it, imin(i, it.nrows - 1));
  const int end = imin(mine_row.end, it.k1);  // of this lane's row
  auto visible = [&](int key) __attribute__((always_inline)) {
    if constexpr (kIsChunk<Args>) return (key < end) & ((key >= mine_row.lo) | (key < a.sinks));
    else return key < end;
  };
  __syncthreads();

  const int64_t row_elems = (int64_t)a.kv_heads * D;
  const float* const kb = (const float*)a.k + it.kvh * D;
  const float* const vb = (const float*)a.v + it.kvh * D;
  auto key_offset = [&](int key) __attribute__((always_inline)) -> int64_t {
    if (key >= it.k1) return -1;
    if constexpr (kIsChunk<Args>) {
      if (key >= a.sinks && key < it.w0) return -1;
    }
    const int kk = walk_key(it, key), e = page_of(a, kk);
    int at = e - page0;
    if constexpr (kIsChunk<Args>) at = key < it.gap_at ? e - wp.p0 : wp.n0 + (e - wp.p1);
    const int p = pages[at];
    return p < 0 ? -1 : ((int64_t)p * a.page_size + (kk - e * a.page_size)) * row_elems;
  };
  auto row_of = [&](const float* base, int64_t off) { return off < 0 ? (const float*)zero_row_f32 : base + off; };
  const double c = (double)a.scale * kLog2eD;

  AccTiles<D> acc;
  acc.zero();
  double m = -INFINITY, l = 0.0;
  const int ntiles = (nkeys + 15) / 16;
  fl4 kx[NC];
  auto load_keys = [&](int64_t mine) __attribute__((always_inline)) {
    const float* p = row_of(kb, mine) + 4 * g;
#pragma unroll
    for (int k = 0; k < NC; ++k) kx[k] = *(const fl4*)(p + 16 * k);
  };
  int64_t mine = key_offset(it.k0 + w * 16 + i);
  if (w < ntiles) load_keys(mine);
  for (int t = w; t < ntiles; t += kWaves) {
    const int key0 = it.k0 + t * 16;
    ColOps<D> vx;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int r = 4 * kk + g;
      const int lo = __shfl((int)(uint32_t)mine, r), hi = __shfl((int)(mine >> 32), r);
      const float* p = row_of(vb, ((int64_t)hi << 32) | (uint32_t)lo) + 4 * i;
#pragma unroll
      for (int h = 0; h < D / 64; ++h) vx.x[kk][h] = *(const fl4*)(p + 64 * h);
    }
    f64x4 s = row_product<D>(kx, lds, lane) * c;
    // the next tile's keys are loaded under the softmax and the products below
    mine = key_offset(key0 + kWaves * 16 + i);
    load_keys(mine);
    bool grow = false;
#pragma unroll
    for (int r = 0; r < 4; ++r) grow |= visible(key0 + 4 * r + g) && !(s[r] <= m + kRescale);
    if (__builtin_amdgcn_ballot_w64(grow) != 0) {
      double mx = -INFINITY;
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = visible(key0 + 4 * r + g) ? fmax(mx, s[r]) : mx;
      const double mn = fmax(m, col_max(mx));
      const double al = m == -INFINITY ? 0.0 : exp2_f64(m - mn);
      l *= al;
      acc.scale(al);
      m = mn;
    }
    f64x4 p;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      p[r] = exp2_f64(visible(key0 + 4 * r + g) ? s[r] - m : kHidden);
      l += p[r];
    }
    col_product<D>(acc, vx, p);
  }

  // Merge the waves, as fwd_f32.hip; each wave also scales its own row sums.
  l = col_sum(l);
  if (g == 0) red_m[w][i] = m;
  __syncthreads();
  double mt = red_m[0][i];
#pragma unroll
  for (int k = 1; k < kWaves; ++k) mt = fmax(mt, red_m[k][i]);
  const double al = m == -INFINITY ? 0.0 : exp2_f64(m - mt);
  if (g == 0) red_l[w][i] = l * al;
  acc.scale(al);
  acc_to_lds<D>(acc, lds + w * 16 * kRedRow<D>, i, g);
  __syncthreads();
  // four elements of a row per thread
  const int q = tid / (D / 4), d0 = (tid % (D / 4)) * 4;
  if (q >= it.nrows) return;
  double M = red_m[0][q], lt = red_l[0][q];
#pragma unroll
  for (int k = 1; k < kWaves; ++k) {
    M = fmax(M, red_m[k][q]);
    lt += red_l[k][q];
  }
  const bool empty = !(lt > 0.0);
  const double inv = empty ? 0.0 : 1.0 / lt;
  const auto pr = item_row(a, it, q);
  const int64_t at = part_row(a, it, pr, q);
  float* op = (single ? (float*)a.o + o_elem<D>(a, pr) : a.part_o + at * D) + d0;
  fl4 out;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    double x = 0.0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) x += lds[(k * 16 + q) * kRedRow<D> + d0 + e];
    out[e] = (float)(x * inv);
  }
  *(fl4*)op = out;
  if (d0 == 0) {
    const double z = M + log2(lt);
    if (single) a.lse[lse_elem(a, pr)] = empty ? -INFINITY : (float)(z * kLn2D);
    else ((double*)a.part_lse)[at] = empty ? -INFINITY : z;
  }
}

template <class Args>
void launch(const Args& a, int head_dim, int n, hipStream_t s) {
  if (head_dim == 128) hipLaunchKernelGGL((prefix_f32_kernel<128, Args>), dim3(n), dim3(kWaves * 64), 0, s, a);
  else hipLaunchKernelGGL((prefix_f32_kernel<64, Args>), dim3(n), dim3(kWaves * 64), 0, s, a);
}

}  // namespace

#ifdef BDLM_CHUNK_CALLS

hipError_t launch_chunk_f32(const ChunkArgs& a, int head_dim, hipStream_t s) {
  const int n = a.max_items * a.kv_heads + (a.fill ? kFillWgs : 0);
  if (n == 0) return hipSuccess;
  launch(a, head_dim, n, s);
  return hipGetLastError();
}

#else

hipError_t launch_prefix_f32(const PrefixArgs& a, int head_dim, hipStream_t s) {
  const int n = a.prefix_items + a.own_items;
  if (n == 0) return hipSuccess;
  launch(a, head_dim, n, s);
  return hipGetLastError();
}

#endif

}  // namespace bdlm
