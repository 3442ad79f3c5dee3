// Attention of decoding requests over a paged cache, bf16, gfx950: a long
// prefix that all requests share is read once for all of them, each request's
// own keys once (PrefixArgs in cache.hpp says how rows and keys are cut up).
//
// Per chunk of keys and tile of rows: S^T = K Q^T, an online softmax, and
// O^T += V^T P^T with v_mfma_f32_32x32x16_bf16, the products, layouts and LDS
// swizzle of the forward (fwd_bf16.hip).  A workgroup of four waves (two fit a
// CU, so that one's start-up overlaps the other's products) runs an item in one
// of two forms:
//  * shared: 128 rows, 32 per wave; the waves share 64-key tiles in two LDS
//    stages.  For the prefix of a batch and for blocks of query rows: bound by
//    the matrix cores from some 300 rows on.
//  * by waves: 32 rows; every wave takes every fourth 32-key tile through its
//    own 16 KB of LDS, without barriers, and the waves' sums are merged at the
//    end.  For single tokens (few rows): bound by reading K and V.  A wave asks
//    for the next tile's keys as soon as its scores are there, and for its
//    values after P V, so that it always has copies in flight.
// Keys come by LDS-DMA copies (a cache may be larger than 4 GB).  Where pages
// are whole groups of 16 tokens (GROUPS), tiles start at groups, the groups'
// byte offsets wait in LDS, and a copy takes a wave-uniform 64-bit base and
// constant lane offsets: no vector work per copy (with an address per lane, the
// shuffles and 64-bit sums of which took as long as the softmax, 16 requests of
// 32 rows behind 16K tokens took 184 us).  Other page sizes, and tiles with
// rows past the chunk or in no page, which come from a row of zeros, take an
// address per lane.
//
// Measured, 32 query heads: 64 requests of 4,000 keys each, 8 KV heads, 196 us
// (5.3 TB/s, a copy's rate); 64 of 60 to 1,500 behind 8K, read again, 38 us.  Blocks
// of 32 rows of 16 requests behind 16K, 4 KV heads, 156 us (0.9 PFLOP/s): operand
// reads take LDS as long as the products take the matrix cores, and copies a quarter
// more (without them 138 us; without the exponentials 145).
#include "cache.hpp"
#include "device.hpp"

namespace bdlm {

namespace {

constexpr int kNW = 4;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kSumLimit = 18446744073709551616.f;  // 2^64: a lane's tile sum of p above which the running max moves

__device__ __attribute__((aligned(256))) const uint32_t zero_row[64] = {};

// Global -> LDS copy of 16 bytes per lane: lane i's land at m0 + 16 i.  Inline
// assembly, as in bwd_dkdv.hip: for the builtin the compiler waits for all
// copies in flight before any LDS read.
__device__ __forceinline__ void dma16(const char* src, uint32_t lds_byte) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds_byte) : "memory");
}
// The same at a wave-uniform base and a 32-bit lane offset.
__device__ __forceinline__ void dma16(const char* base, uint32_t voff, uint32_t lds_byte) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(voff), "s"(base), "{m0}"(lds_byte) : "memory");
}
// (a base from readlane, a vector instruction writing scalar registers, needs five wait states before a copy reads it)
__device__ __forceinline__ void base_ready(const char* a, const char* b) { asm volatile("s_nop 4" ::"s"(a), "s"(b)); }
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void vm_wait() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Softmax state and O^T of a wave's 32 rows (a lane owns row lane % 32; its
// sum covers the keys of its half until the end).
template <int D>
struct RowState {
  f32x16 acc[D / 32];
  float m, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }
};

// P of U 32-key steps from the scores, as bf16 operands (off by at most 2^-8
// relative, as in the forward).  The running max of a row moves on its first
// visible tile, and when a lane's sum over a tile passes 2^64: see fwd_bf16.hip.
template <int D, int U>
__device__ __forceinline__ void softmax_step(RowState<D>& st, const f32x16 (&s)[U], bf16x8 (&pb)[2 * U], float c) {
  float psum;
  auto probs = [&](float m) __attribute__((always_inline)) {
    psum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = exp2f_fast(fmaf(s[u][i], c, -m));
        psum += p;
        pb[2 * u + (i >> 3)][i & 7] = to_bf16(p);
      }
  };
  bool rescale = __builtin_amdgcn_ballot_w64(st.m == -INFINITY) != 0;
  if (!rescale) {
    probs(st.m);
    rescale = __builtin_amdgcn_ballot_w64(psum > kSumLimit) != 0;
  }
  if (rescale) {
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[u][i]);
    mx = fmaxf(mx, partner(mx));
    const float mn = fmaxf(st.m, mx * c);
    const float al = exp2f_fast(st.m - (mn == -INFINITY ? 0.f : mn));
    st.l *= al;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.acc[d][i] *= al;
    st.m = mn;
    probs(mn == -INFINITY ? 0.f : mn);
  }
  st.l += psum;
}

template <int D>
struct Lds {
  static constexpr uint32_t RB = D * 2;
  static constexpr uint32_t Stage = 2 * 64 * RB;     // K and V of 64 keys
  static constexpr uint32_t Wave = 2 * 32 * RB;      // K and V of 32 keys; later 32 rows of sums
  static constexpr uint32_t Tiles = kNW * Wave > 2 * Stage ? kNW * Wave : 2 * Stage;
  static constexpr uint32_t Pages = Tiles;
  static constexpr uint32_t Ml = Pages + kPrefixTableEntries * 4;  // (or kPrefixGroups * 8)
  static constexpr uint32_t Bytes = Ml + kNW * 32 * 8;
  static_assert(Wave == 32 * D * 4, "a wave's sums fit its tiles");
};

template <int D, bool GROUPS>
__global__ __launch_bounds__(kNW * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefix_bf16_kernel(
    const PrefixArgs a) {
  using L = Lds<D>;
  constexpr int KS = D / 16, DT = D / 32, CH = D / 8;
  constexpr uint32_t RB = L::RB;
  __shared__ __attribute__((aligned(1024))) unsigned char lds[L::Bytes];
  const uint32_t L0 = lds_addr(lds);
  int* const pages = (int*)(lds + L::Pages);
  int64_t* const groups = (int64_t*)(lds + L::Pages);
  float* const red_m = (float*)(lds + L::Ml);  // [wave][32], the sums behind it
  float* const red_l = red_m + kNW * 32;

  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5, G = lane >> 4, sl = lane & 15;

  PrefixItem it;
  if (!prefix_item(a, blockIdx.x, a.prefix_shared ? kPrefixSharedRows : kPrefixWaveRows,
                   a.own_shared ? kPrefixSharedRows : kPrefixWaveRows, it))
    return;
  const bool single = a.prefix_chunks + a.own_chunks == 1;
  const float c = a.scale_log2;
  // Tiles start at the chunk's first key, or at the group of 16 that holds it (the keys before it are hidden).
  const int start = GROUPS ? it.k0 & ~15 : it.k0;
  const int nkeys = it.k1 > it.k0 ? it.k1 - start : 0;
  const int64_t row_bytes = (int64_t)a.kv_heads * RB;

  // The byte offsets of the chunk's groups, or its page numbers; -1 for pages
  // outside the cache, whose rows read as zeros.
  const int page0 = it.k0 / a.page_size;
  if (nkeys > 0) {
    const int32_t* const table = a.table + (int64_t)it.seq * a.max_pages;
    const int n = GROUPS ? (nkeys + 15) / 16 : (it.k1 - 1) / a.page_size - page0 + 1;
    for (int e = tid; e < n; e += kNW * 64) {
      const int key = start + e * 16, pe = GROUPS ? key / a.page_size : page0 + e;
      const int p = table[pe];
      const bool ok = (unsigned)p < (unsigned)a.pages;
      if constexpr (GROUPS) groups[e] = ok ? ((int64_t)p * a.page_size + (key - pe * a.page_size)) * row_bytes : -1;
      else pages[e] = ok ? p : -1;
    }
  }

  // This wave's rows as MFMA B fragments.
  const int lrow = (it.shared ? w * 32 : 0) + l32;  // within the item's rows
  const bool row_ok = lrow < it.nrows;
  const PrefixRow row = prefix_row(a, it.kvh, it.row0 + imin(lrow, it.nrows - 1));
  const int64_t out_row = (int64_t)row.token * a.heads + row.head;
  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s)
    qf[s] = *(const bf16x8*)((const bf16*)a.q + out_row * D + 16 * s + 8 * half);
  const int end = imin(row.end, it.k1);
  __syncthreads();
  // (waited for here: the loops' own waits count copies that the compiler does not know of)
#pragma unroll
  for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[s]));

  const char* const kb = a.k + (int64_t)it.kvh * RB;
  const char* const vb = a.v + (int64_t)it.kvh * RB;
  const char* const zero = (const char*)zero_row;
  // Byte offset of a key's row in K (and V), -1: a row of zeros.
  auto key_offset = [&](int key) __attribute__((always_inline)) -> int64_t {
    if (key >= it.k1) return -1;
    if constexpr (GROUPS) {
      const int64_t g = groups[(key - start) >> 4];
      return g < 0 ? -1 : g + (key & 15) * row_bytes;
    } else {
      const int e = key / a.page_size;
      const int p = pages[e - page0];
      return p < 0 ? -1 : ((int64_t)p * a.page_size + (key - e * a.page_size)) * row_bytes;
    }
  };
  // Copies of 32 rows from key `first` (a multiple of 16 with GROUPS) on to LDS.
  constexpr int RPI = 64 / CH, NI = 32 / RPI, GI = 16 / RPI;  // rows per copy; copies of 32 rows, of a group
  uint32_t voff[GI];
#pragma unroll
  for (int i = 0; i < GI; ++i) {
    const int r = i * RPI + lane / CH;
    voff[i] = (uint32_t)(r * (int)row_bytes) + (uint32_t)((lane % CH) ^ chunk_swz<D>(r)) * 16u;
  }
  // Their two groups' offsets, read ahead of the copies (any value where there is no such pair of groups).
  struct Pair {
    int64_t g0, g1;
  };
  auto pair_at = [&](int first) __attribute__((always_inline)) -> Pair {
    if constexpr (!GROUPS) return Pair{-1, -1};
    const int e = imin((first - start) >> 4, kPrefixGroups - 2);
    return Pair{groups[e], groups[e + 1]};
  };
  auto copy32 = [&](const char* base, int first, const Pair& ahead, uint32_t dst) __attribute__((always_inline)) {
    if constexpr (GROUPS) {
      if (first + 32 <= it.k1) {
        auto uniform = [](int64_t x) __attribute__((always_inline)) {
          return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
                           (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
        };
        const int64_t g0 = uniform(ahead.g0), g1 = uniform(ahead.g1);
        if ((g0 | g1) >= 0) {
          const char *b0 = base + g0, *b1 = base + g1;
          lds_done();  // the rows there have been read
          base_ready(b0, b1);
#pragma unroll
          for (int i = 0; i < NI; ++i) dma16(i < GI ? b0 : b1, voff[i % GI], dst + i * 1024);
          return;
        }
      }
    }
    const int64_t mine = key_offset(first + l32);
    lds_done();
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int r = i * RPI + lane / CH;
      const int lo = __shfl((int)(uint32_t)mine, r), hi = __shfl((int)(mine >> 32), r);
      const int64_t off = ((int64_t)hi << 32) | (uint32_t)lo;
      dma16((off < 0 ? zero : base + off) + (uint32_t)((lane % CH) ^ chunk_swz<D>(r)) * 16u, dst + i * 1024);
    }
  };
  const uint32_t yrow = swz_row_part<D>(l32, half);
  const uint32_t ytr0 = swz_tr_part<D>(G, sl, 0), ytr1 = swz_tr_part<D>(G, sl, 8);
  RowState<D> st;
  st.init();

  if (it.shared) {
    // ---- the waves share 64-key tiles; waves 0 and 1 copy K, 2 and 3 V, 32 rows each
    const int ntiles = (nkeys + 63) / 64;
    const char* const base = w < 2 ? kb : vb;
    const int crow = (w & 1) * 32;
    auto first_of = [&](int t) { return t < ntiles ? start + t * 64 + crow : it.k1; };
    auto copy_tile = [&](int t, const Pair& ahead, int stage) __attribute__((always_inline)) {
      copy32(base, first_of(t), ahead, L0 + stage * L::Stage + (w < 2 ? 0u : 64 * RB) + crow * RB);
    };
    const bool any = __builtin_amdgcn_ballot_w64(row_ok && end > it.k0) != 0;
    copy_tile(0, pair_at(first_of(0)), 0);
    Pair ahead = pair_at(first_of(1));
    vm_wait_barrier<0>();
    for (int t = 0; t < ntiles; ++t) {
      copy_tile(t + 1, ahead, (t + 1) & 1);
      ahead = pair_at(first_of(t + 2));
      const int key0 = start + t * 64;
      if (any && __builtin_amdgcn_ballot_w64(end > key0) != 0) {
        const uint32_t sb = L0 + (t & 1) * L::Stage;
        const uint32_t zr = sb + yrow;
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
        {
          // key fragments LA k-steps ahead of their products, as in the forward
          constexpr int LA = 3;
          bf16x8 kf[LA + 1][2];
#pragma unroll
          for (int k = 0; k < LA; ++k)
#pragma unroll
            for (int u = 0; u < 2; ++u) kf[k][u] = lds_load16((zr ^ (32u * k)) + u * 32 * RB);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int k = 0; k < KS; ++k) {
            if (k + LA < KS) {
#pragma unroll
              for (int u = 0; u < 2; ++u) kf[(k + LA) % (LA + 1)][u] = lds_load16((zr ^ (32u * (k + LA))) + u * 32 * RB);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = mfma32(kf[k % (LA + 1)][u], qf[k], s[u]);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (key0 < it.k0 || __builtin_amdgcn_ballot_w64(end < key0 + 64) != 0) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int key = key0 + u * 32 + (i >> 2) * 8 + 4 * half + (i & 3);
              if (key >= end || (GROUPS && key < it.k0)) s[u][i] = -INFINITY;
            }
        }
        // value fragments PA products ahead, the first ones under the softmax
        const uint32_t zt0 = sb + 64 * RB + ytr0, zt1 = sb + 64 * RB + ytr1;
        auto vop = [&](int n) {
          const int u = n / DT, d = n % DT;
          return cat(lds_read_tr_at((zt0 ^ (64u * d)) + u * 16 * RB), lds_read_tr_at((zt1 ^ (64u * d)) + u * 16 * RB));
        };
        constexpr int PA = 4, NP = 4 * DT;
        bf16x8 vr[PA + 1];
#pragma unroll
        for (int n = 0; n < PA; ++n) vr[n] = vop(n);
        bf16x8 pb[4];
        softmax_step<D, 2>(st, s, pb, c);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          if (n + PA < NP) vr[(n + PA) % (PA + 1)] = vop(n + PA);
          st.acc[n % DT] = mfma32(vr[n % (PA + 1)], pb[n / DT], st.acc[n % DT]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      vm_wait_barrier<0>();
    }
    vm_wait<0>();  // copies in flight land before the LDS is released
    const float l = st.l + partner(st.l);
    const bool empty = !(l > 0.f);
    const float inv = empty ? 0.f : 1.f / l;
    if (row_ok) {
      if (single) {
        bf16* op = (bf16*)a.o + out_row * D;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            bf16x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = to_bf16(st.acc[d][4 * g4 + e] * inv);
            *(bf16x4*)(op + 32 * d + 8 * g4 + 4 * half) = x;
          }
        if (half == 0) a.lse[prefix_lse_at(a, row)] = empty ? -INFINITY : (st.m + log2f(l)) * kLn2;
      } else {
        const int64_t at = (int64_t)it.part * a.requests * a.rows * a.heads + out_row;
        if (!empty) {
          float* op = a.part_o + at * D;
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
              f32x4 x;
#pragma unroll
              for (int e = 0; e < 4; ++e) x[e] = st.acc[d][4 * g4 + e] * inv;
              *(f32x4*)(op + 32 * d + 8 * g4 + 4 * half) = x;
            }
        }
        if (half == 0) ((float*)a.part_lse)[at] = empty ? -INFINITY : st.m + log2f(l);
      }
    }
    return;
  }

  // ---- by waves: tile t of 32 keys to wave t % 4
  const int ntiles = (nkeys + 31) / 32;
  const uint32_t wb = L0 + w * L::Wave, wv = wb + 32 * RB;
  if (w < ntiles) {
    Pair ahead = pair_at(start + w * 32);
    copy32(kb, start + w * 32, ahead, wb);
    copy32(vb, start + w * 32, ahead, wv);
    for (int t = w; t < ntiles; t += kNW) {
      const int key0 = start + t * 32, next = key0 + kNW * 32;  // (past the chunk: zeros)
      ahead = pair_at(next);
      vm_wait<NI>();  // the keys are there, the values in flight
      f32x16 s[1];
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) s[0] = mfma32(lds_load16((wb + yrow) ^ (32u * k)), qf[k], s[0]);
      copy32(kb, next, ahead, wb);
      if (key0 < it.k0 || __builtin_amdgcn_ballot_w64(end < key0 + 32) != 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = key0 + (i >> 2) * 8 + 4 * half + (i & 3);
          if (key >= end || (GROUPS && key < it.k0)) s[0][i] = -INFINITY;
        }
      }
      bf16x8 pb[2];
      softmax_step<D, 1>(st, s, pb, c);
      vm_wait<NI>();  // the values are there, the next keys in flight
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          st.acc[d] = mfma32(cat(lds_read_tr_at(((wv + ytr0) ^ (64u * d)) + u * 16 * RB),
                                 lds_read_tr_at(((wv + ytr1) ^ (64u * d)) + u * 16 * RB)),
                             pb[u], st.acc[d]);
      copy32(vb, next, ahead, wv);
    }
    vm_wait<0>();
  }
  // Merge the waves: sums of 32 rows per wave through LDS, [row][D], with the
  // 16-byte pieces of row r rotated by r so that the lanes' stores spread over the banks.
  const float l = st.l + partner(st.l);
  if (half == 0) {
    red_m[w * 32 + l32] = st.m;
    red_l[w * 32 + l32] = l;
  }
  constexpr int PC = D / 4;  // 16-byte pieces of a row of sums
  if (w < ntiles) {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        f32x4 x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = st.acc[d][4 * g4 + e];
        const int piece = (8 * d + 2 * g4 + half + l32) % PC;
        *(f32x4*)(lds + w * L::Wave + l32 * (D * 4) + piece * 16) = x;
      }
  }
  __syncthreads();
  const int used = imin(ntiles, kNW);
  for (int n = tid; n < it.nrows * PC; n += kNW * 64) {
    const int r = n / PC, piece = n % PC;
    float m = -INFINITY;
    for (int k = 0; k < used; ++k) m = fmaxf(m, red_m[k * 32 + r]);
    float lt = 0.f;
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
    for (int k = 0; k < used; ++k) {
      const float mk = red_m[k * 32 + r];
      if (mk == -INFINITY) continue;
      const float f = exp2f_fast(mk - m);
      lt += red_l[k * 32 + r] * f;
      x += *(const f32x4*)(lds + k * L::Wave + r * (D * 4) + ((piece + r) % PC) * 16) * f;
    }
    const bool empty = !(lt > 0.f);
    x *= empty ? 0.f : 1.f / lt;
    const PrefixRow pr = prefix_row(a, it.kvh, it.row0 + r);
    const int64_t orow = (int64_t)pr.token * a.heads + pr.head;
    if (single) {
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = to_bf16(x[e]);
      *(bf16x4*)((bf16*)a.o + orow * D + piece * 4) = y;
      if (piece == 0) a.lse[prefix_lse_at(a, pr)] = empty ? -INFINITY : (m + log2f(lt)) * kLn2;
    } else {
      const int64_t at = (int64_t)it.part * a.requests * a.rows * a.heads + orow;
      if (!empty) *(f32x4*)(a.part_o + at * D + piece * 4) = x;
      if (piece == 0) ((float*)a.part_lse)[at] = empty ? -INFINITY : m + log2f(lt);
    }
  }
}

template <int D>
void launch(const PrefixArgs& a, int n, hipStream_t s) {
  if (a.page_size % 16 == 0) hipLaunchKernelGGL((prefix_bf16_kernel<D, true>), dim3(n), dim3(kNW * 64), 0, s, a);
  else hipLaunchKernelGGL((prefix_bf16_kernel<D, false>), dim3(n), dim3(kNW * 64), 0, s, a);
}

}  // namespace

hipError_t launch_prefix_bf16(const PrefixArgs& a, int head_dim, hipStream_t s) {
  const int n = a.prefix_items + a.own_items;
  if (n == 0) return hipSuccess;
  head_dim == 128 ? launch<128>(a, n, s) : launch<64>(a, n, s);
  return hipGetLastError();
}

}  // namespace bdlm
