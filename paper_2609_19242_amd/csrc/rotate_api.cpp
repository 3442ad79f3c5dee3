// C ABI of rotated queries and keys: argument validation, how rows and heads
// are dealt out, launches.  Declarations and contracts: include/bdlm_attn.h.
#include "bdlm_attn.h"

#include <algorithm>
#include <cmath>

#include "api_util.hpp"
#include "rotate.hpp"

using namespace bdlm;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 28;
constexpr int64_t kMaxStride = (int64_t)1 << 30;
constexpr double kMinEps = 0x1p-100;    // (a sum with it must be an fp32 number, and not 0)
constexpr int64_t kWaves = kRotateWaves;
constexpr int64_t kFullWaves = 2048;    // waves from which on a row's heads stay with one wave
constexpr double kApart = 1.3;          // what a pass over heads of several rows takes longer
constexpr int64_t kMaxFwdWgs = 1 << 20;
constexpr int64_t kMaxBwdWgs = 512;     // (each leaves its sums of the weights' gradients)

bdlm_status check_rotary(const bdlm_rotary* r, int32_t dtype, int64_t rows, const int32_t* pos, int32_t heads,
                         int32_t kv_heads, double eps) {
  if (!r) return fail(BDLM_ERR_INVALID, "rotary is null");
  if (r->head_dim != 64 && r->head_dim != 128)
    return fail(BDLM_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", r->head_dim);
  if (r->dim < 16 || r->dim > r->head_dim || r->dim % 16 != 0)
    return fail(BDLM_ERR_INVALID, "dim %d is not a multiple of 16 in [16, head_dim]", r->dim);
  if (r->interleaved != 0 && r->interleaved != 1) return fail(BDLM_ERR_INVALID, "interleaved must be 0 or 1");
  if (r->axes < 1 || r->axes > BDLM_MAX_AXES)
    return fail(BDLM_ERR_INVALID, "axes %d outside [1, %d]", r->axes, BDLM_MAX_AXES);
  for (int i = 0; i < r->dim / 2; ++i) {
    if (!(std::fabs(r->freq[i]) <= 1048576.0)) return fail(BDLM_ERR_INVALID, "frequency %d is not within 2^20", i);
    if (r->axis[i] < 0 || r->axis[i] >= r->axes)
      return fail(BDLM_ERR_INVALID, "pair %d: axis %d outside [0, %d)", i, r->axis[i], r->axes);
  }
  if (dtype != BDLM_BF16 && dtype != BDLM_F32) return fail(BDLM_ERR_UNSUPPORTED, "dtype %d not supported", dtype);
  if (heads < 1 || kv_heads < 1 || heads > kMaxRows || kv_heads > kMaxRows)
    return fail(BDLM_ERR_INVALID, "heads %d and kv_heads %d must be in [1, 2^28]", heads, kv_heads);
  if (rows < 0 || rows > kMaxRows) return fail(BDLM_ERR_INVALID, "rows %lld outside [0, 2^28]", (long long)rows);
  if (eps != 0.0 && !(eps >= kMinEps && eps <= 1.0 / kMinEps))
    return fail(BDLM_ERR_INVALID, "eps %g is neither 0 nor within [2^-100, 2^100]", eps);
  if (rows > 0 && (!pos || (reinterpret_cast<uintptr_t>(pos) & 3u)))
    return fail(BDLM_ERR_INVALID, "positions are null or not 4-byte aligned");
  return BDLM_OK;
}

bdlm_status check_rows(const bdlm_rows& r, const char* what, int64_t row_elems, int elem) {
  if (!r.ptr || !aligned16(r.ptr)) return fail(BDLM_ERR_INVALID, "%s is null or not 16-byte aligned", what);
  if (r.stride < row_elems || r.stride > kMaxStride || r.stride * elem % 16 != 0)
    return fail(BDLM_ERR_INVALID, "%s row stride %lld outside [%lld, 2^30] or not a multiple of 16 bytes", what,
                (long long)r.stride, (long long)row_elems);
  return BDLM_OK;
}

bdlm_status check_weight(const void* w, const char* what, double eps) {
  if (w && !aligned16(w)) return fail(BDLM_ERR_INVALID, "%s is not 16-byte aligned", what);
  if (w && eps == 0.0) return fail(BDLM_ERR_INVALID, "%s without a norm", what);
  return BDLM_OK;
}

// Rows of a wave, and waves that share a row's heads.  Times are of calls in a row on the same inputs, backward with the
// weights' sums.  Where one row's heads fill a wave, one row at a time: its loads then are of one run of memory (30,011 rows
// of 32/8 heads, d 128, with 8 rows a wave 140 us, with one 112; 16,384 77 and 63).  Few heads, or a row whose
// passes would be few beside its angles, take several (8,190 rows of 16/16 heads, d 64: 16 rows a wave 14.5 us, one
// 15.4, backward 28.0 and 29.7; 2,000 of 12/2, d 128: 6.5 and 7.4, 15.8 and 16.9).  More waves than 2,048 for the same rows
// cost more in angles than they hide (4,000 rows of 32/8 heads, d 64: 2,048 10.6 us, 4,096 11.4, 8,192 13.2, backward 24.2, 24.3,
// 27.8).  Backward: up to 512 workgroups, two per CU, go through the rows (4,000 rows of 32/8 heads, d 64, in 1,024
// 28.9 us, in 512 24.2; 30,011, d 128, 185 and 181).
// fp32, with the same numbers: 16,384 rows of 8/2 heads, d 64, 16 rows a wave 16 us, one 27, backward 30 and 47; 16,384 of
// 32/8, d 128, 149 and 130, 219 and 196; 2,000 of 12/2, d 128, 9.1 and 9.3; 4,000 of 32/8, d 128, 2,048 waves 26.9 us, 4,096
// 27.9.  Rows of 16/16 heads, d 64, would rather be taken one at a time there (8,190: 24 us, as dealt 30, backward 42 and 47).
void deal(const bdlm_rotary& r, int64_t rows, int32_t heads, int32_t kv_heads, int64_t max_wgs, RotateArgs& a) {
  const int side = 64 / (r.head_dim / 16);  // heads of a wave
  auto passes = [&](int64_t h, int per) { return (h + side / per - 1) / (side / per); };
  // passes per row, of which one for the cosines and sines; heads of one row lie side by side, those of several do not
  auto cost = [&](int per) {
    return (double)(passes(heads, per) + passes(kv_heads, per) + 1) / per * (per > 1 ? kApart : 1.0);
  };
  int best = 1;
  for (int per = 2; per <= side; per *= 2)
    if (cost(per) < cost(best)) best = per;
  a.rows_per = best;
  a.t[0].passes = (int32_t)passes(heads, best);
  a.t[1].passes = (int32_t)passes(kv_heads, best);
  const int64_t sets = (rows + best - 1) / best, all = (int64_t)a.t[0].passes + a.t[1].passes;
  a.split = (int32_t)std::min(std::max<int64_t>((kFullWaves + sets - 1) / sets, 1), all);
  a.wgs = (int32_t)std::min((sets * a.split + kWaves - 1) / kWaves, max_wgs);
  const int64_t turns = (sets * a.split + a.wgs * kWaves - 1) / (a.wgs * kWaves);
  a.chain = turns * ((std::max(a.t[0].passes, a.t[1].passes) + a.split - 1) / a.split);
}

RotateArgs rotate_args(const bdlm_rotary& r, int64_t rows, const int32_t* pos, double eps) {
  RotateArgs a{};
  a.pos = pos;
  a.rows = rows;
  a.eps = eps;
  a.axes = r.axes;
  a.dim = r.dim;
  for (int i = 0; i < r.dim / 2; ++i) {
    a.quarters[i] = r.freq[i] * 0.63661977236758134308;  // 2 / pi
    a.axis[i] = (int8_t)r.axis[i];
  }
  return a;
}

RotateTensor tensor(const bdlm_rows& x, const bdlm_rows& dy, const void* w, const bdlm_rows& out, int32_t heads) {
  RotateTensor t{};
  t.x = x.ptr;
  t.xs = x.stride;
  t.dy = dy.ptr;
  t.dys = dy.stride;
  t.w = w;
  t.out = out.ptr;
  t.outs = out.stride;
  t.heads = heads;
  return t;
}

}  // namespace

extern "C" {

bdlm_status bdlm_qk_rotate_fwd(const bdlm_rotary* r, int32_t dtype, int64_t rows, const int32_t* positions, int32_t heads,
                               int32_t kv_heads, bdlm_rows q, bdlm_rows k, const void* q_weight, const void* k_weight,
                               double eps, bdlm_rows q_out, bdlm_rows k_out, hipStream_t stream) {
  bdlm_status st;
  if ((st = check_rotary(r, dtype, rows, positions, heads, kv_heads, eps)) != BDLM_OK) return st;
  if ((st = check_weight(q_weight, "q weight", eps)) != BDLM_OK || (st = check_weight(k_weight, "k weight", eps)) != BDLM_OK)
    return st;
  if (rows == 0) return BDLM_OK;
  const int elem = dtype == BDLM_F32 ? 4 : 2;
  const int64_t qe = (int64_t)heads * r->head_dim, ke = (int64_t)kv_heads * r->head_dim;
  if ((st = check_rows(q, "q", qe, elem)) != BDLM_OK || (st = check_rows(k, "k", ke, elem)) != BDLM_OK ||
      (st = check_rows(q_out, "q_out", qe, elem)) != BDLM_OK || (st = check_rows(k_out, "k_out", ke, elem)) != BDLM_OK)
    return st;
  RotateArgs a = rotate_args(*r, rows, positions, eps);
  a.t[0] = tensor(q, bdlm_rows{}, q_weight, q_out, heads);
  a.t[1] = tensor(k, bdlm_rows{}, k_weight, k_out, kv_heads);
  deal(*r, rows, heads, kv_heads, kMaxFwdWgs, a);
  const hipError_t e = timed(kKQkRotate, stream, [&] {
    return launch_rotate_fwd(a, r->head_dim, dtype == BDLM_BF16, r->interleaved, stream);
  });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "rotation launch");
}

size_t bdlm_qk_rotate_workspace_bytes(int32_t head_dim) {
  return head_dim == 64 || head_dim == 128 ? (size_t)kMaxBwdWgs * 2 * head_dim * sizeof(float) : 0;
}

bdlm_status bdlm_qk_rotate_bwd(const bdlm_rotary* r, int32_t dtype, int64_t rows, const int32_t* positions, int32_t heads,
                               int32_t kv_heads, bdlm_rows q, bdlm_rows k, const void* q_weight, const void* k_weight,
                               double eps, bdlm_rows dq_out, bdlm_rows dk_out, bdlm_rows dq, bdlm_rows dk,
                               float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes,
                               hipStream_t stream) {
  bdlm_status st;
  if ((st = check_rotary(r, dtype, rows, positions, heads, kv_heads, eps)) != BDLM_OK) return st;
  if ((st = check_weight(q_weight, "q weight", eps)) != BDLM_OK || (st = check_weight(k_weight, "k weight", eps)) != BDLM_OK)
    return st;
  float* const dw[2] = {dq_weight, dk_weight};
  for (float* w : dw) {
    if (w && (reinterpret_cast<uintptr_t>(w) & 3u)) return fail(BDLM_ERR_INVALID, "a weight's gradient is not 4-byte aligned");
    if (w && eps == 0.0) return fail(BDLM_ERR_INVALID, "a weight's gradient without a norm");
  }
  const bool weights = dq_weight || dk_weight;
  const size_t need = weights ? bdlm_qk_rotate_workspace_bytes(r->head_dim) : 0;
  if (need > 0 && (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 255u)))
    return fail(BDLM_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu at %p)", need, workspace_bytes,
                workspace);
  if (rows == 0 && !weights) return BDLM_OK;
  RotateArgs a = rotate_args(*r, rows, positions, eps);
  a.partials = weights ? static_cast<float*>(workspace) : nullptr;
  a.dw[0] = dq_weight;
  a.dw[1] = dk_weight;
  if (rows > 0) {
    const int elem = dtype == BDLM_F32 ? 4 : 2;
    const int64_t qe = (int64_t)heads * r->head_dim, ke = (int64_t)kv_heads * r->head_dim;
    if (eps > 0.0 && ((st = check_rows(q, "q", qe, elem)) != BDLM_OK || (st = check_rows(k, "k", ke, elem)) != BDLM_OK))
      return st;
    if ((st = check_rows(dq_out, "dq_out", qe, elem)) != BDLM_OK || (st = check_rows(dk_out, "dk_out", ke, elem)) != BDLM_OK ||
        (st = check_rows(dq, "dq", qe, elem)) != BDLM_OK || (st = check_rows(dk, "dk", ke, elem)) != BDLM_OK)
      return st;
    a.t[0] = tensor(q, dq_out, q_weight, dq, heads);
    a.t[1] = tensor(k, dk_out, k_weight, dk, kv_heads);
    deal(*r, rows, heads, kv_heads, kMaxBwdWgs, a);
  }
  // (no rows: no partial sums to add, zeros)
  const hipError_t e = timed(kKQkRotate, stream, [&] {
    return launch_rotate_bwd(a, r->head_dim, dtype == BDLM_BF16, r->interleaved, stream);
  });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "rotation backward launch");
}

}  // extern "C"
