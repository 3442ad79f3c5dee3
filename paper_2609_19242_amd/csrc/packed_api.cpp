// C ABI of packed attention: argument validation, the plan, launches.
// Declarations and contracts: include/bdlm_attn.h.
#include "bdlm_attn.h"

#include <cmath>
#include <cstring>
#include <exception>

#include "api_util.hpp"
#include "packed.hpp"
#include "packed_plan.hpp"

using namespace bdlm;

namespace {

constexpr int64_t kMaxLen = (int64_t)1 << 28;     // rows of a tensor
constexpr int64_t kMaxStride = (int64_t)1 << 20;  // elements between rows: a tile's offsets stay below 2^31 bytes

bdlm_status check_packed(const bdlm_packed* p) {
  if (!p) return fail(BDLM_ERR_INVALID, "packed problem is null");
  if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads != 0)
    return fail(BDLM_ERR_INVALID, "heads (%d) must be a positive multiple of kv_heads (%d)", p->heads, p->kv_heads);
  if (p->head_dim != 64 && p->head_dim != 128)
    return fail(BDLM_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", p->head_dim);
  if (p->heads > kMaxStride / p->head_dim)
    return fail(BDLM_ERR_UNSUPPORTED, "heads (%d) x head_dim exceeds %lld", p->heads, (long long)kMaxStride);
  if (p->dtype != BDLM_BF16 && p->dtype != BDLM_F32)
    return fail(BDLM_ERR_UNSUPPORTED, "dtype %d not supported", p->dtype);
  if (!std::isfinite(p->scale)) return fail(BDLM_ERR_INVALID, "scale is not finite");
  if (p->scale > 0.f && p->scale < kMinScheduledScale)
    return fail(BDLM_ERR_UNSUPPORTED, "scale %g is below 2^-96", (double)p->scale);
  if (p->sinks < 0 || p->sinks > kMaxLen) return fail(BDLM_ERR_INVALID, "sinks must be in [0, 2^28] (got %d)", p->sinks);
  if (p->block_size < 1 || p->block_size > kMaxLen)
    return fail(BDLM_ERR_INVALID, "block_size must be in [1, 2^28] (got %lld)", (long long)p->block_size);
  if (p->window < 0 || p->window > kMaxLen)
    return fail(BDLM_ERR_INVALID, "window must be in [0, 2^28] (got %lld)", (long long)p->window);
  return BDLM_OK;
}

bdlm_status check_seqs(int64_t n, const bdlm_packed_seq* s, int64_t& q_rows, int64_t& k_rows) {
  if (n < 0 || n > kMaxLen) return fail(BDLM_ERR_INVALID, "number of sequences %lld outside [0, 2^28]", (long long)n);
  if (n > 0 && !s) return fail(BDLM_ERR_INVALID, "sequences are null");
  int64_t qe = 0, ke = 0;
  for (int64_t i = 0; i < n; ++i) {
    if (s[i].q_len < 0 || s[i].k_len < 0 || s[i].q_start < 0 || s[i].k_start < 0)
      return fail(BDLM_ERR_INVALID, "sequence %lld: negative start or length", (long long)i);
    if (s[i].q_len > kMaxLen || s[i].k_len > kMaxLen || s[i].q_start > kMaxLen - s[i].q_len ||
        s[i].k_start > kMaxLen - s[i].k_len)
      return fail(BDLM_ERR_UNSUPPORTED, "sequence %lld: rows past 2^28", (long long)i);
    // in order and apart: no row belongs to two sequences
    if ((s[i].q_len > 0 && s[i].q_start < qe) || (s[i].k_len > 0 && s[i].k_start < ke))
      return fail(BDLM_ERR_INVALID, "sequence %lld: its rows must start behind the rows of the sequences before it",
                  (long long)i);
    if (s[i].q_len > 0) qe = s[i].q_start + s[i].q_len;
    if (s[i].k_len > 0) ke = s[i].k_start + s[i].k_len;
  }
  q_rows = qe;
  k_rows = ke;
  return BDLM_OK;
}

bdlm_status check_rows(const bdlm_rows& r, const char* what, bool used, int64_t row_elems, int elem) {
  if (!used) return BDLM_OK;
  if (!r.ptr) return fail(BDLM_ERR_INVALID, "%s pointer is null", what);
  if (!aligned16(r.ptr)) return fail(BDLM_ERR_INVALID, "%s pointer is not 16-byte aligned", what);
  if (r.stride < row_elems) return fail(BDLM_ERR_INVALID, "%s row stride %lld below heads x head_dim = %lld", what,
                                        (long long)r.stride, (long long)row_elems);
  if (r.stride > kMaxStride)
    return fail(BDLM_ERR_UNSUPPORTED, "%s row stride %lld above 2^20", what, (long long)r.stride);
  if (r.stride * elem % 16 != 0)
    return fail(BDLM_ERR_INVALID, "%s row stride %lld is not a multiple of 16 bytes", what, (long long)r.stride);
  return BDLM_OK;
}

size_t packed_stats_bytes(const bdlm_packed_plan& pl) {
  return align256((size_t)pl.q_rows * pl.problem.heads * sizeof(float));
}

bdlm_status check_workspace(size_t need, const void* p, size_t bytes) {
  if (need > 0 && (!p || bytes < need || (reinterpret_cast<uintptr_t>(p) & 255u)))
    return fail(BDLM_ERR_WORKSPACE, "workspace needs %zu bytes, 256-byte aligned (got %zu at %p)", need, bytes, p);
  return BDLM_OK;
}

// Partial outputs of the forward's cut walks; their LSE lies behind them.
size_t part_bytes(const bdlm_packed_plan& pl) {
  const int per = pl.problem.heads / packed_tile_heads(pl.problem.heads / pl.problem.kv_heads);
  return align256((size_t)pl.fwd.slots * per * kQRowsShortBf16 * pl.problem.head_dim * sizeof(float));
}

bdlm_status check_plan(const bdlm_packed_plan* pl, const void* items) {
  if (!pl) return fail(BDLM_ERR_INVALID, "plan is null");
  const bdlm_status st = check_packed(&pl->problem);
  if (st != BDLM_OK) return st;
  auto bad = [](const bdlm_packed_chunks& c) { return c.items < 0 || c.sums < 0 || c.slots < 0 || c.reserved != 0; };
  if (pl->q_items < 0 || pl->k_items < 0 || pl->n_sums < 0 || pl->slots < 0 || bad(pl->fwd) || bad(pl->dq) ||
      pl->reserved != 0 || pl->q_rows < 0 || pl->k_rows < 0 ||
      pl->teams < 1 || pl->teams > 2)
    return fail(BDLM_ERR_INVALID, "plan was not made by bdlm_packed_plan_make");
  if (pl->bytes > 0 && (!items || !aligned16(items)))
    return fail(BDLM_ERR_INVALID, "plan items are null or not 16-byte aligned");
  return BDLM_OK;
}

PackedArgs packed_args(const bdlm_packed_plan& pl, int64_t lse_pitch) {
  const bdlm_packed& p = pl.problem;
  PackedArgs a{};
  a.heads = p.heads;
  a.kv_heads = p.kv_heads;
  a.group = p.heads / p.kv_heads;
  a.M = (int32_t)p.block_size;
  a.window = (int32_t)p.window;
  a.sinks = p.sinks;
  a.scale = p.scale > 0.f ? p.scale : 1.0f / std::sqrt((float)p.head_dim);
  a.scale_log2 = a.scale * 1.44269504088896340736f;
  a.q_rows = (int32_t)lse_pitch;
  a.stats_form = p.dtype == BDLM_BF16 ? 1 : 0;
  return a;
}

// The chunks of query tiles in place of the whole ones, if there are any (a.items: the plan's).
void take_chunks(const bdlm_packed_plan& pl, bool dq, PackedArgs& a) {
  const bdlm_packed_chunks& c = dq ? pl.dq : pl.fwd;
  if (c.items == 0) return;
  auto behind = [](const PackedItem* items, int n_items, int n_sums) {  // items, then sums
    return reinterpret_cast<const PackedItem*>(reinterpret_cast<const PackedSum*>(items + n_items) + n_sums);
  };
  a.items = behind(a.items, pl.q_items + pl.k_items, pl.n_sums);
  if (dq) a.items = behind(a.items, pl.fwd.items, pl.fwd.sums);
  a.n_items = c.items;
  a.sums = reinterpret_cast<const PackedSum*>(a.items + c.items);
  a.n_sums = c.sums;
}

// bf16(a) or f32(a), as a call with sinks if it has some.
template <class SinksBf16, class SinksF32, class F, class G>
hipError_t launch_as(const PackedArgs& a, int32_t dtype, F&& bf16, G&& f32) {
  if (dtype == BDLM_BF16) return a.sinks > 0 ? bf16(SinksBf16{a}) : bf16(a);
  return a.sinks > 0 ? f32(SinksF32{a}) : f32(a);
}

bdlm_status check_pitch(const bdlm_packed_plan& pl, int64_t pitch) {
  if (pitch < pl.q_rows || pitch > kMaxLen)
    return fail(BDLM_ERR_INVALID, "lse pitch %lld outside [%lld, 2^28]", (long long)pitch, (long long)pl.q_rows);
  return BDLM_OK;
}

}  // namespace

extern "C" {

bdlm_status bdlm_packed_plan_make(const bdlm_packed* p, int64_t n_seqs, const bdlm_packed_seq* seqs, void* items,
                                  size_t items_bytes, bdlm_packed_plan* plan) try {
  if (!plan) return fail(BDLM_ERR_INVALID, "plan is null");
  bdlm_status st;
  if ((st = check_packed(p)) != BDLM_OK) return st;
  int64_t q_rows = 0, k_rows = 0;
  if ((st = check_seqs(n_seqs, seqs, q_rows, k_rows)) != BDLM_OK) return st;
  bdlm_packed problem = *p;
  if (problem.window == 0) problem.sinks = 0;  // (every earlier key is visible)
  const PackedPlanItems it = packed_items(problem, n_seqs, seqs);
  // (a grid dimension holds fewer than 2^32 threads; the fp32 kernels' grids have two)
  const bool f32 = p->dtype == BDLM_F32;
  const int64_t per = p->heads / (f32 ? 1 : packed_tile_heads(p->heads / p->kv_heads));
  const int64_t q_wgs = (int64_t)std::max({it.q.size(), it.fwd.items.size(), it.dq.items.size()}) * per;
  const int64_t wgs = std::max(q_wgs, (int64_t)it.k.size() * p->kv_heads), most = f32 ? (int64_t)1 << 30 : 1 << 22;
  if (wgs > most || (int64_t)it.sums.size() * p->kv_heads > 1 << 18 || (int64_t)std::max(it.fwd.sums.size(), it.dq.sums.size()) * per > 1 << 18)
    return fail(BDLM_ERR_UNSUPPORTED, "packed problem needs %lld workgroups (limit %lld)", (long long)wgs,
                (long long)most);
  bdlm_packed_plan pl{};
  pl.problem = problem;
  pl.q_rows = q_rows;
  pl.k_rows = k_rows;
  pl.q_items = (int32_t)it.q.size();
  pl.k_items = (int32_t)it.k.size();
  pl.n_sums = (int32_t)it.sums.size();
  pl.slots = it.slots;
  pl.teams = it.teams;
  auto put_chunks = [](const PackedPlanItems::Chunks& c, bdlm_packed_chunks& to) {
    to = {(int32_t)c.items.size(), (int32_t)c.sums.size(), c.slots, 0};
  };
  put_chunks(it.fwd, pl.fwd);
  put_chunks(it.dq, pl.dq);
  pl.bytes = (it.q.size() + it.k.size() + it.fwd.items.size() + it.dq.items.size()) * sizeof(PackedItem) +
             (it.sums.size() + it.fwd.sums.size() + it.dq.sums.size()) * sizeof(PackedSum);
  const size_t part_rows = (size_t)it.fwd.slots * per * kQRowsShortBf16;
  pl.fwd_workspace_bytes = align256(part_rows * p->head_dim * sizeof(float)) + align256(part_rows * sizeof(float));
  // (dQ's partial sums are added up before the first of dK and dV are written: in the same place)
  pl.workspace_bytes = 2 * packed_stats_bytes(pl) +
                       std::max((size_t)it.slots * p->kv_heads *
                                    (f32 ? kRowsF32 * sizeof(double) : kBwdKeysBf16 * sizeof(float)) * 2 * p->head_dim,
                                (size_t)it.dq.slots * per * kQRowsShortBf16 * p->head_dim * sizeof(float));
  if (items) {
    if (items_bytes < pl.bytes)
      return fail(BDLM_ERR_INVALID, "plan needs %zu bytes (got %zu)", pl.bytes, items_bytes);
    char* dst = static_cast<char*>(items);
    auto put = [&](const auto& v) {
      if (!v.empty()) std::memcpy(dst, v.data(), v.size() * sizeof(v[0]));
      dst += v.size() * sizeof(v[0]);
    };
    put(it.q);
    put(it.k);
    put(it.sums);
    for (const PackedPlanItems::Chunks* c : {&it.fwd, &it.dq}) {
      put(c->items);
      put(c->sums);
    }
  }
  *plan = pl;
  return BDLM_OK;
} catch (const std::exception& e) {
  return fail(BDLM_ERR_INVALID, "packed plan: %s", e.what());
}

bdlm_status bdlm_packed_fwd(const bdlm_packed_plan* plan, const void* items, bdlm_rows q, bdlm_rows k, bdlm_rows v,
                            bdlm_rows o, float* lse, int64_t lse_pitch, void* workspace, size_t workspace_bytes,
                            hipStream_t stream) {
  bdlm_status st;
  if ((st = check_plan(plan, items)) != BDLM_OK) return st;
  const bdlm_packed& p = plan->problem;
  const int elem = p.dtype == BDLM_F32 ? 4 : 2;
  const int64_t qe = (int64_t)p.heads * p.head_dim, ke = (int64_t)p.kv_heads * p.head_dim;
  const bool rows = plan->q_items > 0, keys = rows && plan->k_rows > 0;
  if ((st = check_rows(q, "q", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_rows(k, "k", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_rows(v, "v", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_rows(o, "o", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_pitch(*plan, lse_pitch)) != BDLM_OK) return st;
  if (rows && !lse) return fail(BDLM_ERR_INVALID, "lse pointer is null");
  if ((st = check_workspace(plan->fwd_workspace_bytes, workspace, workspace_bytes)) != BDLM_OK) return st;
  PackedArgs a = packed_args(*plan, lse_pitch);
  a.items = static_cast<const PackedItem*>(items);
  a.n_items = plan->q_items;
  take_chunks(*plan, false, a);
  if (a.n_sums > 0) {
    a.partials = workspace;
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + part_bytes(*plan));
  }
  a.q = q.ptr;
  a.qs = (int32_t)q.stride;
  a.k = k.ptr;
  a.ks = (int32_t)k.stride;
  a.v = v.ptr;
  a.vs = (int32_t)v.stride;
  a.o = o.ptr;
  a.os = (int32_t)o.stride;
  a.lse = lse;
  const hipError_t e = timed(kKPackedFwd, stream, [&] {
    const hipError_t le = launch_as<SinkQArgs, SinkQArgsF32>(
        a, p.dtype, [&](const auto& c) { return launch_fwd_bf16(c, p.head_dim, plan->teams, stream); },
        [&](const auto& c) { return launch_fwd_f32(c, p.head_dim, stream); });
    return le != hipSuccess || a.n_sums == 0 ? le : launch_packed_fwd_sum(a, p.head_dim, plan->fwd.slots, stream);
  });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "packed forward launch");
}

bdlm_status bdlm_packed_bwd(const bdlm_packed_plan* plan, const void* items, bdlm_rows q, bdlm_rows k, bdlm_rows v,
                            bdlm_rows o, const float* lse, int64_t lse_pitch, bdlm_rows dO, bdlm_rows dq, bdlm_rows dk,
                            bdlm_rows dv, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  bdlm_status st;
  if ((st = check_plan(plan, items)) != BDLM_OK) return st;
  const bdlm_packed& p = plan->problem;
  const int elem = p.dtype == BDLM_F32 ? 4 : 2;
  const int64_t qe = (int64_t)p.heads * p.head_dim, ke = (int64_t)p.kv_heads * p.head_dim;
  const bool rows = plan->q_items > 0, keys = plan->k_items > 0;
  if ((st = check_rows(q, "q", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_rows(k, "k", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_rows(v, "v", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_rows(o, "o", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_rows(dO, "dO", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_rows(dq, "dq", rows, qe, elem)) != BDLM_OK) return st;
  if ((st = check_rows(dk, "dk", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_rows(dv, "dv", keys, ke, elem)) != BDLM_OK) return st;
  if ((st = check_pitch(*plan, lse_pitch)) != BDLM_OK) return st;
  if (rows && !lse) return fail(BDLM_ERR_INVALID, "lse pointer is null");
  if (plan->q_rows * p.heads > ((int64_t)1 << 28))
    return fail(BDLM_ERR_UNSUPPORTED, "query rows x heads = %lld exceeds 2^28", (long long)(plan->q_rows * p.heads));
  const size_t need = plan->workspace_bytes, arr = packed_stats_bytes(*plan);
  if ((st = check_workspace(need, workspace, workspace_bytes)) != BDLM_OK) return st;
  PackedArgs a = packed_args(*plan, lse_pitch);
  a.q = q.ptr;
  a.qs = (int32_t)q.stride;
  a.k = k.ptr;
  a.ks = (int32_t)k.stride;
  a.v = v.ptr;
  a.vs = (int32_t)v.stride;
  a.o = o.ptr;
  a.os = (int32_t)o.stride;
  a.lse = const_cast<float*>(lse);
  a.dO = dO.ptr;
  a.dos = (int32_t)dO.stride;
  a.dq = dq.ptr;
  a.dqs = (int32_t)dq.stride;
  a.dk = dk.ptr;
  a.dks = (int32_t)dk.stride;
  a.dv = dv.ptr;
  a.dvs = (int32_t)dv.stride;
  char* ws = static_cast<char*>(workspace);
  a.l2 = reinterpret_cast<float*>(ws);
  a.delta = reinterpret_cast<float*>(ws + arr);
  a.partials = ws + 2 * arr;
  a.items = static_cast<const PackedItem*>(items);
  a.n_items = plan->q_items;
  take_chunks(*plan, true, a);
  // dQ first: it leaves the row statistics for dK/dV.
  hipError_t e = timed(kKPackedDq, stream, [&] {
    const hipError_t le = launch_as<SinkQArgs, SinkQArgsF32>(
        a, p.dtype, [&](const auto& c) { return launch_bwd_dq_bf16(c, p.head_dim, stream); },
        [&](const auto& c) { return launch_bwd_dq_f32(c, p.head_dim, stream); });
    return le != hipSuccess || a.n_sums == 0 ? le : launch_packed_dq_sum(a, p.head_dim, stream);
  });
  if (e != hipSuccess) return hip_fail(e, "packed dQ launch");
  a.items = static_cast<const PackedItem*>(items) + plan->q_items;
  a.n_items = plan->k_items;
  a.sums = reinterpret_cast<const PackedSum*>(a.items + plan->k_items);
  a.n_sums = plan->n_sums;
  e = timed(kKPackedDkDv, stream, [&] {
    hipError_t le = launch_as<SinkKArgs, SinkKArgs>(
        a, p.dtype, [&](const auto& c) { return launch_bwd_dkdv(c, p.head_dim, stream); },
        [&](const auto& c) { return launch_bwd_dkv_f32(c, p.head_dim, stream); });
    if (le != hipSuccess || a.n_sums == 0) return le;
    return p.dtype == BDLM_BF16 ? launch_bwd_dkdv_sum(a, p.head_dim, stream) : launch_bwd_sum_f32(a, p.head_dim, stream);
  });
  return e == hipSuccess ? BDLM_OK : hip_fail(e, "packed dK/dV launch");
}

}  // extern "C"
