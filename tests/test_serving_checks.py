"""Refusals of packed attention, the cache's operations and attention over the cache: by the binding, for tensors of the
wrong type, shape, layout or device, and by the C ABI, for numbers and pointers out of contract.  Host only: every call
here fails before anything is launched."""
import ctypes
import math

import pytest
import torch

import paper_2609_19242_amd as bd
from paper_2609_19242_amd import cache as cm
from paper_2609_19242_amd import packed as pm

BF, F32 = torch.bfloat16, torch.float32
FAKE = 0x10000  # never dereferenced: these calls fail validation first
host_only = pytest.mark.skipif(torch.cuda.device_count() > 0,
                               reason="passes unmapped pointers that validation must reject; host-only test")


def plan(ql=(5, 3), kl=None, **kw):
    kw = dict(dict(heads=4, kv_heads=2, head_dim=64, dtype=BF, device="cpu"), **kw)
    return bd.packed_plan(ql if isinstance(ql, torch.Tensor) else list(ql), None if kl is None else list(kl), **kw)


# ------------------------------------------------------------------ plans
@pytest.mark.parametrize("kw,what", [
    (dict(heads=3), "multiple of kv_heads"), (dict(kv_heads=0), "multiple of kv_heads"), (dict(head_dim=96), "head_dim"),
    (dict(block_size=0), "block_size"), (dict(block_size=1 << 40), "block_size"), (dict(window=-1), "window"),
    (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"), (dict(scale=1e-38), "2\\^-96"),
    (dict(ql=[-1]), "negative"), (dict(ql=[4], kl=[-4]), "negative"), (dict(ql=[3, 3], q_starts=[0, 2]), "behind"),
    (dict(ql=[3, 3], q_starts=[5, 0]), "behind"), (dict(ql=[3, 3], q_starts=[0, 3], k_starts=[0, 1]), "behind"),
    (dict(ql=[1 << 40]), "2\\^28"), (dict(ql=[3], q_starts=[1 << 40]), "2\\^28"), (dict(ql=[3], q_starts=[-1]), "negative"),
    (dict(heads=40000, kv_heads=20000), "exceeds"), (dict(dtype=torch.float16), "dtype"),
    (dict(ql=[3, 4], kl=[3]), "2 sequences"), (dict(ql=[3, 4], q_starts=[3]), "2 sequences"),
])
def test_plans_refuse(kw, what):
    with pytest.raises((bd.BdlmError, ValueError, TypeError), match=what):
        plan(**kw)


def test_plans_take_lists_and_cpu_tensors():
    a, b = plan([5, 0, 7]), plan(torch.tensor([5, 0, 7]))
    assert a.q_rows == b.q_rows == 12 and a.k_rows == 12
    with pytest.raises(ValueError, match="integer"):
        plan(torch.tensor([5.0]))
    with pytest.raises(TypeError):
        plan([5.5])
    assert plan([]).q_rows == 0 and plan([0, 0]).k_rows == 0
    assert plan([3, 4], q_starts=[2, 9]).q_rows == 13


def test_many_workgroups_are_refused():
    with pytest.raises(bd.BdlmError, match="workgroups"):
        plan([1] * 600000, heads=64, kv_heads=64)


# ------------------------------------------------------------------ packed calls
def tensors(n=8, H=4, KV=2, D=64, dtype=BF):
    return (torch.zeros(n, H, D, dtype=dtype), torch.zeros(n, KV, D, dtype=dtype), torch.zeros(n, KV, D, dtype=dtype))


def test_packed_calls_need_a_gpu():
    with pytest.raises(ValueError, match="GPU"):
        bd.packed_fwd(plan(), *tensors())


@pytest.mark.parametrize("change,err,what", [
    (lambda q, k, v: (q.float(), k, v), TypeError, "q must be torch.bfloat16"),
    (lambda q, k, v: (q, k.half(), v), TypeError, "k must be"), (lambda q, k, v: (q[:7], k, v), ValueError, "q has 7 rows"),
    (lambda q, k, v: (q, k[:2], v), ValueError, "k has 2 rows"), (lambda q, k, v: (q[:, :2], k, v), ValueError, "shape"),
    (lambda q, k, v: (q, k, v[..., :32]), ValueError, "shape"), (lambda q, k, v: (q[None], k, v), ValueError, "shape"),
    (lambda q, k, v: (q.transpose(1, 2).contiguous().transpose(1, 2), k, v), ValueError, "contiguously"),
    (lambda q, k, v: (q[:1].expand(8, 4, 64), k, v), ValueError, "contiguously"), (lambda q, k, v: (None, k, v), TypeError, "q"),
])
def test_packed_fwd_refuses_tensors(change, err, what):
    with pytest.raises(err, match=what):
        bd.packed_fwd(plan(), *change(*tensors()))


def test_packed_outputs_are_checked():
    q, k, v = tensors()
    o, lse = torch.zeros_like(q), torch.zeros(4, 8)
    p = plan()
    with pytest.raises(TypeError, match="plan"):
        bd.packed_fwd(None, q, k, v)
    with pytest.raises(TypeError, match="o must be"):
        bd.packed_fwd(p, q, k, v, out=(o.float(), lse))
    with pytest.raises(ValueError, match="lse must have shape"):
        bd.packed_fwd(p, q, k, v, out=(o, lse.t()))
    with pytest.raises(ValueError, match="o must have 8 rows"):
        bd.packed_fwd(p, q, k, v, out=(torch.zeros(9, 4, 64, dtype=BF), lse))
    with pytest.raises(ValueError, match=r"\(o, lse\)"):
        bd.packed_fwd(p, q, k, v, out=(o,))
    with pytest.raises(TypeError, match="do must be"):
        bd.packed_bwd(p, q, k, v, o, lse, o.float())
    with pytest.raises(ValueError, match="do has 7 rows"):
        bd.packed_bwd(p, q, k, v, o, lse, o[:7])
    with pytest.raises(TypeError, match="lse must be"):
        bd.packed_bwd(p, q, k, v, o, lse.double(), o)
    with pytest.raises(ValueError, match=r"\(dq, dk, dv\)"):
        bd.packed_bwd(p, q, k, v, o, lse, o, out=(q, k))
    with pytest.raises(ValueError, match="dk must have 8 rows"):
        bd.packed_bwd(p, q, k, v, o, lse, o, out=(q, torch.zeros(9, 2, 64, dtype=BF), v))


def _rec(**kw):
    r = plan()._record
    for n, x in kw.items():
        setattr(r, n, x)
    return r


def _fwd(r, q=FAKE, qs=256, k=FAKE, ks=128, o=FAKE, lse=FAKE, pitch=8, items=FAKE):
    R = pm._Rows
    return bd.lib().bdlm_packed_fwd(ctypes.byref(r) if r is not None else None, items, R(q, qs), R(k, ks), R(FAKE, 128),
                                    R(o, 256), lse, pitch, None, 0, None)


@host_only
@pytest.mark.parametrize("kw,status", [
    (dict(q=0), -1), (dict(q=FAKE + 8), -1), (dict(k=0), -1), (dict(o=0), -1), (dict(lse=0), -1), (dict(qs=255), -1),
    (dict(qs=260), -1), (dict(ks=64), -1), (dict(qs=1 << 21), -2), (dict(pitch=7), -1), (dict(pitch=1 << 40), -1),
    (dict(items=0), -1), (dict(items=FAKE + 4), -1)])
def test_the_c_abi_refuses_packed_calls(kw, status):
    assert _fwd(_rec(), **kw) == status
    assert bd.lib().bdlm_last_error()


@host_only
def test_the_c_abi_refuses_plans_and_workspaces():
    assert _fwd(None) == -1
    assert _fwd(_rec(teams=3)) == -1
    assert _fwd(_rec(q_items=-1)) == -1
    R, r = pm._Rows, plan()._record
    a, b = R(FAKE, 256), R(FAKE, 128)

    def bwd(ws, n):
        return bd.lib().bdlm_packed_bwd(ctypes.byref(r), FAKE, a, b, b, a, FAKE, 8, a, a, b, b, ws, n, None)

    assert bwd(0, 1 << 30) == -4 and bwd(FAKE, r.workspace_bytes - 1) == -4 and bwd(FAKE + 128, 1 << 30) == -4
    assert bd.lib().bdlm_packed_plan_make(None, 0, None, None, 0, ctypes.byref(r)) == -1
    p = r.problem
    assert bd.lib().bdlm_packed_plan_make(ctypes.byref(p), 1, None, None, 0, ctypes.byref(r)) == -1
    assert bd.lib().bdlm_packed_plan_make(ctypes.byref(p), 0, None, None, 0, None) == -1
    s = (pm._Seq * 1)(pm._Seq(0, 5, 0, 5))
    buf = ctypes.create_string_buffer(64)
    assert bd.lib().bdlm_packed_plan_make(ctypes.byref(p), 1, s, buf, 1, ctypes.byref(r)) == -1


# ------------------------------------------------------------------ the cache
def cache(**kw):
    d = dict(dict(layers=2, pages=6, page_size=16, kv_heads=2, head_dim=64, seqs=3, max_pages=4, dtype=BF, device="cpu"), **kw)
    return bd.cache_new(**d)


def i32(*xs):
    return torch.tensor(xs, dtype=torch.int32)


def test_cache_tensors_are_checked():
    c = cache()
    parts = dict(k=c.k, v=c.v, table=c.table, lens=c.lens, refs=c.refs, status=c.status)
    assert bd.Cache(**parts).pages == 6
    for name, bad, err in (("k", c.k[0], ValueError), ("k", c.k.half(), TypeError), ("v", c.v.float(), TypeError),
                           ("v", c.v[:, :5], ValueError), ("table", c.table.long(), TypeError), ("table", c.lens, ValueError),
                           ("lens", c.lens[:2], ValueError), ("refs", c.refs[:5], ValueError), ("status", c.lens, ValueError),
                           ("table", c.table.t(), ValueError), ("k", None, ValueError)):
        with pytest.raises(err):
            bd.Cache(**dict(parts, **{name: bad}))


def test_page_operations_refuse_lists():
    c = cache()
    with pytest.raises(ValueError, match="GPU"):
        bd.cache_grow(c, i32(0), i32(1))
    with pytest.raises(TypeError, match="cache"):
        bd.cache_free(None, i32(0))
    with pytest.raises(TypeError, match="int32"):
        bd.cache_free(c, torch.tensor([0]))
    with pytest.raises(TypeError, match="Tensor"):
        bd.cache_free(c, [0])
    with pytest.raises(ValueError, match="shape"):
        bd.cache_grow(c, i32(0, 1), i32(1))
    with pytest.raises(ValueError, match="shape"):
        bd.cache_fork(c, i32(0, 1), i32(1)[None])
    with pytest.raises(ValueError, match="contiguous"):
        bd.cache_free(c, i32(0, 1, 2, 3)[::2])
    k = torch.zeros(4, 2, 64, dtype=BF)
    with pytest.raises(TypeError, match="k must be"):
        bd.cache_write(c, 0, i32(0), i32(4), k.float(), k)
    with pytest.raises(ValueError, match="v has 3"):
        bd.cache_write(c, 0, i32(0), i32(4), k, k[:3])
    with pytest.raises(ValueError, match="shape"):
        bd.cache_write(c, 0, i32(0), i32(4), k, k[..., :32])
    with pytest.raises(ValueError, match="starts"):
        bd.cache_write(c, 0, i32(0), i32(4), k, k, starts=i32(0, 1))


def test_prefix_attn_refuses_tensors():
    c = cache()
    q = torch.zeros(2, 1, 4, 64, dtype=BF)
    with pytest.raises(ValueError, match="GPU"):
        bd.prefix_attn(q, c, 0, i32(0, 1))
    for bad, err in ((q.float(), TypeError), (q[0], ValueError), (q[..., :32], ValueError), (q.transpose(0, 2), ValueError)):
        with pytest.raises(err):
            bd.prefix_attn(bad, c, 0, i32(0, 1))
    with pytest.raises(ValueError, match="seqs"):
        bd.prefix_attn(q, c, 0, i32(0))
    with pytest.raises(ValueError, match="lse must have shape"):
        bd.prefix_attn(q, c, 0, i32(0, 1), out=(q, torch.zeros(2, 1, 4)))
    with pytest.raises(TypeError, match="o must be"):
        bd.prefix_attn(q, c, 0, i32(0, 1), out=(q.float(), torch.zeros(2, 4, 1)))


def crec(**kw):
    r = cm._Cache(*[FAKE] * 7, 2, 6, 16, 3, 4, 2, 64, bd.BF16, 0)
    for n, x in kw.items():
        setattr(r, n, x)
    return r


BAD_CACHES = [(dict(k=0), -1), (dict(v=FAKE + 8), -1), (dict(table=0), -1), (dict(lens=FAKE + 2), -1), (dict(work=0), -1),
              (dict(layers=0), -1), (dict(pages=0), -1), (dict(pages=1 << 30), -1), (dict(page_size=0), -1),
              (dict(page_size=1 << 21), -1), (dict(seqs=0), -1), (dict(seqs=(1 << 19) + 1), -1), (dict(max_pages=0), -1),
              (dict(max_pages=1 << 27), -1), (dict(kv_heads=0), -1), (dict(head_dim=32), -2), (dict(dtype=7), -2),
              (dict(reserved=1), -1)]


@host_only
@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_the_c_abi_refuses_caches(kw, status):
    L, r = bd.lib(), ctypes.byref(crec(**kw))
    rows = pm._Rows(FAKE, 128)
    assert L.bdlm_cache_grow(r, 1, FAKE, FAKE, None) == status
    assert L.bdlm_cache_fork(r, 1, FAKE, FAKE, None) == status
    assert L.bdlm_cache_free(r, 1, FAKE, None) == status
    assert L.bdlm_cache_compact(r, None) == status
    assert L.bdlm_cache_write(r, 0, 1, FAKE, FAKE, None, 4, rows, rows, None) == status
    assert L.bdlm_prefix_attn(r, 0, 1, FAKE, 1, 4, 0, 0, 0.0, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == status
    assert L.bdlm_prefix_attn_workspace_bytes(r, 1, 1, 4, 0) == 0


@host_only
def test_the_c_abi_refuses_page_operations():
    L, c = bd.lib(), crec()
    r = ctypes.byref(c)
    for n, a, b in ((-1, FAKE, FAKE), (4, FAKE, FAKE), (1, 0, FAKE), (1, FAKE, 0), (1, FAKE + 1, FAKE)):
        assert L.bdlm_cache_grow(r, n, a, b, None) == -1
        assert L.bdlm_cache_fork(r, n, a, b, None) == -1
    assert L.bdlm_cache_free(r, 1, 0, None) == -1 and L.bdlm_cache_free(r, 4, FAKE, None) == -1
    ok = dict(layer=0, n=1, seqs=FAKE, counts=FAKE, starts=None, rows=4, k=FAKE, ks=128)
    for kw in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(seqs=0), dict(counts=0), dict(starts=FAKE + 1), dict(rows=-1),
               dict(rows=1 << 30), dict(n=3), dict(k=0), dict(k=FAKE + 8), dict(ks=127), dict(ks=132)):
        x = dict(ok, **kw)
        assert L.bdlm_cache_write(r, x["layer"], x["n"], x["seqs"], x["counts"], x["starts"], x["rows"],
                                  pm._Rows(x["k"], x["ks"]), pm._Rows(FAKE, 128), None) == -1, kw
    assert L.bdlm_cache_work_bytes(0, 1) == 0 and L.bdlm_cache_work_bytes(6, 1 << 20) == 0
    assert L.bdlm_cache_work_bytes(6, 3) == 4 * (16 + 18)


@host_only
def test_the_c_abi_refuses_attention():
    L, c = bd.lib(), crec()
    r = ctypes.byref(c)
    ok = dict(layer=0, R=1, seqs=FAKE, n=1, heads=4, prefix=0, block=0, scale=0.0, q=FAKE, o=FAKE, lse=FAKE, ws=FAKE, nb=1 << 30)

    def call(**kw):
        x = dict(ok, **kw)
        return L.bdlm_prefix_attn(r, x["layer"], x["R"], x["seqs"], x["n"], x["heads"], x["prefix"], x["block"], x["scale"],
                                  x["q"], x["o"], x["lse"], x["ws"], x["nb"], None)

    for kw in (dict(layer=2), dict(R=-1), dict(n=-1), dict(seqs=0), dict(heads=3), dict(heads=0), dict(prefix=-1),
               dict(prefix=65), dict(block=2), dict(scale=math.nan), dict(q=0), dict(q=FAKE + 8), dict(o=0), dict(lse=0)):
        assert call(**kw) == -1, kw
    assert call(R=1 << 20, n=16) == -2 and call(R=1 << 40) == -2
    assert call(R=0) == 0 and call(n=0) == 0  # nothing to do, nothing launched
    big = crec(max_pages=1 << 16)
    need = L.bdlm_prefix_attn_workspace_bytes(ctypes.byref(big), 1, 1, 4, 0)
    assert need > 0
    for ws, nb in ((0, 1 << 30), (FAKE, need - 1), (FAKE + 128, 1 << 30)):
        assert L.bdlm_prefix_attn(ctypes.byref(big), 0, 1, FAKE, 1, 4, 0, 0, 0.0, FAKE, FAKE, FAKE, ws, nb, None) == -4
