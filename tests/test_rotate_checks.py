"""Rotated queries and keys on the CPU: the oracle's gradient against differences and its rotation against products of
complex numbers; what the records of rotations hold; refusals by the binding and the C ABI."""
import ctypes
import math

import pytest
import torch

import paper_2609_19242_amd as bd
from paper_2609_19242_amd import packed as pm
from paper_2609_19242_amd import rotate as rm
from tests import rotate_oracle as ro

BF, F32 = torch.bfloat16, torch.float32
FAKE = 0x10000  # never dereferenced: these calls fail validation first
host_only = pytest.mark.skipif(torch.cuda.device_count() > 0,
                               reason="passes unmapped pointers that validation must reject; host-only test")


# ------------------------------------------------------------------ the oracle
@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_rotation_is_a_complex_product(interleaved):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 2, 64, generator=g, dtype=torch.float64)
    t = torch.randn(5, 1, 16, generator=g, dtype=torch.float64) * 100
    y = ro.turned(x, t, interleaved)
    re, im = (x[..., 0:32:2], x[..., 1:32:2]) if interleaved else (x[..., :16], x[..., 16:32])
    z = torch.complex(re.contiguous(), im.contiguous()) * torch.polar(torch.ones_like(t), t)
    yr, yi = (y[..., 0:32:2], y[..., 1:32:2]) if interleaved else (y[..., :16], y[..., 16:32])
    assert torch.allclose(yr, z.real, rtol=0, atol=1e-13) and torch.allclose(yi, z.imag, rtol=0, atol=1e-13)
    assert torch.equal(y[..., 32:], x[..., 32:])


@pytest.mark.parametrize("eps", [None, 1e-6, 0.5])
def test_oracle_gradient_against_differences(eps):
    g = torch.Generator().manual_seed(2)
    x, dy, step = (torch.randn(3, 2, 64, generator=g, dtype=F32) for _ in range(3))
    w, wstep = (torch.randn(64, generator=g, dtype=F32) for _ in range(2))
    if eps is None:
        w = None
    t = torch.randn(3, 1, 24, generator=g, dtype=torch.float64)
    ref = ro.backward(x, w, t, eps, True, dy)

    def f(a, b):  # the forward in 64 bits
        ww = torch.ones(64, dtype=torch.float64) if w is None else w.double() + b * wstep.double()
        xx = x.double() + a * step.double()
        n = xx if eps is None else xx / torch.sqrt((xx * xx).mean(-1, keepdim=True) + eps) * ww
        return float((ro.turned(n, t, True) * dy).sum())

    h = 1e-5  # differences are off by h^2 times a third derivative and 1e-16 / h
    assert abs((f(h, 0) - f(-h, 0)) / (2 * h) - float((ref["dx"][0] * step).sum())) < 1e-7
    if eps is not None:
        assert abs((f(0, h) - f(0, -h)) / (2 * h) - float((ref["dw"][0] * wstep).sum())) < 1e-7


# ------------------------------------------------------------------ records
def test_ladders_and_axes():
    r = bd.rotary(128)
    assert r.dim == 128 and r.axes == 1 and r.pair_axes == [0] * 64
    assert r.freqs == [10000.0 ** (-i / 64) for i in range(64)]
    r = bd.rotary(128, sections=(16, 24, 24), base=1e6)
    assert r.pair_axes == [0] * 16 + [1] * 24 + [2] * 24 and r.freqs == [1e6 ** (-i / 64) for i in range(64)]
    r = bd.rotary(64, dim=32, sections=(4, 12), own_ladders=True, interleaved=True)
    assert r.freqs == [10000.0 ** (-j / 4) for j in range(4)] + [10000.0 ** (-j / 12) for j in range(12)]
    assert bd.rotary(64, dim=16, freqs=range(8)).freqs == list(range(8))
    assert bd.rotary(64, sections=(0, 32)).pair_axes == [1] * 32


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(dim=0), dict(dim=24), dict(dim=144), dict(sections=(16, 16)),
                                dict(sections=(65, -1)), dict(sections=()), dict(sections=(13, 13, 13, 13, 12)), dict(base=0),
                                dict(base=math.inf), dict(base=math.nan), dict(freqs=[1.0] * 63), dict(freqs=[math.nan] * 64),
                                dict(freqs=[math.inf] * 64), dict(freqs=[2.0 ** 21] * 64)])
def test_rotations_that_are_refused(kw):
    with pytest.raises(ValueError):
        bd.rotary(**dict(dict(head_dim=128), **kw))


# ------------------------------------------------------------------ refusals
def args(n=6, H=4, KV=2, D=64, dtype=BF, axes=1):
    rot = bd.rotary(D, sections=[D // 2 // axes] * axes)
    pos = torch.zeros((n,) if axes == 1 else (axes, n), dtype=torch.int32)
    return dict(rot=rot, q=torch.zeros(n, H, D, dtype=dtype), k=torch.zeros(n, KV, D, dtype=dtype), positions=pos,
                q_weight=torch.ones(D, dtype=dtype), k_weight=torch.ones(D, dtype=dtype), eps=1e-6)


def test_calls_need_a_gpu():
    a = args()
    with pytest.raises(ValueError, match="GPU"):
        bd.qk_rotate_fwd(**a)
    with pytest.raises(ValueError, match="GPU"):
        bd.qk_rotate_bwd(**a, dq_out=a["q"], dk_out=a["k"])


@pytest.mark.parametrize("change,err,what", [
    (dict(rot=None), TypeError, "Rotary"), (dict(q=None), ValueError, "q must"), (dict(q=torch.zeros(6, 256, dtype=BF)), ValueError, "q must"),
    (dict(q=torch.zeros(6, 4, 64, dtype=torch.half)), TypeError, "dtype"), (dict(q=torch.zeros(6, 4, 128, dtype=BF)), ValueError, "shape"),
    (dict(q=torch.zeros(64, 4, 6, dtype=BF).transpose(0, 2)), ValueError, "contiguously"),
    (dict(k=torch.zeros(6, 2, 64)), TypeError, "k must be"), (dict(k=torch.zeros(5, 2, 64, dtype=BF)), ValueError, "rows"),
    (dict(k=torch.zeros(7, 2, 64, dtype=BF)), ValueError, "6 rows"), (dict(k=None), ValueError, "k must"),
    (dict(positions=torch.zeros(6)), TypeError, "int32"), (dict(positions=torch.zeros(6, dtype=torch.int64)), TypeError, "int32"),
    (dict(positions=torch.zeros(5, dtype=torch.int32)), ValueError, "shape"), (dict(positions=None), ValueError, "positions"),
    (dict(positions=torch.zeros(2, 6, dtype=torch.int32)), ValueError, "shape"),
    (dict(positions=torch.zeros(12, dtype=torch.int32)[::2]), ValueError, "contiguous"),
    (dict(eps=0.0), ValueError, "eps"), (dict(eps=-1.0), ValueError, "eps"), (dict(eps=math.nan), ValueError, "eps"),
    (dict(eps=math.inf), ValueError, "eps"), (dict(eps=1e-40), ValueError, "eps"), (dict(eps=None), ValueError, "needs a norm"),
    (dict(q_weight=torch.ones(64)), TypeError, "q_weight"), (dict(k_weight=torch.ones(32, dtype=BF)), ValueError, "k_weight"),
])
def test_both_directions_refuse(change, err, what):
    a = dict(args(), **change)
    with pytest.raises(err, match=what):
        bd.qk_rotate_fwd(**a)
    with pytest.raises(err, match=what):
        bd.qk_rotate_bwd(**a, dq_out=torch.zeros(6, 4, 64, dtype=BF), dk_out=torch.zeros(6, 2, 64, dtype=BF))


def test_outputs_and_gradients_are_checked():
    a = args()
    q, k = a["q"], a["k"]
    for out, err in (((q,), ValueError), ((q, q), ValueError), ((q.float(), k), TypeError), ((q[:5], k), ValueError)):
        with pytest.raises(err):
            bd.qk_rotate_fwd(**a, out=out)
        with pytest.raises(err):
            bd.qk_rotate_bwd(**a, dq_out=q, dk_out=k, out=out)
    with pytest.raises(TypeError, match="dq_out"):
        bd.qk_rotate_bwd(**a, dq_out=q.float(), dk_out=k)
    with pytest.raises(ValueError, match="dk_out"):
        bd.qk_rotate_bwd(**a, dq_out=q, dk_out=k[:5])
    three = args(axes=2)
    with pytest.raises(ValueError, match="positions"):
        bd.qk_rotate_fwd(**dict(three, positions=torch.zeros(6, dtype=torch.int32)))


GOOD = dict(dtype=bd.BF16, rows=6, pos=FAKE, heads=4, kv=2, q=FAKE, qs=256, k=FAKE, ks=128, qw=FAKE, kw=FAKE, eps=1e-6, o=FAKE,
            os=256, dqw=FAKE, dkw=FAKE, ws=FAKE, nb=1 << 30)


def call(record=None, bwd=False, **kw):
    x, R = dict(GOOD, **kw), pm._Rows
    head = (ctypes.byref(record or bd.rotary(64)._record), x["dtype"], x["rows"], x["pos"], x["heads"], x["kv"], R(x["q"], x["qs"]),
            R(x["k"], x["ks"]), x["qw"], x["kw"], x["eps"])
    if not bwd:
        return bd.lib().bdlm_qk_rotate_fwd(*head, R(x["o"], x["os"]), R(FAKE, 128), None)
    return bd.lib().bdlm_qk_rotate_bwd(*head, R(FAKE, 256), R(FAKE, 128), R(x["o"], x["os"]), R(FAKE, 128), x["dqw"], x["dkw"],
                                       x["ws"], x["nb"], None)


@host_only
@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), -2), (dict(rows=-1), -1), (dict(rows=1 << 29), -1), (dict(pos=0), -1), (dict(pos=FAKE + 2), -1), (dict(heads=0), -1),
    (dict(kv=0), -1), (dict(q=0), -1), (dict(q=FAKE + 8), -1), (dict(qs=255), -1), (dict(qs=260), -1), (dict(qs=(1 << 30) + 8), -1),
    (dict(ks=64), -1), (dict(qw=FAKE + 4), -1), (dict(eps=0.0), -1), (dict(eps=-1.0), -1), (dict(eps=math.nan), -1),
    (dict(eps=math.inf), -1), (dict(eps=1e-40), -1), (dict(eps=1e40), -1), (dict(o=0), -1), (dict(os=128), -1)])
def test_the_c_abi_refuses(kw, status):
    assert call(**kw) == status and call(bwd=True, **kw) == status
    assert bd.lib().bdlm_last_error()


@host_only
@pytest.mark.parametrize("kw", [dict(head_dim=32), dict(dim=8), dict(dim=80), dict(interleaved=2), dict(axes=0), dict(axes=5)])
def test_the_c_abi_refuses_rotations(kw):
    r = bd.rotary(64)._record
    for n, v in kw.items():
        setattr(r, n, v)
    assert call(r) < 0 and call(r, bwd=True) < 0
    r = bd.rotary(64)._record
    r.axis[31] = 1
    assert call(r) == -1
    r.axis[31], r.freq[31] = 0, math.nan
    assert call(r) == -1
    assert bd.lib().bdlm_qk_rotate_fwd(None, 0, 0, None, 1, 1, pm._Rows(0, 0), pm._Rows(0, 0), None, None, 0.0, pm._Rows(0, 0),
                                       pm._Rows(0, 0), None) == -1


@host_only
def test_the_c_abi_refuses_workspaces():
    need = bd.lib().bdlm_qk_rotate_workspace_bytes(64)
    assert need > 0 and bd.lib().bdlm_qk_rotate_workspace_bytes(96) == 0
    for ws, nb in ((0, need), (FAKE, need - 1), (FAKE + 128, need)):
        assert call(bwd=True, ws=ws, nb=nb) == -4
    assert call(bwd=True, dqw=FAKE + 2) == -1
    assert call(bwd=True, eps=0.0, qw=None, kw=None) == -1  # a weight's gradient without a norm
    assert call(rows=0, pos=0, q=0, o=0) == 0  # nothing to do


def test_new_outputs_of_a_given_stream(monkeypatch):
    """They come from that stream's memory and are kept for the current one too."""
    import contextlib
    at, new, kept = ["current"], [], []

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    for owner, name in ((torch, "empty"), (torch, "empty_like"), (torch.Tensor, "new_empty")):
        plain = getattr(owner, name)
        monkeypatch.setattr(owner, name, lambda *a, plain=plain, **kw: new.append((plain(*a, **kw), at[-1])) or new[-1][0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t, s)))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at[-1])
    monkeypatch.setattr(bd, "_torch_stream", lambda s, device: s)
    monkeypatch.setattr(rm, "_launch", lambda *a: None)
    a = args()
    res = bd.qk_rotate_fwd(**a, stream="side")
    assert len(new) == 2 and all(s == "side" for _, s in new) and all(any(r is t and s == "current" for t, s in kept) for r in res)
    new.clear()
    res = bd.qk_rotate_bwd(**a, dq_out=a["q"], dk_out=a["k"], stream="side")
    assert len(new) == 5 and all(s == "side" for _, s in new) and all(any(r is t and s == "current" for t, s in kept) for r in res)
