"""Norms and rotation of queries and keys against the 64-bit oracle, within derived bounds."""
import pytest
import torch

import paper_2609_19242_amd as bd
from tests import rotate_oracle as ro
from tests.serving_util import check

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


def make(n, H, KV, rot, dtype, seed=0, far=4096, weights=True, fused=False, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    D = rot.head_dim
    rnd = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    if fused:
        qkv = (rnd(n, H + 2 * KV, D) * scale).to(dtype).to(DEV)
        q, k = qkv[:, :H], qkv[:, H:H + KV]
    else:
        q, k = (rnd(n, H, D) * scale).to(dtype).to(DEV), (rnd(n, KV, D) * scale).to(dtype).to(DEV)
    pos = torch.randint(-far, far, (n,) if rot.axes == 1 else (rot.axes, n), generator=g, dtype=torch.int64)
    w = [(1 + 0.3 * rnd(D)).to(dtype).to(DEV) if weights else None for _ in range(2)]
    dy = [rnd(n, h, D).to(dtype).to(DEV) for h in (H, KV)]
    return q, k, pos.clamp(-2 ** 31, 2 ** 31 - 1).to(torch.int32).to(DEV), w, dy


def both(rot, q, k, pos, w, dy, eps, what=""):
    """Forward and backward against the oracle."""
    out = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=eps)
    grads = bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=eps)
    torch.cuda.synchronize()
    t = ro.angles(rot.freqs, rot.pair_axes, pos)
    for i, (name, x) in enumerate((("q", q), ("k", k))):
        check(f"{what} {name}", out[i], *ro.forward(x, w[i], t, eps, rot.interleaved))
        ref = ro.backward(x, w[i], t, eps, rot.interleaved, dy[i])
        check(f"{what} d{name}", grads[i], *ref["dx"])
        if w[i] is None:
            assert grads[2 + i] is None
        else:
            assert grads[2 + i].dtype == F32
            check(f"{what} d{name} weight", grads[2 + i], *ref["dw"])
    return out, grads


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,H,KV", [(1, 1, 1), (1, 32, 8), (2, 5, 1), (7, 3, 3), (65, 12, 2), (130, 4, 2), (33, 17, 9)])
def test_sizes(dtype, D, n, H, KV):
    rot = bd.rotary(D)
    both(rot, *make(n, H, KV, rot, dtype, seed=n), 1e-6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D,kw", [
    (64, dict(dim=16)), (64, dict(dim=48)), (128, dict(dim=96)), (128, dict(dim=32, interleaved=True)),
    (64, dict(interleaved=True)), (128, dict(interleaved=True)), (128, dict(sections=(16, 24, 24))),
    (64, dict(sections=(8, 12, 12), own_ladders=True)), (64, dict(dim=32, sections=(1, 0, 7, 8), interleaved=True)),
    (128, dict(sections=(5, 59), base=5e5)), (64, dict(dim=16, freqs=[0.0, -1.5, 3.0, 1e-3, 100.0, 2.0 ** 20, 0.25, 1e-9]))])
def test_rotations(dtype, D, kw):
    rot = bd.rotary(D, **kw)
    both(rot, *make(37, 6, 2, rot, dtype, seed=3), 1e-5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("eps,weights", [(None, False), (1e-6, False), (0.3, True)])
def test_norms(dtype, eps, weights):
    rot = bd.rotary(128, dim=64)
    both(rot, *make(21, 8, 4, rot, dtype, seed=4, weights=weights), eps)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_one_weight(dtype):
    rot = bd.rotary(64)
    q, k, pos, w, dy = make(21, 8, 4, rot, dtype, seed=5)
    both(rot, q, k, pos, (w[0], None), dy, 1e-6, "q only")
    both(rot, q, k, pos, (None, w[1]), dy, 1e-6, "k only")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_far_positions(dtype):
    rot = bd.rotary(128, sections=(32, 32))
    q, k, pos, w, dy = make(19, 4, 4, rot, dtype, seed=6, far=2 ** 31)
    pos[0, :2] = torch.tensor([2 ** 31 - 1, -2 ** 31], device=DEV)
    both(rot, q, k, pos, w, dy, 1e-6)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scale", [2.0 ** -30, 2.0 ** 40])
def test_rows_of_any_size(dtype, scale):
    rot = bd.rotary(64)
    q, k, pos, w, dy = make(9, 4, 2, rot, dtype, seed=7, scale=scale)
    q[3, 1] = 0
    both(rot, q, k, pos, w, dy, 1e-12)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_rows(dtype):
    # more rows than one round of workgroups takes, backward's sums over several
    rot = bd.rotary(64)
    both(rot, *make(9001, 2, 1, rot, dtype, seed=8), 1e-6)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_parts_of_a_projection_and_outputs_in_place(dtype):
    rot = bd.rotary(128, interleaved=True)
    q, k, pos, w, dy = make(29, 8, 2, rot, dtype, seed=9, fused=True)
    out, grads = both(rot, q, k, pos, w, dy, 1e-6)
    # into strided outputs: what lies between their rows stays
    wide = [torch.full((29, h + 3, 128), 7.0, dtype=dtype, device=DEV) for h in (8, 2)]
    bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6, out=tuple(t[:, 1:-2] for t in wide))
    for t, o in zip(wide, out):
        assert torch.equal(t[:, 1:-2], o) and bool((t[:, 0] == 7).all()) and bool((t[:, -2:] == 7).all())
    # in place, forward and backward
    qkv = torch.zeros(29, 12, 128, dtype=dtype, device=DEV)
    qkv[:, :8], qkv[:, 8:10], qkv[:, 10:] = q, k, 5.0
    got = bd.qk_rotate_fwd(rot, qkv[:, :8], qkv[:, 8:10], pos, *w, eps=1e-6, out=(qkv[:, :8], qkv[:, 8:10]))
    assert torch.equal(got[0], out[0]) and torch.equal(got[1], out[1]) and bool((qkv[:, 10:] == 5).all())
    d = [t.clone() for t in dy]
    got = bd.qk_rotate_bwd(rot, q, k, pos, *d, *w, eps=1e-6, out=tuple(d))
    for a, b in zip(got, grads):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_no_rows(dtype):
    rot = bd.rotary(64)
    q, k, pos, w, dy = make(0, 4, 2, rot, dtype)
    out = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6)
    assert out[0].shape == (0, 4, 64) and out[1].shape == (0, 2, 64)
    dq, dk, dqw, dkw = bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6)
    assert dq.shape == (0, 4, 64) and bool((dqw == 0).all()) and bool((dkw == 0).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_nan_and_infinity_stay_in_their_row(dtype):
    rot = bd.rotary(128)
    q, k, pos, w, dy = make(12, 8, 8, rot, dtype, seed=10)
    good = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6)
    grads = bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6)
    q[4, 3, 17], k[0, 7, 0], dy[0][9, 2, 1] = float("nan"), float("inf"), float("nan")
    out = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6)
    bad = bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6)
    hit = [torch.zeros(12, 8, dtype=torch.bool, device=DEV) for _ in range(2)]
    hit[0][4, 3] = hit[1][0, 7] = True
    for i in range(2):
        assert torch.equal(out[i][~hit[i]], good[i][~hit[i]])
        gone = hit[i].clone()
        if i == 0:
            gone[9, 2] = True
        assert torch.equal(bad[i][~gone], grads[i][~gone])
    assert bool(out[0][4, 3].isnan().any()) and bool(bad[0][9, 2].isnan().any())


def test_same_bits_again_and_in_a_graph():
    rot = bd.rotary(128, sections=(16, 24, 24))
    sets = [make(300, 32, 8, rot, BF, seed=s) for s in (11, 12, 13)]

    def step(q, k, pos, w, dy):
        return bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6) + bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6)

    expect = [[t.clone() for t in step(*s)] for s in sets]
    assert all(torch.equal(a, b) for a, b in zip(expect[0], step(*sets[0])))
    q, k, pos, w, dy = [t.clone() if isinstance(t, torch.Tensor) else [x.clone() for x in t] for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(q, k, pos, w, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(q, k, pos, w, dy)
    for i in (1, 2, 0, 1):
        for dst, src in zip([q, k, pos, *w, *dy], [*sets[i][:3], *sets[i][3], *sets[i][4]]):
            dst.copy_(src)
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.randn(512, 512, device=DEV).sum().item()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, expect[i])), i


def test_on_a_given_stream():
    rot = bd.rotary(64)
    q, k, pos, w, dy = make(100, 8, 2, rot, BF, seed=14)
    a = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6) + bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    b = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6, stream=s) + \
        bd.qk_rotate_bwd(rot, q, k, pos, *dy, *w, eps=1e-6, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_rows_past_32_bits_of_elements():
    # 2^20 rows that lie 4,096 elements apart: offsets beyond 2^31 elements and 2^32 bytes
    n, rot = (1 << 20) + 3, bd.rotary(64)
    wide = torch.zeros(n, 64, 64, dtype=BF, device=DEV)
    wide[-2:] = torch.randn(2, 64, 64, generator=torch.Generator().manual_seed(15)).to(BF).to(DEV)
    q, k = wide[:, 60:62], wide[:, 62:63]
    pos = torch.arange(n, dtype=torch.int32, device=DEV)
    t = ro.angles(rot.freqs, rot.pair_axes, pos[-2:])
    out = bd.qk_rotate_fwd(rot, q, k, pos, eps=1e-6, out=(q, k))
    check("q", out[0][-2:], *ro.forward(torch.randn(2, 64, 64, generator=torch.Generator().manual_seed(15)).to(BF)[:, 60:62], None,
                                        t, 1e-6, False))
    assert bool((out[1][:-2] == 0).all())
