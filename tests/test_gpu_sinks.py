"""Packed attention with a window and first tokens that stay visible, forward and backward, against the 64-bit oracle."""
import pytest
import torch

import paper_2609_19242_amd as bd
from tests import rotate_oracle, window_util
from tests.serving_util import check

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


def make(nq, nk, H, KV, D, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(n, h, D, generator=g).to(dtype).to(DEV) for n, h in ((nq, H), (nk, KV), (nk, KV), (nq, H))]


def both(ql, kl, H, KV, D, dtype, block, window, sinks, seed=0, backward=True, scale=0.0, tensors=None):
    kl = kl or ql
    plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, block_size=block, window=window, sinks=sinks,
                          scale=scale)
    q, k, v, do = tensors or make(sum(ql), sum(kl), H, KV, D, dtype, seed)
    o, lse = bd.packed_fwd(plan, q, k, v)
    got = dict(o=o, lse=lse)
    if backward:
        got.update(zip(("dq", "dk", "dv"), bd.packed_bwd(plan, q, k, v, o, lse, do)))
    torch.cuda.synchronize()
    at = lambda n: [sum(n[:i]) for i in range(len(n))]  # noqa: E731
    ref = window_util.packed(q, k, v, list(zip(at(ql), ql, at(kl), kl)), scale or None, block, window, sinks,
                             do if backward else None)
    for n in got:
        check(n, got[n], *ref[n])
    return plan, got


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sinks", [1, 3, 16, 64, 65, 130])
@pytest.mark.parametrize("window", [1, 16, 64, 200])
def test_windows_and_sinks(dtype, D, sinks, window):
    both([1, 63, 130, 333], None, 4, 2, D, dtype, 1, window, sinks, seed=sinks + window)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ql,kl", [([1], [1]), ([1], [700]), ([2, 1, 5], [64, 65, 66]), ([33, 0, 7, 90], [500, 20, 7, 1000]),
                                   ([40, 6, 9], [10, 0, 9]), ([128, 129], None), ([200], [201])])
def test_lengths(dtype, ql, kl):
    both(ql, kl, 8, 2, 128, dtype, 1, 40, 5, seed=len(ql))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KV", [(1, 1), (2, 2), (3, 1), (6, 2), (8, 2), (7, 7)])
def test_heads(dtype, H, KV):
    for D in (64, 128):
        both([150, 20], [170, 300], H, KV, D, dtype, 1, 50, 9, seed=H)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block,window,sinks", [(2, 7, 3), (32, 48, 4), (32, 32, 64), (17, 5, 40), (128, 60, 1), (500, 90, 7)])
def test_blocks(dtype, block, window, sinks):
    both([150, 64, 9], [150, 300, 5], 4, 2, 64, dtype, block, window, sinks, seed=block)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("ql,kl,window,sinks", [([1], [4000], 3000, 100), ([64], [3000], 2000, 1), ([3], [5000], 4990, 4)])
def test_cut_walks(D, ql, kl, window, sinks):
    plan, _ = both(ql, kl, 8, 2, D, BF, 1, window, sinks, seed=window)
    assert plan.fwd_workspace_bytes > 0


def test_cut_walks_of_keys():
    plan, _ = both([1500], None, 4, 2, 64, BF, 1, 100, 3, seed=5)
    assert plan._record.n_sums > 0
    plan, _ = both([400], None, 4, 2, 64, F32, 1, 30, 3, seed=6)
    assert plan._record.n_sums > 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales_and_large_scores(dtype):
    both([200], None, 4, 2, 64, dtype, 1, 70, 4, seed=7, scale=0.5)
    q, k, v, do = make(200, 200, 4, 2, 64, dtype, 8)
    k[2] *= 30  # a sink that takes nearly all of some rows, and nothing of others
    both([200], None, 4, 2, 64, dtype, 1, 70, 4, tensors=(q, k, v, do))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sinks,window,bad", [(4, 30, float("nan")), (70, 30, float("inf")), (64, 64, float("nan"))])
def test_keys_that_no_row_sees_may_hold_anything(dtype, D, sinks, window, bad):
    # the last 20 rows of 400 tokens: nobody sees the keys between the sinks and the first row's window
    q, k, v, do = make(20, 400, 4, 2, D, dtype, 9)
    hole = slice(sinks, 400 - 20 + 1 - window)
    k[hole], v[hole] = bad, bad
    _, got = both([20], [400], 4, 2, D, dtype, 1, window, sinks, tensors=(q, k, v, do))
    assert bool((got["dk"][hole] == 0).all()) and bool((got["dv"][hole] == 0).all())
    # a hole inside the first tile
    q, k, v, do = make(3, 50, 4, 2, D, dtype, 10)
    k[5:38], v[5:38] = bad, bad
    both([3], [50], 4, 2, D, dtype, 1, 10, 5, tensors=(q, k, v, do))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_padded_batches_and_strides(dtype):
    H, KV, D, ql = 4, 2, 64, [70, 130, 5]
    starts = [2, 100, 240]
    qkv = torch.randn(250, H + 2 * KV, D, generator=torch.Generator().manual_seed(11)).to(dtype).to(DEV)
    q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    plan = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, window=33, sinks=6, q_starts=starts)
    seqs = [(s, n, s, n) for s, n in zip(starts, ql)]
    mine = torch.zeros(250, dtype=torch.bool)
    for s, n in zip(starts, ql):
        mine[s:s + n] = True
    qkv[~mine.to(DEV)] = float("nan")
    do = torch.randn(250, H, D, generator=torch.Generator().manual_seed(12)).to(dtype).to(DEV)
    o, lse = bd.packed_fwd(plan, q, k, v)
    grads = bd.packed_bwd(plan, q, k, v, o, lse, do)
    ref = window_util.packed(q, k, v, seqs, None, 1, 33, 6, do)
    for n, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, *grads)):
        check(n, t, *ref[n])
    assert bool((o[~mine] == 0).all()) and all(bool((t[~mine] == 0).all()) for t in grads)
    # into given outputs: other rows as they were
    out = (torch.full_like(o, 7.0), torch.full_like(lse, 7.0))
    bd.packed_fwd(plan, q, k, v, out=out)
    assert torch.equal(out[0][mine], o[mine]) and bool((out[0][~mine] == 7).all()) and bool((out[1][:, ~mine] == 7).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_many_sinks_are_no_window_and_none_a_window(dtype):
    args = dict(heads=4, kv_heads=2, head_dim=64, dtype=dtype)
    q, k, v, do = make(300, 300, 4, 2, 64, dtype, 13)
    for a, b in ((dict(window=20, sinks=300), dict()), (dict(window=300, sinks=9), dict()), (dict(window=20, sinks=0), dict(window=20))):
        one, two = bd.packed_plan([300], **args, **a), bd.packed_plan([300], **args, **b)
        o, lse = bd.packed_fwd(one, q, k, v)
        ref = window_util.packed(q, k, v, [(0, 300, 0, 300)], None, 1, a["window"], a["sinks"], do)
        check("o", o, *ref["o"])
        o2, lse2 = bd.packed_fwd(two, q, k, v)
        check("o of the other call", o2, *ref["o"])
        for n, x, y in zip(("dq", "dk", "dv"), bd.packed_bwd(one, q, k, v, o, lse, do), bd.packed_bwd(two, q, k, v, o2, lse2, do)):
            check(n, x, *ref[n])
            check(n + " of the other call", y, *ref[n])


def test_few_keys_of_large_values():
    # rows whose keys all lie in one tile: dQ is a small difference of large numbers
    q, k, v, do = make(64, 64, 4, 2, 64, BF, 14)
    v = (v.float() * 0.01 + 20).to(BF)
    both([64], None, 4, 2, 64, BF, 1, 16, 3, tensors=(q, k, v, do))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_training_step_of_a_layer(dtype):
    """As it is used: rotated queries and keys, attention, and both backward passes, each against the oracle of what it
    was given."""
    ql, H, KV, D = [70, 1, 150], 4, 2, 64
    n, rot = sum(ql), bd.rotary(64, sections=(16, 16))
    g = torch.Generator().manual_seed(18)
    qkv = torch.randn(n, H + 2 * KV, D, generator=g).to(dtype).to(DEV)
    w = [(1 + 0.2 * torch.randn(D, generator=g)).to(dtype).to(DEV) for _ in range(2)]
    do = torch.randn(n, H, D, generator=g).to(dtype).to(DEV)
    pos = torch.cat([torch.arange(x) for x in ql]).to(torch.int32)
    pos = torch.stack([pos // 12, pos % 12]).to(DEV)
    q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    plan = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, window=40, sinks=3)
    qr, kr = bd.qk_rotate_fwd(rot, q, k, pos, *w, eps=1e-6)
    o, lse = bd.packed_fwd(plan, qr, kr, v)
    dqr, dkr, dv = bd.packed_bwd(plan, qr, kr, v, o, lse, do)
    dq, dk, dqw, dkw = bd.qk_rotate_bwd(rot, q, k, pos, dqr, dkr, *w, eps=1e-6)
    seqs = [(sum(ql[:i]), x, sum(ql[:i]), x) for i, x in enumerate(ql)]
    ref = window_util.packed(qr, kr, v, seqs, None, 1, 40, 3, do)
    for name, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse, dqr, dkr, dv)):
        check(name, t, *ref[name])
    t = rotate_oracle.angles(rot.freqs, rot.pair_axes, pos)
    for x, y, dy, dx, ww, dw in ((q, qr, dqr, dq, w[0], dqw), (k, kr, dkr, dk, w[1], dkw)):
        check("rotated", y, *rotate_oracle.forward(x, ww, t, 1e-6, False))
        back = rotate_oracle.backward(x, ww, t, 1e-6, False, dy)
        check("dx", dx, *back["dx"])
        check("dw", dw, *back["dw"])


def test_replays_of_a_graph_equal_eager_calls():
    plan = bd.packed_plan([300, 1, 77], [300, 2000, 100], heads=8, kv_heads=2, head_dim=128, dtype=BF, window=128, sinks=4)
    sets = [make(378, 2400, 8, 2, 128, BF, s) for s in (15, 16, 17)]

    def step(q, k, v, do):
        o, lse = bd.packed_fwd(plan, q, k, v)
        return (o, lse, *bd.packed_bwd(plan, q, k, v, o, lse, do))

    expect = [[t.clone() for t in step(*s)] for s in sets]
    static = [t.clone() for t in sets[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*static)
    for i in (1, 2, 0, 1):
        for dst, src in zip(static, sets[i]):
            dst.copy_(src)
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.randn(512, 512, device=DEV).sum().item()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, expect[i])), i
