"""Where the new tensors of a call on a given stream come from: that stream's own memory (the current stream's may still
be in use there by work that the given one does not wait for), and results are kept for the current stream as well, on
which the caller goes on with them."""
import contextlib
import types

import pytest
import torch

import paper_2609_19242_amd as bd
from paper_2609_19242_amd import cache as cm
from paper_2609_19242_amd import packed as pm

BF = torch.bfloat16
SIDE, CURRENT = "side", "current"


@pytest.fixture
def made(monkeypatch):
    """[(tensor, the stream whose memory it is)] and [(tensor, stream it was recorded on)], with no GPU: the calls take
    CPU tensors and launch nothing."""
    at, new, kept = [CURRENT], [], []

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    def watch(owner, name):
        plain = getattr(owner, name)

        def call(*a, **kw):
            t = plain(*a, **kw)
            new.append((t, at[-1]))
            return t

        monkeypatch.setattr(owner, name, call)

    for name in ("empty", "empty_like", "full", "zeros", "zeros_like"):
        watch(torch, name)
    for name in ("new_empty", "new_full", "new_zeros"):
        watch(torch.Tensor, name)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t, s)))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at[-1])
    monkeypatch.setattr(bd, "_torch_stream", lambda s, device: s)
    for m in (pm, cm):
        monkeypatch.setattr(m, "_launch", lambda *a: None)
        if hasattr(m, "_torch_stream"):
            monkeypatch.setattr(m, "_torch_stream", lambda s, device: s)
    return types.SimpleNamespace(new=new, kept=kept)


def holds(made, results, workspaces):
    mine = [t for t, _ in made.new]
    assert len(mine) == len(results) + workspaces
    assert all(s == SIDE for _, s in made.new)
    for r in results:
        assert any(r is t for t in mine)
        assert any(r is t and s == CURRENT for t, s in made.kept)


@pytest.mark.parametrize("rows", [8, 11])  # (11: rows of no sequence, which new outputs fill)
def test_packed_calls(made, rows):
    plan = bd.packed_plan([5, 3], heads=4, kv_heads=2, head_dim=64, dtype=BF, device="cpu")
    q, k, v = (torch.ones(rows, h, 64, dtype=BF) for h in (4, 2, 2))
    made.new.clear()
    o, lse = bd.packed_fwd(plan, q, k, v, stream=SIDE)
    holds(made, (o, lse), 0)
    made.new.clear()
    holds(made, bd.packed_bwd(plan, q, k, v, o, lse, q, stream=SIDE), 1)
    long = bd.packed_plan([1], [4000], heads=8, kv_heads=2, head_dim=128, dtype=BF, device="cpu")
    assert long.fwd_workspace_bytes > 0
    made.new.clear()
    holds(made, bd.packed_fwd(long, torch.ones(1, 8, 128, dtype=BF), *[torch.ones(4000, 2, 128, dtype=BF)] * 2,
                              stream=SIDE), 1)


def test_attention_over_the_cache(made):
    c = bd.cache_new(1, 4, 16, 2, 64, 2, 200, BF, "cpu")
    q = torch.ones(2, 1, 4, 64, dtype=BF)
    made.new.clear()
    holds(made, bd.prefix_attn(q, c, 0, torch.tensor([0, 1], dtype=torch.int32), stream=SIDE), 1)


def test_joint_calls(made, monkeypatch):
    monkeypatch.setattr(bd, "_on_device", lambda *a, **kw: None)
    monkeypatch.setattr(bd, "_stream", lambda s: 0)
    ok = lambda *a: 0  # noqa: E731
    monkeypatch.setattr(bd, "lib", lambda: types.SimpleNamespace(bdlm_attn_fwd=ok, bdlm_attn_bwd=ok,
                                                                 bdlm_attn_bwd_workspace_bytes=lambda *a: 512))
    q, k, v = (torch.ones(1, 64, h, 64, dtype=BF) for h in (4, 2, 2))
    made.new.clear()
    o, lse = bd.joint_fwd(q, k, v, 16, stream=SIDE)
    holds(made, (o, lse), 0)
    made.new.clear()
    holds(made, bd.joint_bwd(q, k, v, o, lse, q, 16, stream=SIDE), 1)


def test_calls_on_the_current_stream_record_nothing(made):
    plan = bd.packed_plan([5, 3], heads=4, kv_heads=2, head_dim=64, dtype=BF, device="cpu")
    q, k, v = (torch.ones(8, h, 64, dtype=BF) for h in (4, 2, 2))
    made.new.clear()
    bd.packed_bwd(plan, q, k, v, *bd.packed_fwd(plan, q, k, v), q)
    assert all(s == CURRENT for _, s in made.new) and not made.kept


@pytest.mark.gpu
def test_results_dropped_while_their_kernels_wait():
    """Each call's LSE, and a backward's dK and dV, go back to the allocator while the kernels that write them wait."""
    q, k, v, do = (torch.randn(6000, h, 128, device="cuda").to(BF) for h in (8, 2, 2, 8))
    plan = bd.packed_plan([6000], heads=8, kv_heads=2, head_dim=128, dtype=BF)
    c = bd.cache_new(1, 40, 16, 2, 128, 2, 400)
    c.lens.fill_(300)
    c.table[:, :20] = torch.arange(40, device="cuda").view(2, 20)
    qs, seqs = torch.randn(2, 1, 8, 128, device="cuda").to(BF), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    want = bd.packed_fwd(plan, q, k, v)
    grads = bd.packed_bwd(plan, q, k, v, *want, do)
    step = bd.prefix_attn(qs, c, 0, seqs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for use in (side, side.cuda_stream):
        torch.cuda.synchronize()
        for _ in range(10):  # (work for the kernels to wait behind)
            bd.packed_bwd(plan, q, k, v, *want, do, stream=use)
        o = bd.packed_fwd(plan, q, k, v, stream=use)[0]
        dq = bd.packed_bwd(plan, q, k, v, *want, do, stream=use)[0]
        so = bd.prefix_attn(qs, c, 0, seqs, stream=use)[0]
        others = [torch.full_like(t, 7) for t in (want[1], grads[1], grads[2], step[1], qs) for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(dq, grads[0]) and torch.equal(so, step[0])
        assert all(bool((t == 7).all()) for t in others)


@pytest.mark.gpu
def test_joint_results_dropped_while_their_kernels_wait():
    q, k, v, do = (torch.randn(1, 4096, h, 128, device="cuda").to(BF) for h in (8, 2, 2, 8))
    want = bd.joint_fwd(q, k, v, 32)
    grads = bd.joint_bwd(q, k, v, *want, do, 32)
    side = torch.cuda.Stream()
    for use in (side, side.cuda_stream):
        torch.cuda.synchronize()
        for _ in range(5):
            bd.joint_bwd(q, k, v, *want, do, 32, stream=use)
        o = bd.joint_fwd(q, k, v, 32, stream=use)[0]
        dq = bd.joint_bwd(q, k, v, *want, do, 32, stream=use)[0]
        others = [torch.full_like(t, 7) for t in (want[1], grads[1], grads[2]) for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(o, want[0]) and torch.equal(dq, grads[0])
        assert all(bool((t == 7).all()) for t in others)
