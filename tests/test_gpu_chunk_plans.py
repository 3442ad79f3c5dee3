"""Attention of chunks with a plan that is not of its sizes: every row becomes NaN, and nothing of the plan is followed."""
import math

import pytest
import torch

import paper_2609_19242_amd as bd

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32
LENS, COUNTS = [3000, 700, 90], [3, 100, 1]


def i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def make(dtype, max_pages=200, page=16):
    g = torch.Generator().manual_seed(1)
    need = [-(-n // page) for n in LENS]
    table = torch.full((len(LENS), max_pages), -1, dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = torch.arange(sum(need[:r]), sum(need[:r]) + n)
    k, v = (torch.randn(1, sum(need), page, 2, 64, generator=g).to(dtype).to(DEV) for _ in range(2))
    return bd.Cache(k, v, table.to(DEV), i32(LENS), torch.ones(sum(need), dtype=torch.int32, device=DEV),
                    torch.zeros(2, dtype=torch.int32, device=DEV))


def plan_of(cache, out=None, **kw):
    return bd.chunk_plan(cache, i32([0, 1, 2]), i32(COUNTS), rows=sum(COUNTS) + 2, heads=4, out=out, **kw)


def queries(dtype):
    return torch.randn(sum(COUNTS) + 2, 4, 64, generator=torch.Generator().manual_seed(2)).to(dtype).to(DEV)


def all_nan(*ts):
    return all(bool(t.isnan().all()) for t in ts)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("made,name,called", [
    (dict(), "window", 60), (dict(window=60, sinks=4), "window", 0), (dict(window=60, sinks=4), "sinks", 3),
    (dict(window=60), "block_size", 8), (dict(), "requests", 2)])
def test_another_record(dtype, made, name, called):
    cache, q = make(dtype), queries(dtype)
    plan = plan_of(cache, **made)
    good = bd.chunk_attn(plan, q, 0)
    assert not any(bool(t.isnan().any()) for t in good)
    was = getattr(plan._record, name)
    setattr(plan._record, name, called)
    plan._workspace_bytes = None
    assert all_nan(*bd.chunk_attn(plan, q, 0))
    out = torch.zeros_like(q), torch.zeros(4, len(q), device=DEV)
    assert all_nan(*bd.chunk_attn(plan, q, 0, out=out))  # (rows of no request are left only where the plan says which)
    setattr(plan._record, name, was)
    plan._workspace_bytes = None
    assert all(torch.equal(a, b) for a, b in zip(good, bd.chunk_attn(plan, q, 0)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_another_cache_and_memory_of_no_plan(dtype):
    cache, q = make(dtype), queries(dtype)
    plan = plan_of(cache)
    good = bd.chunk_attn(plan, q, 0)
    plan.cache = make(dtype, max_pages=188)
    assert all_nan(*bd.chunk_attn(plan, q, 0))
    plan.cache = make(dtype)  # (one of the same sizes)
    assert all(torch.equal(a, b) for a, b in zip(good, bd.chunk_attn(plan, q, 0)))
    plan.cache = cache
    for fill in (0, -1):
        plan._items.fill_(fill)
        assert all_nan(*bd.chunk_attn(plan, q, 0))


def test_sinks_without_a_window_and_other_scales_are_the_same_plan():
    cache, q = make(BF), queries(BF)
    plan = plan_of(cache)
    good = bd.chunk_attn(plan, q, 0)
    plan._record.sinks = 7
    assert all(torch.equal(a, b) for a, b in zip(good, bd.chunk_attn(plan, q, 0)))
    plan._record.scale = 0.25
    assert not any(bool(t.isnan().any()) for t in bd.chunk_attn(plan, q, 0))


def test_a_captured_call_whose_plan_was_made_anew():
    cache, q = make(BF), queries(BF)
    plan = plan_of(cache)
    want = [t.clone() for t in bd.chunk_attn(plan, q, 0)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        bd.chunk_attn(plan, q, 0)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = bd.chunk_attn(plan, q, 0)
    for window in (0, 60, 0, 400, 0):
        plan_of(cache, out=plan, window=window, sinks=3 if window else 0)
        for t in got:
            t.fill_(math.pi)
        graph.replay()
        torch.randn(256, 256, device=DEV).sum().item()
        torch.cuda.synchronize()
        if window:
            assert all_nan(*got)
        else:
            assert all(torch.equal(a, b) for a, b in zip(got, want))
