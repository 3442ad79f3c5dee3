"""Offsets past 32 bits: a cache of more than 4 GB a layer, and packed rows whose elements lie past 2^31."""
import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import check, packed
from tests.test_gpu_prefix import oracle

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("ps", [16, 12])
def test_pages_past_4_gb(ps):
    pages, KV, D, H = 2_300_000 // ps, 8, 128, 16  # 4.7 GB of K
    held = pages - 60
    k, v = (torch.empty((1, pages, ps, KV, D), dtype=BF, device=DEV) for _ in range(2))
    assert k.numel() * 2 > 1 << 32
    refs = torch.ones(pages, dtype=torch.int32, device=DEV)
    refs[held:] = 0
    c = bd.Cache(k, v, torch.full((4, 20), -1, dtype=torch.int32, device=DEV), i32([0] * 4), refs, i32([0, 0]))
    lens = [200, 130]
    bd.cache_grow(c, i32([0, 1]), i32(lens))
    kn, vn = (synth.normal((sum(lens), KV, D), s, BF).to(DEV) for s in (3, 4))
    bd.cache_write(c, 0, i32([0, 1]), i32(lens), kn, vn, starts=i32([0, 200]))
    bd.cache_fork(c, i32([0, 0]), i32([2, 3]))
    torch.cuda.synchronize()
    assert c.status.tolist() == [0, 0] and int(c.table[0, 0]) == held
    q = synth.normal((4, 2, H, D), 5, BF).to(DEV)

    def attend():
        o, lse = bd.prefix_attn(q, c, 0, i32([0, 1, 2, 3]))
        torch.cuda.synchronize()
        return o, lse

    # a small cache with the same rows for the oracle
    used = sorted({p for row in c.table.tolist() for p in row if p >= 0})
    small = bd.Cache(k[:, used], v[:, used],
                     torch.tensor([[used.index(p) if p >= 0 else -1 for p in row] for row in c.table.tolist()],
                                  dtype=torch.int32, device=DEV), c.lens, refs[used].contiguous(), c.status)
    ref = oracle(q, small, 0, [0, 1, 2, 3], False)
    o, lse = attend()
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])
    refs[5:5 + len(used)] = 0  # holes at the bottom: every used page moves down
    bd.cache_compact(c)
    o2, lse2 = attend()
    assert int(c.table.max()) < 5 + len(used) and torch.equal(o, o2) and torch.equal(lse, lse2)


def test_packed_rows_past_2_31_elements():
    H, KV, D, rows = 32, 8, 128, 600_000  # 2.46e9 elements of Q
    ql, starts = [70, 40], [3, rows - 40]
    q, do, o, dq = (torch.empty((rows, H, D), dtype=BF, device=DEV) for _ in range(4))
    k, v, dk, dv = (torch.empty((rows, KV, D), dtype=BF, device=DEV) for _ in range(4))
    lse = torch.empty((H, rows), device=DEV)
    assert q.numel() > 1 << 31
    part = {}
    for i, (t, h) in enumerate(((q, H), (k, KV), (v, KV), (do, H))):
        x = synth.normal((sum(ql), h, D), 11 + i, BF)
        part[i] = x
        for s, n, a in zip(starts, ql, (0, ql[0])):
            t[s:s + n] = x[a:a + n].to(DEV)
    plan = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=D, dtype=BF, q_starts=starts)
    bd.packed_fwd(plan, q, k, v, out=(o, lse))
    bd.packed_bwd(plan, q, k, v, o, lse, do, out=(dq, dk, dv))
    torch.cuda.synchronize()
    ref = packed(part[0], part[1], part[2], [(0, 70, 0, 70), (70, 40, 70, 40)], do=part[3])
    for n, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        check(n, torch.cat([t[s:s + m] for s, m in zip(starts, ql)]), *ref[n])
    check("lse", torch.cat([lse[:, s:s + m] for s, m in zip(starts, ql)], 1), *ref["lse"])


def test_more_pages_asked_for_than_32_bits_hold():
    S, mp = 1024, 1 << 21
    k, v = (torch.zeros((1, 100, 1, 1, 64), dtype=BF, device=DEV) for _ in range(2))
    table = torch.full((S, mp), -1, dtype=torch.int32, device=DEV)
    c = bd.Cache(k, v, table, i32([0] * S), i32([0] * 100), i32([0, 0]))
    for n in (S, S - 1):
        bd.cache_grow(c, i32(range(n)), i32([mp] * n))
        torch.cuda.synchronize()
        assert c.status.tolist() == [2, min(n * mp - 100, 2 ** 31 - 1)]
        assert int(c.lens.sum()) == 0 and int(c.refs.sum()) == 0 and bool((table[::128] == -1).all())
