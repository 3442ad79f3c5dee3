"""The plan of packed calls: every tile of query rows once, every step of every key tile's walk once, partial sums in
places of their own and added up, heaviest items first.  CPU only."""
import random

import numpy as np
import pytest
import torch

import paper_2609_19242_amd as bd

BIG = 0x3fffffff


def items(p):
    r = p._record
    a = np.frombuffer(p._items.numpy().tobytes(), dtype=np.int32)[:8 * (r.q_items + r.k_items + r.n_sums)].reshape(-1, 8)
    return a[:r.q_items], a[r.q_items:r.q_items + r.k_items], a[r.q_items + r.k_items:]


def steps_of(ql, kl, first, last, block, window, rows, per_block):
    """Steps of the walk of keys [first, last]: blocks of `rows` query rows from the first that sees one of them to the last."""
    seen = []
    for i in range(ql):
        x = kl - ql + i
        e = (x // block + 1) * block
        lo = e - window if window else 0
        if x >= 0 and first < e and lo <= last:
            seen.append(i)
    return (seen[-1] // rows - seen[0] // rows + 1) * per_block if seen else 0


def walked(ql, kl, a, b, block, window):
    """Keys that rows [a, b) see, from the first to the last."""
    lo, hi = kl, 0
    for i in range(a, b):
        x = kl - ql + i
        if x < 0:
            continue
        e = (x // block + 1) * block
        lo, hi = min(lo, max(0, e - window) if window else 0), max(hi, min(e, kl))
    return max(0, hi - lo)


def check(ql, kl, H, KV, D, dtype, block, window):
    p = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, block_size=block, window=window, device="cpu")
    q, k, sums = items(p)
    f32, group = dtype == torch.float32, H // KV
    heads = 1 if f32 else 4 if group % 4 == 0 else 2 if group % 2 == 0 else 1
    qt, kt = (16, 16) if f32 else (128 // heads, 128)
    rows = 16 if f32 else 64 if group % 2 else 32
    per_block = group if f32 or group % 2 else group // 2
    q0 = np.cumsum([0] + list(ql))
    k0 = np.cumsum([0] + list(kl))
    want = [(q0[i], n, k0[i], kl[i], t) for i, n in enumerate(ql) for t in range(-(-n // qt))]
    assert sorted(map(tuple, q[:, :5].tolist())) == sorted(want)
    cost = [walked(n, m, t * qt, min(n, (t + 1) * qt), block, window) for _, n, _, m, t in q[:, :5].tolist()]
    assert all(a >= b for a, b in zip(cost, cost[1:]))
    chunks = {}
    for a in k.tolist():
        chunks.setdefault(tuple(a[:5]), []).append(a[5:])
    assert sorted(chunks) == sorted((q0[i], ql[i], k0[i], m, t) for i, m in enumerate(kl) for t in range(-(-m // kt)))
    slots, longest = [], []
    for (_, n, kk, m, t), parts in chunks.items():
        parts.sort()
        total = steps_of(n, m, t * kt, min(m, (t + 1) * kt) - 1, block, window, rows, per_block)
        assert parts[0][0] == 0 and parts[-1][1] == BIG and all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
        assert parts[-1][0] < total or total == 0 == parts[-1][0]
        if len(parts) == 1:
            assert parts[0][2] == -1
        else:
            mine = [a[2] for a in parts]
            assert mine == list(range(mine[0], mine[0] + len(mine)))
            assert [kk, m, t, mine[0], len(mine)] in sums[:, :5].tolist()
            slots += mine
        longest += [b - a for a, b, _ in parts[:-1]]
    assert sorted(slots) == list(range(p._record.slots)) and len(sums) == sum(len(x) > 1 for x in chunks.values())
    assert not longest or len(set(longest)) == 1
    return p


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,KV", [(4, 4), (4, 2), (8, 2), (6, 2), (3, 1)])
def test_items_cover_the_work_once(H, KV, dtype):
    rng = random.Random(7 * H + KV)
    for _ in range(12):
        n = rng.randint(1, 5)
        ql = [rng.choice([0, 1, rng.randint(1, 400)]) for _ in range(n)]
        kl = [max(0, x + rng.choice([0, 0, rng.randint(-50, 300)])) for x in ql]
        check(ql, kl, H, KV, rng.choice([64, 128]), dtype, rng.choice([1, 1, 7, 32, 300]), rng.choice([0, 0, 1, 30, 200]))


def test_long_walks_are_cut():
    p = check([900, 40], [900, 40], 4, 1, 128, torch.bfloat16, 1, 0)
    assert p._record.n_sums > 0 and p.workspace_bytes > 4 * 2 * 940 * 4


def test_a_full_card_is_not_cut():
    p = check([130] * 160, [130] * 160, 8, 8, 128, torch.bfloat16, 1, 0)
    assert p._record.n_sums == 0 and p._record.teams == 1


def test_few_tiles_take_two_teams():
    assert check([64], [64], 4, 2, 128, torch.bfloat16, 1, 0)._record.teams == 2


def chunk_items(p, dq):
    r = p._record
    a = np.frombuffer(p._items.numpy().tobytes(), dtype=np.int32)
    at = r.q_items + r.k_items + r.n_sums + (r.fwd.items + r.fwd.sums if dq else 0)
    c = r.dq if dq else r.fwd
    a = a[8 * at:8 * (at + c.items + c.sums)].reshape(-1, 8)
    return c, a[:c.items].tolist(), a[c.items:].tolist()


@pytest.mark.parametrize("ql,kl,H,KV,block,window", [
    ([1], [2500], 4, 1, 1, 0), ([70, 1, 3, 300], [2000, 1700, 0, 300], 4, 2, 1, 0), ([130, 40], [2400, 20], 3, 1, 1, 1900),
    ([1800], [1700], 2, 2, 7, 0), ([3000, 10], [3000, 5000], 8, 2, 1, 0)])
def test_forward_chunks_cover_each_walk_once(ql, kl, H, KV, block, window):
    p = check(ql, kl, H, KV, 128, torch.bfloat16, block, window)
    for dq in (False, True):
        check_chunks(p, dq, ql, H, KV, block, window)
    assert p._record.teams == 1


def check_chunks(p, dq, ql, H, KV, block, window):
    c, chunks, sums = chunk_items(p, dq)
    r, group = p._record, H // KV
    heads = 4 if group % 4 == 0 else 2 if group % 2 == 0 else 1
    qt = 128 // heads
    assert c.items > r.q_items and len(sums) == c.sums > 0
    by_tile = {}
    for a in chunks:
        by_tile.setdefault(tuple(a[:5]), []).append(a[5:])
    whole = items(p)[0]
    assert sorted(by_tile) == sorted(map(tuple, whole[:, :5].tolist()))
    slots = []
    for (q0, n, _, m, t), parts in by_tile.items():
        parts.sort()
        assert parts[0][0] == 0 and parts[-1][1] == BIG and all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
        keys = walked(n, m, t * qt, min(n, (t + 1) * qt), block, window)
        assert parts[-1][0] * 64 < keys + 64 or len(parts) == 1
        if len(parts) > 1:
            mine = [a[2] for a in parts]
            assert mine == list(range(mine[0], mine[0] + len(mine)))
            assert [q0, n, t, mine[0], len(mine)] in [x[:5] for x in sums]
            slots += mine
        else:
            assert parts[0][2] == -1
    assert sorted(slots) == list(range(c.slots))
    rows = c.slots * (H // heads) * 128
    if dq:
        assert p.workspace_bytes >= rows * 128 * 4 + 2 * p.q_rows * H * 4
    else:
        assert p.fwd_workspace_bytes >= rows * 129 * 4


def test_walks_that_fill_the_card_or_are_short_are_not_cut():
    for ql, H in (([4000] * 8, 16), ([1000], 4), ([30] * 100, 8)):
        p = bd.packed_plan(ql, heads=H, kv_heads=4, head_dim=128, dtype=torch.bfloat16, device="cpu")
        assert p.fwd_workspace_bytes == 0 and p._record.fwd.items == 0
    p = bd.packed_plan([1], [2500], heads=4, kv_heads=4, head_dim=64, dtype=torch.float32, device="cpu")
    assert p.fwd_workspace_bytes == 0


def test_two_teams_where_a_cu_ends_sooner_one_workgroup_at_a_time():
    for ql, H, KV, teams in (([2213, 600, 152], 16, 16, 2), ([1355, 8], 24, 8, 2), ([500] * 8, 16, 4, 1), ([200] * 40, 8, 8, 1)):
        p = bd.packed_plan(ql, heads=H, kv_heads=KV, head_dim=128, dtype=torch.bfloat16, device="cpu")
        assert p._record.teams == teams and p._record.fwd.items == 0, (ql, H, KV)
