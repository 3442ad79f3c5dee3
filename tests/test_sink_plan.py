"""The plan of packed calls with a window and sinks: every tile of query rows once, its walk whole or in chunks that
cover it; the sinks' key tiles and the others', every step of their walks once, partial sums in places of their own; the
oracle's rule against a second form of it; refusals.  CPU only."""
import math

import numpy as np
import pytest
import torch

import paper_2609_19242_amd as bd
from tests import serving_util, window_util

BIG = 0x3fffffff
BF, F32 = torch.bfloat16, torch.float32


def plan(ql, kl=None, **kw):
    return bd.packed_plan(ql, kl, **dict(dict(heads=4, kv_heads=2, head_dim=64, dtype=BF, device="cpu"), **kw))


def parts(p):
    r = p._record
    a = np.frombuffer(p._items.numpy().tobytes(), dtype=np.int32)
    a = a[:a.size // 8 * 8].reshape(-1, 8)
    out, at = {}, 0
    for name, n in (("q", r.q_items), ("k", r.k_items), ("sums", r.n_sums), ("fwd", r.fwd.items), ("fwd_sums", r.fwd.sums),
                    ("dq", r.dq.items), ("dq_sums", r.dq.sums)):
        out[name] = a[at:at + n].tolist()
        at += n
    return out


def span(vis_rows, to_tile):
    """Tiles from the first to the last that some row sees."""
    seen = sorted({to_tile(j) for j in vis_rows})
    return (seen[0], seen[-1] + 1) if seen else (0, 0)


CASES = [([5], None, 1, 16, 4), ([1], [4000], 1, 3000, 100), ([300, 1, 0, 77], [300, 900, 50, 10], 8, 64, 70),
         ([700, 41], None, 32, 96, 4), ([130] * 5, [130, 200, 131, 5, 1000], 1, 33, 128), ([6, 9], [3, 0], 4, 8, 2),
         ([2500], None, 1, 1024, 200), ([64], [8000], 1, 6000, 1)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ql,kl,block,window,sinks", CASES)
@pytest.mark.parametrize("H,KV,D", [(4, 2, 64), (4, 1, 128), (3, 1, 128)])
def test_items(dtype, ql, kl, block, window, sinks, H, KV, D):
    p = plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, block_size=block, window=window, sinks=sinks)
    kl = kl or ql
    f32, group = dtype == F32, H // KV
    heads = 1 if f32 else 4 if group % 4 == 0 else 2 if group % 2 == 0 else 1
    qt, kt, step = (16, 16, 16) if f32 else (128 // heads, 128, 64 if group % 2 else 32)
    per = group if f32 or group % 2 else group // 2
    x = parts(p)
    q0, k0 = np.cumsum([0] + list(ql)).tolist(), np.cumsum([0] + list(kl)).tolist()
    which = {a: i for i, (a, n) in enumerate(zip(q0, ql)) if n}
    bykey = {a: i for i, (a, n) in enumerate(zip(k0, kl)) if n}
    want = sorted((q0[i], n, k0[i], kl[i], t) for i, n in enumerate(ql) for t in range(-(-n // qt)))
    assert sorted(tuple(a[:5]) for a in x["q"]) == want
    vis = [window_util.visible(n, m, block, window, sinks) for n, m in zip(ql, kl)]
    # chunks of query tiles: contiguous, to the end; each with a slot of its own
    for kind in ("fwd", "dq"):
        chunks = {}
        for a in x[kind]:
            chunks.setdefault(tuple(a[:5]), []).append(tuple(a[5:]))
        slots = [c[2] for cs in chunks.values() for c in cs if c[2] >= 0]
        assert len(slots) == len(set(slots)) == (getattr(p._record, kind).slots if x[kind] else 0)
        if x[kind]:
            assert sorted(chunks) == want
        sums = {(s[0], s[2]): (s[3], s[4]) for s in x[kind + "_sums"]}
        for key, cs in chunks.items():
            cs.sort()
            assert cs[0][0] == 0 and cs[-1][1] == BIG and all(a[1] == b[0] for a, b in zip(cs, cs[1:]))
            if len(cs) > 1:
                assert sums[(key[0], key[4])] == (cs[0][2], len(cs)) and [c[2] for c in cs] == list(range(cs[0][2], cs[0][2] + len(cs)))
                # no chunk is empty: the walk has the sinks and the window, without the gap between in multiples of 16
                i, t = which[key[0]], key[4]
                keys = torch.nonzero(vis[i][t * qt:(t + 1) * qt].any(0)).flatten().tolist()
                first = min(j for j in keys if j >= min(sinks, kl[i])) // 16 * 16
                below = (min(sinks, kl[i]) + 15) // 16 * 16
                walk = below + keys[-1] + 1 - first if first > below else keys[-1] + 1
                assert cs[-1][0] < -(-walk // 64)
    # key tiles: the sinks' and the others'
    want_k = sorted((q0[i], ql[i], k0[i], m, t) for i, m in enumerate(kl) for s in [min(sinks, m)]
                    for t in [-1 - t for t in range(-(-s // kt))] + list(range(-(-(m - s) // kt))))
    walks = {}
    for a in x["k"]:
        walks.setdefault(tuple(a[:5]), []).append(tuple(a[5:]))
    assert sorted(walks) == want_k
    sums = {(s[0], s[2]): s for s in x["sums"]}
    slots = []
    for key, cs in walks.items():
        i = bykey[key[2]]
        s = min(sinks, kl[i])
        first, last = ((-1 - key[4]) * kt, s) if key[4] < 0 else (s + key[4] * kt, kl[i])
        rows = torch.nonzero(vis[i][:, first:min(first + kt, last)].any(1)).flatten().tolist()
        a, b = span(rows, lambda r: r // step)
        steps = (b - a) * per
        cs.sort()
        assert cs[0][0] == 0 and cs[-1][1] == BIG and all(u[1] == w[0] for u, w in zip(cs, cs[1:]))
        assert len(cs) == 1 or cs[-1][0] < steps
        slots += [c[2] for c in cs if c[2] >= 0]
        if len(cs) > 1:
            tile = -1 - key[4] if key[4] < 0 else key[4]
            row0, n = (key[2], s) if key[4] < 0 else (key[2] + s, kl[i] - s)
            assert tuple(sums[(row0, tile)][:5]) == (row0, n, tile, cs[0][2], len(cs))
    assert sorted(slots) == list(range(p._record.slots))


def test_sinks_without_a_window_or_none_are_the_plain_plan():
    a = plan([300, 20], window=0, sinks=7)
    b = plan([300, 20])
    assert bytes(a._record) == bytes(b._record) and torch.equal(a._items, b._items)
    assert a._record.problem.sinks == 0
    assert plan([300], window=32, sinks=0)._record.problem.sinks == 0


@pytest.mark.parametrize("block,window,sinks", [(1, 0, 0), (1, 5, 0), (4, 6, 3), (1, 1, 1), (8, 40, 100), (3, 2, 7)])
def test_the_rule(block, window, sinks):
    for nq, nk in ((9, 9), (1, 20), (7, 3), (4, 0), (5, 23)):
        vis = window_util.visible(nq, nk, block, window, sinks)
        x, j = (torch.arange(nq) + (nk - nq))[:, None], torch.arange(nk)[None]
        e = torch.div(x, block, rounding_mode="floor") * block + block
        want = (j < e) & (x >= 0)
        if window:
            want &= (j >= e - window) | (j < sinks)
        assert torch.equal(vis, want)
        if not sinks or not window:
            assert torch.equal(vis, serving_util.visible(nq, nk, block, window))


@pytest.mark.parametrize("sinks", [-1, (1 << 28) + 1])
def test_sinks_out_of_range(sinks):
    with pytest.raises(bd.BdlmError, match="sinks"):
        plan([5], window=4, sinks=sinks)
    with pytest.raises(bd.BdlmError, match="sinks"):
        plan([5], sinks=sinks)


def test_sinks_that_do_not_fit():
    with pytest.raises(ValueError, match="sinks"):
        plan([5], window=4, sinks=1 << 40)
    with pytest.raises(TypeError):
        plan([5], window=4, sinks=1.5)
    assert math.isfinite(plan([5], window=4, sinks=1 << 28).q_rows)
