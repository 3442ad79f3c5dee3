"""Attention of chunks of new tokens over a paged cache against the 64-bit oracle, and the plans that it runs."""
import math

import numpy as np
import pytest
import torch

import paper_2609_19242_amd as bd
from tests import window_util
from tests.serving_util import check, head

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


def i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def make_cache(lens, KV, D, dtype, page, layers=1, seed=0, spare=2, extra=1):
    """Sequences of the given lengths over shuffled pages, which hold random rows; every spare row NaN."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(need + [1]) + extra), -1, dtype=torch.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn(layers, pages, page, KV, D, generator=g).to(dtype) for _ in range(2))
    held = torch.zeros(pages, page, dtype=torch.bool)
    for r, n in enumerate(lens):
        for p in range(need[r]):
            held[int(table[r, p]), :min(page, n - p * page)] = True
    k[:, ~held], v[:, ~held] = math.nan, math.nan
    refs = torch.bincount(table[table >= 0].long(), minlength=pages).to(torch.int32)
    return bd.Cache(k.to(DEV), v.to(DEV), table.to(DEV), i32(lens), refs.to(DEV), torch.zeros(2, dtype=torch.int32, device=DEV))


def rows_of(cache, seq, n, layer):
    page = cache.page_size
    where = cache.table[seq].cpu().long()[torch.arange(n) // page] * page + torch.arange(n) % page
    return [x[layer].flatten(0, 1).cpu()[where].double() for x in (cache.k, cache.v)]


def oracle(cache, seqs, counts, q, layer=0, scale=None, block=1, window=0, sinks=0):
    n, H, D = q.shape
    o, lse = [window_util.nan(n, H, D) for _ in range(2)], [window_util.nan(H, n) for _ in range(2)]
    lens = cache.lens.cpu().tolist()
    Q, at = q.cpu().double(), 0
    for s, c in zip(seqs, counts):
        c = max(c, 0)
        length = lens[s] if 0 <= s < len(lens) else 0
        mine = min(c, n - at)
        if mine > 0:
            vis = window_util.visible(c, length, block, window, sinks)[:mine]
            k, v = rows_of(cache, s, length, layer) if length else [torch.zeros(0, cache.kv_heads, D, dtype=torch.float64)] * 2
            for h in range(H):
                g = h // (H // cache.kv_heads)
                r = head(Q[at:at + mine, h], k[:, g], v[:, g], vis, scale or 1 / math.sqrt(D), q.dtype)
                for i in range(2):
                    o[i][at:at + mine, h], lse[i][h, at:at + mine] = r["o"][i], r["lse"][i]
        at = min(at + c, n)
    return o, lse, at


def items_of(plan):
    """The plan's header, items [12] and units of the merge [8]."""
    a = plan._items.cpu().numpy()
    n, j, rows, room = a[:4].tolist()
    at = 16 + 2 * plan.requests + 1
    joins = at + 12 * room
    assert n <= room and joins + 8 * j <= len(a)
    return n, j, rows, a[at:at + 12 * n].reshape(-1, 12), a[joins:joins + 8 * j].reshape(-1, 8)


def check_plan(plan, lens, seqs, counts, group, f32, block, window, sinks):
    """Every tile of rows once, its chunks in order over the keys that its rows see; partial rows apart."""
    n, j, rows, items, joins = items_of(plan)
    starts = plan.starts.cpu().tolist()
    at, want = 0, {}
    for r, (s, c) in enumerate(zip(seqs, counts)):
        c = max(c, 0)
        assert starts[r] == min(at, plan.rows)
        used = min(c, plan.rows - min(at, plan.rows))
        per = used * group
        tr = 16 if f32 else 128 if per > 64 else 32
        length = lens[s] if 0 <= s < len(lens) else 0
        vis = window_util.visible(c, length, block, window, sinks)
        for t in range(-(-per // tr)):
            r0, r1 = t * tr, min(per, t * tr + tr)
            mine = slice(r0 // group, (r1 - 1) // group + 1)
            seen = torch.nonzero(vis[mine].any(0)).flatten().tolist()
            # (windows shorter than a block leave keys between them, and behind the last, that no row sees: they are walked too)
            ends = [block * (x // block + 1) for x in (length - c + i for i in range(mine.start, mine.stop)) if x >= 0]
            if ends:
                seen = sorted(set(seen) | set(range(max(0, ends[0] - window) if window else 0, min(ends[-1], length))))
            want[(starts[r], r0)] = (r1 - r0, seen, s if length or 0 <= s < len(lens) else -1, tr)
        at += used if at >= plan.rows else c
    assert rows == min(sum(max(c, 0) for c in counts), plan.rows)
    got = {}
    for x in items.tolist():
        got.setdefault((x[1], x[4]), []).append(x)
    assert sorted(got) == sorted(want)
    parts = []
    for key, xs in got.items():
        nrows, seen, seq, tr = want[key]
        xs.sort(key=lambda x: x[6])
        assert all(x[5] == nrows and x[0] == seq for x in xs)
        assert xs[0][6] == 0 and all(a[7] == b[6] for a, b in zip(xs, xs[1:]))
        gap_at, gap, w0, end = xs[0][8], xs[0][9], xs[0][10], xs[-1][7]
        walked = [v if v < gap_at else v + gap for v in range(end) if v < sinks or not window or v >= w0]
        assert walked == seen, (key, len(walked), len(seen))
        assert all(x[7] - x[6] > 0 for x in xs) or (len(xs) == 1 and not seen)
        for c, x in enumerate(xs):
            part = x[11]
            shared = bool((part if part >= 0 else ~part) & 1 << 30)
            assert shared == (tr == 128) and (part < 0) == (len(xs) == 1)
            if part >= 0:
                p = part & ~(1 << 30)
                assert p == (xs[0][11] & ~(1 << 30)) + c * nrows
                parts.append((p, p + nrows))
    parts.sort()
    assert all(a[1] <= b[0] for a, b in zip(parts, parts[1:]))
    # the merge's units: every row of the cut tiles once
    joined = {}
    for token0, row0, nrows, part, m, step, *_ in joins.tolist():
        assert nrows >= 1
        for i in range(nrows):
            assert joined.setdefault((token0, row0 + i), (part + i, m, step)) == (part + i, m, step)
    cut = {(key[0], key[1] + i): ((xs[0][11] & ~(1 << 30)) + i, len(xs), xs[0][5])
           for key, xs in got.items() if len(xs) > 1 for i in range(xs[0][5])}
    assert joined == cut and sum(x[2] for x in joins.tolist()) == len(cut)
    return n, j


def attend(lens, counts, H, KV, D, dtype, page=16, seqs=None, pad=0, seed=0, block=1, window=0, sinks=0, scale=0.0, cache=None,
           layer=0, layers=1, q=None):
    cache = cache or make_cache(lens, KV, D, dtype, page, layers, seed)
    seqs = list(range(len(counts))) if seqs is None else seqs
    rows = sum(max(c, 0) for c in counts) + pad
    if q is None:
        q = torch.randn(rows, H, D, generator=torch.Generator().manual_seed(seed + 1)).to(dtype).to(DEV)
    plan = bd.chunk_plan(cache, i32(seqs), i32(counts), rows=rows, heads=H, block_size=block, window=window, sinks=sinks, scale=scale)
    o, lse = bd.chunk_attn(plan, q, layer)
    torch.cuda.synchronize()
    check_plan(plan, cache.lens.tolist(), seqs, counts, H // KV, dtype == F32, block, window, sinks)
    ro, rl, used = oracle(cache, seqs, counts, q, layer, scale or None, block, window, sinks)
    check("o", o, *ro)
    check("lse", lse, *rl)
    assert bool((o[used:] == 0).all()) and bool((lse[:, used:] == -math.inf).all())
    return cache, plan, q, o, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 24, 1, 100])
def test_mixed_requests(dtype, D, page):
    attend([1, 40, 333, 17, 64, 500], [1, 1, 70, 17, 5, 1], 4, 2, D, dtype, page, pad=3, seed=page)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [2, 4, 7, 8, 12, 40])
def test_pages_that_are_no_whole_groups(D, page):
    # copies of 4 or 8 rows share a page or do not; walks with a gap; whole tiles and ends of pages inside them
    attend([900, 333, 40, 1], [130, 1, 33, 1], 4, 2, D, BF, page, pad=2, seed=page)
    attend([900, 333, 40, 1], [130, 1, 33, 1], 4, 2, D, BF, page, seed=page + 1, window=150, sinks=5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KV", [(1, 1), (3, 1), (8, 2), (6, 6), (24, 1)])
def test_heads(dtype, H, KV):
    for D in (64, 128):
        attend([77, 300], [33, 1], H, KV, D, dtype, seed=H)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (40, 0), (100, 16), (64, 70), (1000, 4), (7, 300)])
def test_windows_and_sinks(dtype, page, window, sinks):
    attend([1, 200, 333, 450, 90], [1, 1, 100, 3, 90], 4, 2, 64, dtype, page, seed=window + sinks, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block,window,sinks", [(2, 0, 0), (32, 0, 0), (32, 48, 4), (17, 5, 3), (128, 5, 4), (1000, 30, 2), (1 << 28, 0, 0)])
def test_blocks(dtype, block, window, sinks):
    attend([10, 200, 333, 130], [10, 1, 100, 64], 4, 2, 64, dtype, 10, seed=3, block=block, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_short_tables(dtype):
    # the last page of a table that is as long as its sequence, blocks that end behind it
    cache = make_cache([10, 20, 7], 2, 64, dtype, 10, extra=0)
    for kw in (dict(block=128, window=5, sinks=4), dict(block=64), dict(window=3, sinks=30), dict(block=16, window=16, sinks=1)):
        attend(None, [10, 3, 1], 4, 2, 64, dtype, cache=cache, **kw)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_lists_that_name_nothing(dtype):
    cache = make_cache([40, 0, 12], 2, 64, dtype, 16)
    attend(None, [3, 2, 5, 4], 4, 2, 64, dtype, cache=cache, seqs=[0, 7, -1, 1])   # numbers out of range, an empty sequence
    attend(None, [0, -5, 3, 0], 4, 2, 64, dtype, cache=cache, seqs=[0, 2, 0, 2])   # counts of nothing
    attend(None, [20, 50], 4, 2, 64, dtype, cache=cache, seqs=[2, 0])              # more rows than tokens
    attend(None, [2, 2, 2], 4, 2, 64, dtype, cache=cache, seqs=[0, 0, 0])          # the same sequence again
    attend(None, [], 4, 2, 64, dtype, cache=cache, seqs=[], pad=5)                 # no request
    plan = bd.chunk_plan(cache, i32([0]), i32([3]), rows=0, heads=4)
    o, lse = bd.chunk_attn(plan, torch.zeros(0, 4, 64, dtype=dtype, device=DEV), 0)
    assert o.shape == (0, 4, 64) and lse.shape == (4, 0)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_past_the_tensors_are_passed_over(dtype):
    cache = make_cache([300, 40, 50], 2, 64, dtype, 16)
    q = torch.randn(25, 4, 64, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    seqs, counts = [0, 1, 2], [20, 2 ** 31 - 1, 10]
    plan = bd.chunk_plan(cache, i32(seqs), i32(counts), rows=25, heads=4)
    o, lse = bd.chunk_attn(plan, q, 0)
    ro, rl, _ = oracle(cache, [0], [20], q[:20])
    check("o", o[:20], *ro)
    check("lse", lse[:, :20], *rl)
    assert bool((o[20:] == 0).all()) and bool((lse[:, 20:] == -math.inf).all())  # far before their sequence's start
    assert plan.starts.tolist() == [0, 20, 25]


def test_lengths_and_pages_out_of_contract():
    # lens past the table or negative, pages out of the cache (rows of zeros): nothing is read outside the tensors
    cache = make_cache([64, 64, 64], 2, 64, BF, 16, extra=0)
    cache.lens.copy_(i32([1 << 30, -5, 64]))
    cache.table[2, 1], cache.table[2, 3] = 999, -7
    q = torch.randn(9, 4, 64, generator=torch.Generator().manual_seed(6)).to(BF).to(DEV)
    plan = bd.chunk_plan(cache, i32([0, 1, 2]), i32([3, 3, 3]), rows=9, heads=4)
    o, lse = bd.chunk_attn(plan, q, 0)
    torch.cuda.synchronize()
    good = make_cache([64, 64, 64], 2, 64, BF, 16, extra=0)
    for p in (999, -7):
        good.table[2][cache.table[2] == p] = 0
    k, v = rows_of(good, 2, 64, 0)
    for a in (slice(16, 32), slice(48, 64)):
        k[a], v[a] = 0, 0
    vis = window_util.visible(3, 64)
    for h in range(4):
        r = head(q[6:, h].cpu().double(), k[:, h // 2], v[:, h // 2], vis, 0.125, BF)
        check("o", o[6:, h], *r["o"])
    ro, _, _ = oracle(make_cache([64, 64, 64], 2, 64, BF, 16, extra=0), [0], [3], q[:3])
    check("o", o[:3], *ro)
    assert bool((o[3:6] == 0).all()) and bool((lse[:, 3:6] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("page", [16, 24])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_keys_that_no_row_sees_may_hold_anything(dtype, page, bad):
    cache = make_cache([400, 90, 50], 2, 64, dtype, page, seed=7)
    window, sinks, counts = 30, 5, [20, 1, 3]
    for s, (n, c) in enumerate(zip((400, 90, 50), counts)):
        for t in range(sinks, n - c + 1 - window):
            p, r = int(cache.table[s, t // page]), t % page
            cache.k[0, p, r], cache.v[0, p, r] = bad, bad
    attend(None, counts, 4, 2, 64, dtype, cache=cache, window=window, sinks=sinks)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 24])
def test_cut_walks(D, page):
    lens, counts = [9000, 3000, 50, 5000], [1, 40, 50, 2]
    _, plan, *_ = attend(lens, counts, 8, 2, D, BF, page, seed=8)
    assert items_of(plan)[1] > 0
    _, plan, *_ = attend(lens, counts, 8, 2, D, BF, page, seed=9, window=2500, sinks=70)
    assert items_of(plan)[1] > 0


def test_cut_walks_fp32():
    _, plan, *_ = attend([3000, 900, 20], [1, 6, 20], 4, 2, 64, F32, 24, seed=10)
    assert items_of(plan)[1] > 0


def test_many_chunks_of_a_walk():
    # one request of one KV head: more parts than are joined the short way
    _, plan, *_ = attend([20000], [1], 2, 1, 64, BF, 16, seed=11)
    assert items_of(plan)[0] > 16


def test_walks_longer_than_a_chunk_may_be():
    # pages of one token: 2,044 keys a chunk
    _, plan, *_ = attend([9000] * 3, [1, 2, 1], 2, 2, 64, BF, 1, seed=12)
    assert items_of(plan)[0] >= 15


@pytest.mark.parametrize("rows", [1, 100])
def test_a_whole_chunk_of_groups(rows):
    # one sequence named 56 times: walks of 32,600 keys, which a workgroup's table of groups just holds, and longer ones
    _, plan, *_ = attend([32600], [rows] * 56, 8, 8, 64, BF, 16, seqs=[0] * 56, seed=14)
    assert items_of(plan)[0] == 56
    _, plan, *_ = attend([32700], [rows] * 56, 8, 8, 64, BF, 16, seqs=[0] * 56, seed=15)
    assert items_of(plan)[0] == 112


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scales_and_layers(dtype):
    attend([100, 50], [10, 1], 4, 2, 64, dtype, seed=13, scale=0.5, layers=3, layer=2)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_and_given_outputs(dtype):
    cache = make_cache([100, 50], 2, 64, dtype, 16, seed=14)
    wide = torch.randn(15, 9, 64, generator=torch.Generator().manual_seed(14)).to(dtype).to(DEV)
    q = wide[:, 2:6]
    plan = bd.chunk_plan(cache, i32([0, 1]), i32([10, 2]), rows=15, heads=4, window=20, sinks=3)
    o, lse = bd.chunk_attn(plan, q, 0)
    ro, rl, _ = oracle(cache, [0, 1], [10, 2], q, 0, None, 1, 20, 3)
    check("o", o, *ro)
    out = torch.full((15, 7, 64), 7.0, dtype=dtype, device=DEV)
    z = torch.full((4, 15), 7.0, device=DEV)
    ws = torch.empty(max(256, bd.chunk_attn_workspace_bytes(plan)), dtype=torch.uint8, device=DEV)
    bd.chunk_attn(plan, q, 0, out=(out[:, 1:5], z), workspace=ws)
    assert torch.equal(out[:12, 1:5], o[:12]) and torch.equal(z[:, :12], lse[:, :12])
    assert bool((out[12:] == 7).all()) and bool((z[:, 12:] == 7).all()) and bool((out[:, 0] == 7).all()) and bool((out[:, 5:] == 7).all())


@pytest.mark.parametrize("dtype", [BF, F32])
def test_it_is_packed_attention_over_pages(dtype):
    # the same rule as packed calls: chunks of prompts, keys gathered from the pages
    lens, counts, H, KV, D = [130, 300, 70], [130, 40, 1], 4, 2, 64
    cache = make_cache(lens, KV, D, dtype, 16, seed=15)
    q = torch.randn(sum(counts), H, D, generator=torch.Generator().manual_seed(15)).to(dtype).to(DEV)
    k, v = (torch.cat([rows_of(cache, s, n, 0)[i] for s, n in enumerate(lens)]).to(dtype).to(DEV) for i in range(2))
    for kw in (dict(), dict(window=50, sinks=9), dict(block_size=32, window=50, sinks=9)):
        plan = bd.packed_plan(counts, lens, heads=H, kv_heads=KV, head_dim=D, dtype=dtype, **kw)
        po, pz = bd.packed_fwd(plan, q, k, v)
        o, z = bd.chunk_attn(bd.chunk_plan(cache, i32([0, 1, 2]), i32(counts), rows=sum(counts), heads=H, **kw), q, 0)
        ro, rl, _ = oracle(cache, [0, 1, 2], counts, q, 0, None, kw.get("block_size", 1), kw.get("window", 0), kw.get("sinks", 0))
        for a, b in ((po, o), (pz, z)):
            bound = (ro if a.dim() == 3 else rl)[1]
            assert bool(((a - b).abs().double().cpu() <= 2 * bound).all())
        check("o", o, *ro)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_steps_of_a_layer(dtype):
    """As it is used: prompts in pieces beside decoding, with rotated queries and keys, through a cache that grows."""
    H, KV, D, page, window, sinks = 4, 2, 64, 16, 24, 3
    dims = dict(layers=2, pages=60, page_size=page, kv_heads=KV, head_dim=D, seqs=4, max_pages=12)
    cache = bd.cache_new(**dims, dtype=dtype)
    rot, gen = bd.rotary(D), torch.Generator().manual_seed(16)
    w = [(1 + 0.1 * torch.randn(D, generator=gen)).to(dtype).to(DEV) for _ in range(2)]
    past = {s: [[], []] for s in range(4)}  # rotated keys and values of each layer
    length = [0] * 4
    for seqs, counts in (([2], [50]), ([0, 2], [33, 1]), ([0, 2, 1], [1, 1, 70]), ([1, 0, 3, 2], [20, 1, 5, 1]), ([3, 2, 1, 0], [1, 1, 1, 1])):
        rows = sum(counts) + 2
        s, c = i32(seqs), i32(counts)
        bd.cache_grow(cache, s, c)
        plan = bd.chunk_plan(cache, s, c, rows=rows, heads=H, window=window, sinks=sinks)
        pos = torch.zeros(rows, dtype=torch.int32)
        at = 0
        for x, n in zip(seqs, counts):
            pos[at:at + n] = torch.arange(length[x], length[x] + n)
            at += n
            length[x] += n
        for layer in range(2):
            qkv = torch.randn(rows, H + 2 * KV, D, generator=gen).to(dtype).to(DEV)
            q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
            qr, kr = bd.qk_rotate_fwd(rot, q, k, pos.to(DEV), *w, eps=1e-6)
            bd.cache_write(cache, layer, s, c, kr, v, starts=plan.starts)
            o, lse = bd.chunk_attn(plan, qr, layer)
            at = 0
            for x, n in zip(seqs, counts):
                past[x][layer].append((kr[at:at + n].cpu(), v[at:at + n].cpu()))
                kk, vv = (torch.cat([p[i] for p in past[x][layer]]).double() for i in range(2))
                vis = window_util.visible(n, length[x], 1, window, sinks)
                for h in range(H):
                    r = head(qr[at:at + n, h].cpu().double(), kk[:, h // 2], vv[:, h // 2], vis, D ** -0.5, dtype)
                    check("o", o[at:at + n, h], *r["o"])
                at += n
    assert cache.status.tolist() == [0, 0] and cache.lens.tolist() == length


def test_replays_of_a_graph_equal_eager_steps():
    """A decoding step captured with its plan: lengths and lists change between the replays."""
    H, KV, D = 8, 2, 128
    cache = make_cache([3000, 500, 64, 1000], KV, D, BF, 16, layers=2, seed=17, extra=4)
    sets = [([0, 1, 2, 3], [1, 1, 1, 1]), ([3, 1, 0, 2], [2, 0, 1, 1]), ([0, 0, 2, 1], [1, 1, 1, 1])]
    lens = [[3000, 500, 64, 1000], [2000, 3, 40, 999], [1, 500, 64, 10]]
    s, c = i32(sets[0][0]), i32(sets[0][1])
    q = torch.randn(2, 6, H, D, generator=torch.Generator().manual_seed(17)).to(BF).to(DEV)

    def step():
        plan = bd.chunk_plan(cache, s, c, rows=6, heads=H, window=700, sinks=4)
        return plan, [bd.chunk_attn(plan, q[layer], layer) for layer in range(2)]

    def load(i):
        s.copy_(i32(sets[i][0]))
        c.copy_(i32(sets[i][1]))
        cache.lens.copy_(i32(lens[i]))

    expect = []
    for i in range(3):
        load(i)
        expect.append([t.clone() for o in step()[1] for t in o])
    load(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        plan, outs = step()
    for i in (1, 2, 0, 1, 2):
        load(i)
        for o in outs:
            for t in o:
                t.fill_(math.nan)
        graph.replay()
        torch.randn(512, 512, device=DEV).sum().item()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([t for o in outs for t in o], expect[i])), i


def test_one_plan_on_two_streams_and_again():
    cache = make_cache([2000, 500, 64], 2, 128, BF, 16, seed=18)
    q = torch.randn(2, 42, 8, 128, generator=torch.Generator().manual_seed(18)).to(BF).to(DEV)
    plan = bd.chunk_plan(cache, i32([0, 1, 2]), i32([1, 1, 40]), rows=42, heads=8)
    a = [bd.chunk_attn(plan, q[i], 0) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    b = [bd.chunk_attn(plan, q[i], 0, stream=streams[i]) for i in range(2)]
    for st in streams:
        torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(x, y) for p, r in zip(a, b) for x, y in zip(p, r))
    # another step's plan in the same memory
    again = bd.chunk_plan(cache, i32([2, 1, 0]), i32([20, 20, 2]), rows=42, heads=8, window=30, sinks=2, out=plan)
    fresh = bd.chunk_plan(cache, i32([2, 1, 0]), i32([20, 20, 2]), rows=42, heads=8, window=30, sinks=2)
    assert again is plan
    assert all(torch.equal(x, y) for x, y in zip(bd.chunk_attn(plan, q[0], 0), bd.chunk_attn(fresh, q[0], 0)))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_plan_made_anew_with_another_window(dtype):
    lens, counts = [3000, 700, 90, 1], [3, 100, 90, 1]
    cache = make_cache(lens, 2, 64, dtype, 16, seed=21)
    q = torch.randn(sum(counts), 4, 64, generator=torch.Generator().manual_seed(22)).to(dtype).to(DEV)
    lists = cache, i32([0, 1, 2, 3]), i32(counts)
    plan = bd.chunk_plan(*lists, rows=len(q), heads=4, window=30, sinks=3)
    for window, sinks in ((30, 3), (0, 0), (500, 0), (30, 3), (64, 700)):
        assert bd.chunk_plan(*lists, rows=len(q), heads=4, window=window, sinks=sinks, out=plan) is plan
        got = bd.chunk_attn(plan, q, 0)
        want = attend(lens, counts, 4, 2, 64, dtype, cache=cache, q=q, window=window, sinks=sinks)[3:]
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_many_requests():
    # more requests than the planner's threads, and than its table in LDS
    n, KV, D = 9000, 1, 64
    lens = [1 + (i * 7) % 40 for i in range(n)]
    cache = make_cache(lens, KV, D, BF, 16, seed=19)
    counts = [min(1 + i % 3, lens[i]) if i % 5 else 0 for i in range(n)]
    rows = sum(counts)
    q = torch.randn(rows, 2, D, generator=torch.Generator().manual_seed(19)).to(BF).to(DEV)
    plan = bd.chunk_plan(cache, i32(range(n)), i32(counts), rows=rows, heads=2)
    o, lse = bd.chunk_attn(plan, q, 0)
    starts = np.cumsum([0] + counts)
    assert plan.starts.tolist() == starts[:-1].tolist()
    some = list(range(0, n, 401)) + [n - 1]
    pick = torch.cat([torch.arange(starts[i], starts[i + 1]) for i in some])
    ro, rl, _ = oracle(cache, some, [counts[i] for i in some], q[pick.to(DEV)])
    check("o", o[pick.to(DEV)], *ro)
    check("lse", lse[:, pick.to(DEV)], *rl)
    assert not bool(o.isnan().any())


def test_caches_past_32_bits():
    # 5 GB of keys: rows beyond 2^32 bytes and 2^31 elements
    KV, D, page, pages = 8, 128, 64, 39000
    k, v = (torch.zeros(1, pages, page, KV, D, dtype=BF, device=DEV) for _ in range(2))
    g = torch.Generator().manual_seed(20)
    table = torch.tensor([[pages - 1, 3, pages - 2, pages // 2]], dtype=torch.int32)
    for p in table[0].tolist():
        k[0, p], v[0, p] = (torch.randn(page, KV, D, generator=g).to(BF).to(DEV) for _ in range(2))
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    cache = bd.Cache(k, v, table.to(DEV), i32([230]), refs, torch.zeros(2, dtype=torch.int32, device=DEV))
    where = table[0].long()[torch.arange(230) // page] * page + torch.arange(230) % page
    kk, vv = (x[0].flatten(0, 1)[where.to(DEV)].cpu().double() for x in (k, v))
    for count in (1, 40):
        q = torch.randn(count, 8, D, generator=g).to(BF).to(DEV)
        o, _ = bd.chunk_attn(bd.chunk_plan(cache, i32([0]), i32([count]), rows=count, heads=8, window=100, sinks=70), q, 0)
        vis = window_util.visible(count, 230, 1, 100, 70)
        for h in range(8):
            check("o", o[:, h], *head(q[:, h].cpu().double(), kk[:, h], vv[:, h], vis, D ** -0.5, BF)["o"])
