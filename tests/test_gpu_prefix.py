"""Attention of decoding requests over a paged cache against the 64-bit oracle: rows from one token to blocks, prefixes
that end inside pages and tiles, pages of every size, requests without tokens, chunks and partial sums."""
import math
import random

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import check, head

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def build(lens, prefix, ps, KV, D, dtype, seed, layers=1, spare=2, slots=None):
    """A cache whose first sequences hold `lens` tokens; full prefix pages shared, a partial one copied; whatever no
    token holds is NaN."""
    rng = random.Random(seed)
    full = prefix // ps
    need = [-(-n // ps) for n in lens]
    pages = full + sum(max(0, n - full) for n in need) + 3
    order = list(range(pages))
    rng.shuffle(order)
    S, mp = slots or len(lens), max(need + [1]) + spare
    table = torch.full((S, mp), -1, dtype=torch.int32)
    at = full
    for r, n in enumerate(need):
        for i in range(n):
            if i < full:
                table[r, i] = order[i]
            else:
                table[r, i] = order[at]
                at += 1
    shape = (layers, pages, ps, KV, D)
    kv = [torch.full(shape, math.nan, dtype=dtype) for _ in range(2)]
    for r, n in enumerate(lens):
        for t, x in enumerate(kv):
            for p0 in range(0, n, ps):
                m = min(ps, n - p0)
                x[:, table[r, p0 // ps], :m] = synth.normal((layers, m, KV, D), seed * 1000 + 2 * p0 + t if p0 < prefix
                                                            else seed * 1000 + 7919 * (r + 1) + 2 * p0 + t, dtype)
    if prefix % ps:  # the prefix's rows in each request's own page
        for r in range(1, len(lens)):
            if need[r] > full and need[0] > full:
                for x in kv:
                    m = min(prefix % ps, lens[r] - full * ps, lens[0] - full * ps)
                    x[:, table[r, full], :m] = x[:, table[0, full], :m]
    ln = torch.zeros(S, dtype=torch.int32)
    ln[:len(lens)] = torch.tensor(lens, dtype=torch.int32)
    refs = torch.bincount(table[table >= 0].long(), minlength=pages).int()
    return bd.Cache(*[t.to(DEV) for t in (*kv, table, ln, refs, torch.zeros(2, dtype=torch.int32))])


def oracle(q, cache, layer, seqs, block, scale=None):
    R, n, H, D = q.shape
    KV, ps = cache.kv_heads, cache.page_size
    table, lens = cache.table.cpu(), cache.lens.cpu().tolist()
    k, v = cache.k[layer].cpu().double(), cache.v[layer].cpu().double()
    Q = q.cpu().double()
    scale = scale or 1.0 / math.sqrt(D)
    out = {"o": [torch.zeros(R, n, H, D, dtype=torch.float64) for _ in range(2)],
           "lse": [torch.zeros(R, H, n, dtype=torch.float64) for _ in range(2)]}
    for r, s in enumerate(seqs):
        L = lens[s] if 0 <= s < cache.seqs else 0
        pages = table[s, :-(-L // ps)].long() if L else torch.zeros(0, dtype=torch.long)
        kk, vv = (x[pages].reshape(-1, KV, D)[:L] for x in (k, v))
        i, j = torch.arange(n)[:, None], torch.arange(L)[None]
        vis = (j < L).expand(n, L) if block else j <= L - n + i
        for h in range(H):
            res = head(Q[r, :, h], kk[:, h // (H // KV)], vv[:, h // (H // KV)], vis, scale, q.dtype)
            for t in range(2):
                out["o"][t][r, :, h] = res["o"][t]
                out["lse"][t][r, h] = res["lse"][t]
    return out


def run(lens, prefix, n, H, KV, D, dtype, ps=16, block=False, seqs=None, seed=1, scale=0.0, layers=1, layer=0, **kw):
    c = build(lens, prefix, ps, KV, D, dtype, seed, layers=layers, **kw)
    seqs = list(range(len(lens))) if seqs is None else seqs
    q = synth.normal((len(seqs), n, H, D), seed + 50, dtype).to(DEV)
    o, lse = bd.prefix_attn(q, c, layer, i32(seqs), prefix, block=block, scale=scale)
    torch.cuda.synchronize()
    ref = oracle(q, c, layer, seqs, block, scale or None)
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])
    return c, q, o, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("H,KV,D", [(4, 2, 128), (4, 4, 64), (6, 1, 128), (8, 8, 64), (3, 1, 64), (40, 1, 64)])
def test_one_token_each(H, KV, D, dtype):
    run([130, 101, 300, 170], 100, 1, H, KV, D, dtype)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("ps", [1, 5, 16, 24, 64, 100, 256])
def test_page_sizes(ps, dtype):
    run([90, 71, 140], 70, 2, 4, 2, 64, dtype, ps=ps, seed=3)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 64, 65, 128, 200])
@pytest.mark.parametrize("block", [False, True])
def test_prefixes(prefix, block, dtype):
    run([205, 204, 333], prefix, 4, 4, 2, 128, dtype, block=block, seed=5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [False, True])
@pytest.mark.parametrize("n,H,KV", [(3, 4, 4), (9, 4, 2), (17, 8, 2), (32, 8, 1), (33, 4, 2), (70, 4, 1)])
def test_blocks_of_rows(n, H, KV, block, dtype):
    run([200, 150, 90, 161], 80, n, H, KV, 64, dtype, block=block, seed=7)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("block", [False, True])
def test_rows_that_see_nothing(block, dtype):
    """More rows than tokens, sequences without tokens, numbers out of range."""
    run([3, 0, 20, 1], 0, 5, 4, 2, 128, dtype, block=block, seed=9)
    run([40, 0, 33], 0, 2, 4, 2, 64, dtype, block=block, seqs=[0, 1, 2, 99, -1, 2, 2], seed=11)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_requests_shorter_than_the_prefix(dtype):
    run([64, 20, 64, 7], 64, 3, 4, 2, 64, dtype, seed=13)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_long_prefix_in_chunks(dtype):
    run([2100, 2071, 2600], 2064, 1, 4, 2, 64 if dtype == F32 else 128, dtype, seed=15)


# Prefixes long enough to be kept apart (shorter ones are read with each request's own keys): few rows and many, pages
# that the prefix ends in, rows that lie in the prefix themselves, requests that are not longer than it.
@pytest.mark.parametrize("ps", [16, 24, 100])
@pytest.mark.parametrize("dtype,R,P,n,H,KV,D,block", [
    (BF, 9, 2003, 1, 16, 4, 128, False), (BF, 9, 2003, 1, 4, 4, 64, False), (BF, 24, 1100, 1, 8, 2, 128, False),
    (BF, 8, 2500, 5, 8, 2, 128, False), (BF, 8, 2500, 5, 8, 2, 128, True), (BF, 6, 3001, 32, 16, 2, 128, True),
    (BF, 33, 1025, 9, 4, 2, 64, False), (F32, 7, 1200, 1, 4, 2, 128, False), (F32, 9, 1601, 6, 6, 2, 64, False)])
def test_prefixes_kept_apart(ps, dtype, R, P, n, H, KV, D, block):
    lens = [P + (0 if r == 3 else 1 + (r * 37) % 130) for r in range(R)]
    c, q, o, lse = run(lens, P, n, H, KV, D, dtype, ps=ps, block=block, seed=33)
    parts = bd.prefix_attn_workspace_bytes(q, c, P) // (R * n * H * (D + 1) * 4)
    assert parts >= 2


# Requests whose rows fill tiles by themselves, cut up whole into equal chunks (the last two tables hold too much beside
# the prefix, or the tiles too few rows, for that): ragged, one without tokens, one in the prefix, one out of range.
@pytest.mark.parametrize("ps", [16, 24])
@pytest.mark.parametrize("P,n,H,KV,D,block,spare", [
    (3001, 32, 16, 2, 128, True, 2), (3001, 33, 8, 1, 128, False, 2), (2500, 120, 2, 2, 64, False, 2),
    (3001, 32, 16, 2, 128, False, 300), (3001, 9, 16, 2, 128, False, 2)])
def test_requests_that_fill_tiles(P, n, H, KV, D, block, spare, ps):
    lens = [P + 40, P + 513, 0, P - 700, P + 128, P + 1]
    c, q, o, lse = run(lens, P, n, H, KV, D, BF, ps=ps, block=block, seed=35, spare=spare, seqs=[0, 1, 2, 3, 4, 5, 77])
    assert bd.prefix_attn_workspace_bytes(q, c, P) >= 2 * 7 * n * H * (D + 1) * 4


def test_one_long_request():
    run([5000], 0, 1, 8, 1, 128, BF, seed=17)
    run([5000], 4999, 1, 8, 1, 128, BF, seed=17)


def test_many_rows_share_the_prefix():
    run([700 + 13 * r for r in range(12)], 672, 8, 8, 2, 128, BF, seed=19)
    run([700 + 13 * r for r in range(5)], 672, 32, 8, 1, 64, BF, block=True, seed=19)


def test_layers_and_scale():
    run([130, 60], 48, 2, 4, 2, 64, BF, layers=3, layer=2, scale=0.3, seed=21)


def test_sequences_in_another_order():
    run([130, 101, 300, 170], 96, 1, 4, 2, 128, BF, seqs=[2, 0, 3, 3], seed=23)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_page_numbers_outside_the_cache_read_as_zeros(dtype):
    c = build([100, 90], 0, 16, 2, 64, dtype, 25)
    c.table[0, 2] = c.pages
    c.table[1, 0] = -7
    c.table[1, 3] = 1 << 30
    q = synth.normal((2, 1, 4, 64), 75, dtype).to(DEV)
    o, lse = bd.prefix_attn(q, c, 0, i32([0, 1]))
    torch.cuda.synchronize()
    z = bd.Cache(torch.cat([c.k, torch.zeros_like(c.k[:, :1])], 1), torch.cat([c.v, torch.zeros_like(c.v[:, :1])], 1),
                 torch.where((c.table < 0) | (c.table >= c.pages), c.pages, c.table), c.lens,
                 torch.cat([c.refs, c.refs[:1]]), c.status)
    ref = oracle(q, z, 0, [0, 1], False)
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])


def test_lengths_outside_the_table_are_taken_at_its_end():
    c = build([100, 90], 0, 16, 2, 64, BF, 27, spare=0)
    top = c.max_pages * 16
    assert top == 112
    c.k.nan_to_num_(0.25), c.v.nan_to_num_(0.5)
    q = synth.normal((2, 1, 4, 64), 75, BF).to(DEV)
    c.lens[0] = 1 << 30
    c.lens[1] = -3
    o, lse = bd.prefix_attn(q, c, 0, i32([0, 1]))
    torch.cuda.synchronize()
    c.lens[0], c.lens[1] = top, 0
    ref = oracle(q, c, 0, [0, 1], False)
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])


def test_prefix_given_or_not_is_the_same_attention():
    c, q, o, lse = run([700, 650, 800], 640, 1, 8, 2, 128, BF, seed=29)
    o2, lse2 = bd.prefix_attn(q, c, 0, i32([0, 1, 2]), 0)
    torch.cuda.synchronize()
    ref = oracle(q, c, 0, [0, 1, 2], False)
    check("o", o2, *ref["o"])
    check("lse", lse2, *ref["lse"])


def test_graph_replays_follow_the_lengths():
    c = build([130, 101, 300], 96, 16, 2, 128, BF, 31)
    for x in (c.k, c.v):
        x.nan_to_num_(0.5)
    q = synth.normal((3, 1, 4, 128), 75, BF).to(DEV)
    seqs = i32([0, 1, 2])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        bd.prefix_attn(q, c, 0, seqs, 96)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, lse = bd.prefix_attn(q, c, 0, seqs, 96)
    for i in range(4):
        c.lens.copy_(torch.tensor([130 + i, 101 + 2 * i, 300 + i], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        e, el = bd.prefix_attn(q, c, 0, seqs, 96)
        torch.cuda.synchronize()
        assert torch.equal(o, e) and torch.equal(lse, el)
        ref = oracle(q, c, 0, [0, 1, 2], False)
        check("o", o, *ref["o"])


def test_a_whole_decoding_run():
    """Prompts of different lengths through packed attention, their keys into the cache, forks that share them, and steps
    of one token against the cache: every step equals packed attention over the sequence as a whole."""
    H, KV, D, ps = 4, 2, 64, 16
    plens, steps = [50, 33], 3
    c = bd.cache_new(1, 64, ps, KV, D, 8, 8, BF, DEV)
    n = sum(plens)
    qkv = synth.normal((n, H + 2 * KV, D), 3, BF).to(DEV)
    q, k, v = qkv[:, :H], qkv[:, H:H + KV], qkv[:, H + KV:]
    plan = bd.packed_plan(plens, heads=H, kv_heads=KV, head_dim=D, dtype=BF)
    bd.packed_fwd(plan, q, k, v)
    bd.cache_grow(c, i32([0, 1]), i32(plens))
    bd.cache_write(c, 0, i32([0, 1]), i32(plens), k, v, starts=i32([0, plens[0]]))
    bd.cache_fork(c, i32([0, 0, 1]), i32([2, 3, 4]))
    live = [2, 3, 4]
    keys = {2: [k[:50], v[:50]], 3: [k[:50], v[:50]], 4: [k[50:], v[50:]]}
    bd.cache_free(c, i32([0, 1]))
    for t in range(steps):
        new = synth.normal((3, H + 2 * KV, D), 40 + t, BF).to(DEV)
        bd.cache_grow(c, i32(live), i32([1] * 3))
        bd.cache_write(c, 0, i32(live), i32([1] * 3), new[:, H:H + KV], new[:, H + KV:])
        group, gl = bd.prefix_attn(new[:2, None, :H].contiguous(), c, 0, i32([2, 3]), 48)  # the two forks of one prompt
        alone, al = bd.prefix_attn(new[2:, None, :H].contiguous(), c, 0, i32([4]))
        for i, s in enumerate(live):
            keys[s] = [torch.cat([keys[s][0], new[i:i + 1, H:H + KV]]), torch.cat([keys[s][1], new[i:i + 1, H + KV:]])]
            m = keys[s][0].shape[0]
            p1 = bd.packed_plan([1], [m], heads=H, kv_heads=KV, head_dim=D, dtype=BF)
            want, wl = bd.packed_fwd(p1, new[i:i + 1, :H].contiguous(), *keys[s])
            got, g2 = (group[i], gl[i]) if i < 2 else (alone[0], al[0])
            torch.cuda.synchronize()
            # both round P and O to bf16: twice the half steps of each, |O| <= max |V| < 5
            assert float((got.float() - want.float()).abs().max()) <= 4 * 5 * 2.0 ** -8
            assert float((g2 - wl).abs().max()) <= 1e-4
    assert c.status.tolist() == [0, 0]
