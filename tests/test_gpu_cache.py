"""Page operations of the cache against their definitions on host lists, after every step of mixed sequences of them."""
import random

import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.cache_oracle import CacheOracle

pytestmark = pytest.mark.gpu
DEV = "cuda"


def i32(xs):
    return torch.tensor(list(xs), dtype=torch.int32, device=DEV)


def fresh(layers=2, pages=40, ps=16, KV=2, D=64, seqs=12, max_pages=6, dtype=torch.bfloat16, seed=1):
    c = bd.cache_new(layers, pages, ps, KV, D, seqs, max_pages, dtype, DEV)
    c.k.copy_(synth.normal(c.k.shape, seed, dtype))
    c.v.copy_(synth.normal(c.v.shape, seed + 1, dtype))
    return c, CacheOracle(c.k.cpu(), c.v.cpu(), c.table.cpu(), c.lens.cpu(), c.refs.cpu())


def rows(n, KV, D, dtype, seed):
    return synth.normal((n, KV, D), seed, dtype)


def both_grow(c, o, seqs, counts):
    bd.cache_grow(c, i32(seqs), i32(counts))
    o.grow(seqs, counts)
    o.compare(c)


@pytest.mark.parametrize("ps", [1, 7, 16, 64])
@pytest.mark.parametrize("dtype,KV,D", [(torch.bfloat16, 2, 64), (torch.float32, 3, 128)])
def test_a_beam_step(ps, dtype, KV, D):
    c, o = fresh(ps=ps, pages=120 if ps < 8 else 40, max_pages=60 if ps < 8 else 6, KV=KV, D=D, dtype=dtype)
    both_grow(c, o, [0, 3, 1], [5, 0, 33])
    for layer in range(2):
        k, v = rows(38, KV, D, dtype, 5 + layer), rows(38, KV, D, dtype, 9 + layer)
        bd.cache_write(c, layer, i32([0, 3, 1]), i32([5, 0, 33]), k.to(DEV), v.to(DEV), starts=i32([0, 5, 5]))
        o.write(layer, [0, 3, 1], [5, 0, 33], k, v, [0, 5, 5])
    o.compare(c)
    pa, ch = [0, 1, 1, 3], [5, 6, 7, 8]
    bd.cache_fork(c, i32(pa), i32(ch))
    o.fork(pa, ch)
    o.compare(c)
    both_grow(c, o, ch, [1, 1, 2, 1])
    k, v = rows(8, KV, D, dtype, 20), rows(8, KV, D, dtype, 21)
    bd.cache_write(c, 1, i32(ch), i32([1, 1, 2, 1]), k.to(DEV), v.to(DEV))
    o.write(1, ch, [1, 1, 2, 1], k, v)
    o.compare(c)
    bd.cache_free(c, i32([1, 0, 1]))
    o.free([1, 0, 1])
    o.compare(c)
    bd.cache_compact(c)
    o.compact()
    o.compare(c)
    bd.cache_free(c, i32([5, 6, 7, 8, 3]))
    o.free([5, 6, 7, 8, 3])
    o.compare(c)
    assert sum(o.refs) == 0


@pytest.mark.parametrize("seed", range(4))
def test_mixed_operations(seed):
    rng = random.Random(seed)
    c, o = fresh(pages=rng.choice([30, 60]), ps=rng.choice([3, 8, 16]), seqs=20, max_pages=9, seed=seed)
    for step in range(25):
        live = [s for s in range(20) if o.lens[s]]
        empty = [s for s in range(20) if not o.lens[s]]
        what = rng.choice(["grow", "grow", "write", "fork", "free", "compact"])
        if what == "grow":
            n = rng.sample(range(20), rng.randint(0, 6))
            both_grow(c, o, n, [rng.randint(0, 3 * o.ps) for _ in n])
        elif what == "write" and live:
            n = rng.sample(live, rng.randint(1, len(live)))
            cnt = [rng.randint(0, min(5, o.lens[s])) for s in n]
            # (pages that are shared are full and stay as they are: only rows behind the shared ones)
            cnt = [min(x, o.lens[s] % o.ps) for x, s in zip(cnt, n)]
            k, v = rows(5 * len(n), 2, 64, torch.bfloat16, step), rows(5 * len(n), 2, 64, torch.bfloat16, 90 + step)
            bd.cache_write(c, 1, i32(n), i32(cnt), k.to(DEV), v.to(DEV))
            o.write(1, n, cnt, k, v)
        elif what == "fork" and live and empty:
            ch = rng.sample(empty, rng.randint(1, len(empty)))
            pa = [rng.choice(live) for _ in ch]
            bd.cache_fork(c, i32(pa), i32(ch))
            o.fork(pa, ch)
        elif what == "free" and live:
            n = [rng.choice(live) for _ in range(rng.randint(1, 4))]
            bd.cache_free(c, i32(n))
            o.free(n)
        else:
            bd.cache_compact(c)
            o.compact()
        o.compare(c)


def test_lists_that_do_not_hold_change_nothing():
    c, o = fresh(pages=8)
    both_grow(c, o, [0, 1], [40, 20])
    for seqs, counts in (([2, 2], [1, 1]), ([-1], [1]), ([12], [1]), ([3], [-1]), ([0], [60]), ([4, 99999], [1, 1])):
        both_grow(c, o, seqs, counts)
        assert o.status[0] == bd.CACHE_BAD_LIST
    for pa, ch in (([0, 0], [5, 5]), ([0], [1]), ([0], [0]), ([50], [3]), ([0], [-3]), ([2, 0], [4, 2])):
        bd.cache_fork(c, i32(pa), i32(ch))
        o.fork(pa, ch)
        o.compare(c)
        assert o.status[0] == bd.CACHE_BAD_LIST
    bd.cache_free(c, i32([99, 1, -5]))
    o.free([99, 1, -5])
    o.compare(c)


def test_too_few_pages():
    c, o = fresh(pages=8)
    both_grow(c, o, [0, 1], [40, 20])  # 5 pages
    both_grow(c, o, [2, 3], [33, 17])  # 5 more of 3
    assert o.status == [bd.CACHE_NO_PAGES, 2]
    both_grow(c, o, [2], [48])
    bd.cache_fork(c, i32([0, 1]), i32([5, 6]))
    o.fork([0, 1], [5, 6])
    o.compare(c)
    assert o.status == [bd.CACHE_NO_PAGES, 2]


def test_empty_lists_and_parents_without_tokens():
    c, o = fresh()
    both_grow(c, o, [], [])
    bd.cache_fork(c, i32([]), i32([]))
    bd.cache_free(c, i32([]))
    bd.cache_write(c, 0, i32([]), i32([]), rows(0, 2, 64, torch.bfloat16, 0).to(DEV), rows(0, 2, 64, torch.bfloat16, 0).to(DEV))
    bd.cache_compact(c)
    o.compare(c)
    bd.cache_fork(c, i32([0, 0]), i32([1, 2]))
    o.fork([0, 0], [1, 2])
    o.compare(c)


def test_rows_and_counts_that_do_not_fit_are_passed_over():
    c, o = fresh()
    both_grow(c, o, [0, 1], [3, 20])
    k, v = (rows(8, 2, 64, torch.bfloat16, s) for s in (3, 4))
    for seqs, counts, starts in (([0, 1], [9, 9], None), ([0, 1], [3, 9], [6, -4]), ([99, -1], [1, 1], None)):
        bd.cache_write(c, 0, i32(seqs), i32(counts), k.to(DEV), v.to(DEV), starts=i32(starts) if starts else None)
        if seqs[0] == 0 and starts is None:
            o.write(0, [0, 1], [9, 9], k, v)
        elif seqs[0] == 0:  # rows 6, 7 of three; rows -4 .. 4 of nine: 0 .. 4 are there
            o.write(0, [0], [3], k, v, [6])
            for j in range(4, 9):
                pos = 20 - 9 + j
                o.k[0, o.table[1][pos // 16], pos % 16] = k[j - 4]
                o.v[0, o.table[1][pos // 16], pos % 16] = v[j - 4]
        o.compare(c)


def test_many_pages_and_sequences():
    """Scans over several rounds of the bookkeeping's threads."""
    c, o = fresh(layers=1, pages=5000, ps=2, KV=1, seqs=1500, max_pages=12)
    seqs = list(range(1500))
    both_grow(c, o, seqs, [(7 * s) % 6 for s in seqs])
    bd.cache_free(c, i32(seqs[::2]))
    o.free(seqs[::2])
    bd.cache_fork(c, i32([1] * 600 + [3] * 150), i32(seqs[::2]))
    o.fork([1] * 600 + [3] * 150, seqs[::2])
    o.compare(c)
    bd.cache_free(c, i32(seqs[1:1200:2]))
    o.free(seqs[1:1200:2])
    bd.cache_compact(c)
    o.compact()
    o.compare(c)


def test_strided_rows_and_another_stream():
    c, o = fresh()
    both_grow(c, o, [2, 4], [17, 17])
    qkv = synth.normal((34, 8, 64), 3, torch.bfloat16).to(DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    seqs, counts = i32([2, 4]), i32([17, 17])
    torch.cuda.synchronize()
    bd.cache_write(c, 0, seqs, counts, qkv[:, 4:6], qkv[:, 6:8], stream=s)
    o.write(0, [2, 4], [17, 17], qkv[:, 4:6].cpu(), qkv[:, 6:8].cpu())
    o.compare(c)


def test_graph_replays():
    c, o = fresh(pages=60)
    both_grow(c, o, [0, 1], [20, 5])
    seqs, one = i32([0, 1]), i32([1, 1])
    k, v = (rows(2, 2, 64, torch.bfloat16, s).to(DEV) for s in (3, 4))
    child, par = i32([7]), i32([0])

    def step():
        bd.cache_grow(c, seqs, one)
        bd.cache_write(c, 0, seqs, one, k, v)
        bd.cache_fork(c, par, child)
        bd.cache_free(c, child)
        bd.cache_compact(c)

    def host():
        o.grow([0, 1], [1, 1])
        o.write(0, [0, 1], [1, 1], k.cpu(), v.cpu())
        o.fork([0], [7])
        o.free([7])
        o.compact()

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    host()
    o.compare(c)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(14):
        k.copy_(rows(2, 2, 64, torch.bfloat16, 40 + i))
        g.replay()
        host()
        o.compare(c)


@pytest.mark.parametrize("pages", [16384, 40007])
def test_many_pages(pages):
    """More pages than a step of the scans takes, sequences that grow by thousands of pages, more than a round of them."""
    S = 1500
    c, o = fresh(layers=1, pages=pages, ps=2, KV=1, seqs=S, max_pages=9000)
    both_grow(c, o, [3], [17001])
    both_grow(c, o, [7, 3, 9], [2000, 0, 1])
    rng = random.Random(pages)
    order = [s for s in rng.sample(range(S), S) if s not in (3, 7, 9)]
    both_grow(c, o, order, [rng.choice([0, 0, 1, 2, 3, 5]) for _ in order])
    gone = [3] + order[::3]
    bd.cache_free(c, i32(gone))
    o.free(gone)
    o.compare(c)
    both_grow(c, o, order[:40], [rng.randrange(0, 300) for _ in range(40)])
    bd.cache_compact(c)
    o.compact()
    o.compare(c)
    both_grow(c, o, [3], [4001])
    both_grow(c, o, [order[0]], [9000])
    both_grow(c, o, [order[1], order[2], order[4]], [16000] * 3)
    both_grow(c, o, [order[5], order[7], order[8]], [17000] * 3)
