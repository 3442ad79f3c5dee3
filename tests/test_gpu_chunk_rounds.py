"""Plans of steps with more tiles, or requests, than the planner takes at a time, in which long walks are cut in several of
its rounds: the plans item by item, and the outputs of the cut rows and of some others."""
import math

import numpy as np
import pytest
import torch

import paper_2609_19242_amd as bd
from tests.serving_util import check
from tests.test_gpu_chunk import check_plan, i32, items_of, make_cache, oracle

pytestmark = pytest.mark.gpu
DEV, BF, F32 = "cuda", torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,n,rows,tiles,window,sinks", [
    (BF, 700, 2, 700, 0, 0), (F32, 700, 2, 700, 0, 0),             # two rounds of 512 tiles
    (BF, 700, 2, 700, 2000, 70),
    (BF, 1100, 60, 2200, 0, 0), (F32, 700, 48, 2100, 0, 0),        # more tiles than are kept in LDS
    (F32, 700, 48, 2100, 1500, 5),
    (BF, 2500, 1, 2500, 0, 0), (F32, 2500, 1, 2500, 2000, 3)])     # more requests than are kept there
def test_rounds_with_cut_walks(dtype, n, rows, tiles, window, sinks):
    D, every = 64, n // 9
    lens = [4000 + 300 * (i // every) if i % every == every // 2 else rows + (i * 7) % 90 for i in range(n)]
    counts = [rows] * n
    cache = make_cache(lens, 1, D, dtype, 16, seed=n)
    q = torch.randn(n * rows, 1, D, generator=torch.Generator().manual_seed(n)).to(dtype).to(DEV)
    seqs = np.random.RandomState(n).permutation(n).tolist()
    plan = bd.chunk_plan(cache, i32(seqs), i32(counts), rows=n * rows, heads=1, window=window, sinks=sinks)
    o, lse = bd.chunk_attn(plan, q, 0)
    torch.cuda.synchronize()
    items, joins = check_plan(plan, lens, seqs, counts, 1, dtype == F32, 1, window, sinks)
    rec = items_of(plan)[3]
    cut = {int(x[1]) // rows for x in rec if x[11] >= 0}  # requests with tiles in parts
    long = {r for r, s in enumerate(seqs) if lens[s] >= 4000}
    assert len({(int(x[1]), int(x[4])) for x in rec}) == tiles and long <= cut and items > tiles and joins > 0
    tile_of = {int(t): i for i, t in enumerate(sorted({int(x[1]) * 1024 + int(x[4]) for x in rec}))}
    assert len({tile_of[r * rows * 1024] // 512 for r in cut}) > 1  # in several rounds
    some = sorted(long | set(range(0, n, 97)) | {n - 1})
    pick = torch.cat([torch.arange(r * rows, (r + 1) * rows) for r in some]).to(DEV)
    ro, rl, _ = oracle(cache, [seqs[r] for r in some], [rows] * len(some), q[pick], 0, None, 1, window, sinks)
    check("o", o[pick], *ro)
    check("lse", lse[:, pick], *rl)
    assert not bool(o.isnan().any()) and bool((lse > -math.inf).all())
