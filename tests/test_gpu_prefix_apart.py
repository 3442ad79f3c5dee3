"""Attention over the cache where the prefix is read once for all requests, through the first one's table: another first
sequence, repeated ones, layers, graphs, requests inside the prefix; and tables far longer than their sequences.

That the prefix really is read through the first request's table shows when the other sequences' entries for its full
pages are taken away: the results stay the same bits."""
import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import check
from tests.test_gpu_prefix import build, i32, oracle

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# dtype, prefix, rows, heads, KV heads, head_dim, page size, block
APART = [(BF, 2003, 1, 16, 4, 128, 16, False), (BF, 2003, 1, 8, 4, 128, 24, False), (BF, 2048, 1, 8, 8, 64, 64, False),
         (BF, 2003, 5, 16, 4, 128, 16, True), (BF, 2500, 3, 8, 4, 128, 100, False), (F32, 2003, 1, 8, 4, 64, 16, False),
         (F32, 2111, 2, 4, 4, 64, 24, True)]
LENS = [50, 3, 0, -700, 333]  # beyond the prefix
SEQS = [2, 0, 3, 3, 1, 2, 4]


def attend(c, q, layer, seqs, prefix, block):
    o, lse = bd.prefix_attn(q, c, layer, i32(seqs), prefix, block=block)
    torch.cuda.synchronize()
    return o, lse


def only_the_first_holds_it(c, seqs, prefix):
    """The cache with no entry for the prefix's full pages but the first request's."""
    table = c.table.clone()
    for s in range(c.seqs):
        if s != seqs[0]:
            table[s, :prefix // c.page_size] = -1
    return bd.Cache(c.k, c.v, table, c.lens, c.refs, c.status)


@pytest.mark.parametrize("dtype,prefix,n,H,KV,D,ps,block", APART)
def test_another_first_sequence_and_repeated_ones(dtype, prefix, n, H, KV, D, ps, block):
    c = build([prefix + x for x in LENS], prefix, ps, KV, D, dtype, 81, layers=3)
    q = synth.normal((len(SEQS), n, H, D), 82, dtype).cuda()
    for layer in (2, 0):
        o, lse = attend(c, q, layer, SEQS, prefix, block)
        ref = oracle(q, c, layer, SEQS, block)
        check("o", o, *ref["o"])
        check("lse", lse, *ref["lse"])
        o1, lse1 = attend(only_the_first_holds_it(c, SEQS, prefix), q, layer, SEQS, prefix, block)
        assert torch.equal(o, o1) and torch.equal(lse, lse1)
        o0, lse0 = attend(c, q, layer, SEQS, 0, block)  # the same attention, each request through its own table
        check("o", o0, *ref["o"])
        check("lse", lse0, *ref["lse"])


@pytest.mark.parametrize("dtype,prefix,n,H,KV,D,ps,block", [APART[0], APART[3], APART[5]])
def test_graph_replays_follow_lengths_and_lists(dtype, prefix, n, H, KV, D, ps, block):
    c = build([prefix + 300] * 5, prefix, ps, KV, D, dtype, 83)
    for x in (c.k, c.v):
        x.nan_to_num_(0.5)
    q, seqs = synth.normal((len(SEQS), n, H, D), 84, dtype).cuda(), i32(SEQS)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        bd.prefix_attn(q, c, 0, seqs, prefix, block=block)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, lse = bd.prefix_attn(q, c, 0, seqs, prefix, block=block)
    for i in range(3):
        c.lens.copy_(torch.tensor([prefix + 10 + i, prefix + 290 - 90 * i, prefix + i, 40 * i, prefix + 1], dtype=torch.int32))
        now = SEQS[i:] + SEQS[:i]
        now = [2] + [x for x in now if x != 2][:5] + [2]
        seqs.copy_(torch.tensor(now, dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        e, el = attend(c, q, 0, now, prefix, block)
        assert torch.equal(o, e) and torch.equal(lse, el)
        check("o", o, *oracle(q, c, 0, now, block)["o"])


@pytest.mark.parametrize("dtype,n,H,KV,D,ps,block", [
    (BF, 1, 16, 4, 128, 16, False), (BF, 1, 4, 4, 64, 24, False), (BF, 40, 8, 2, 128, 16, True), (BF, 70, 4, 2, 64, 64, False),
    (F32, 1, 8, 2, 64, 16, False), (F32, 3, 4, 2, 128, 24, False)])
@pytest.mark.parametrize("tokens", [20_000, 1_000_000])
def test_tables_far_longer_than_their_sequences(dtype, n, H, KV, D, ps, block, tokens):
    """Up to some thousand chunks of keys, nearly all of them empty."""
    lens = [900, 0, 5, 1300, 64]
    c = build(lens, 0, ps, KV, D, dtype, 85, spare=tokens // ps)
    q = synth.normal((len(lens), n, H, D), 86, dtype).cuda()
    assert bd.prefix_attn_workspace_bytes(q, c) < 6 << 30
    o, lse = attend(c, q, 0, range(len(lens)), 0, block)
    ref = oracle(q, c, 0, range(len(lens)), block)
    check("o", o, *ref["o"])
    check("lse", lse, *ref["lse"])
