"""A sequence in different batches: alone, or beside others whose load has its walks cut or its tiles taken by two teams.
The order of sums may differ, so bits may; each result stays within the error bound."""
import pytest
import torch

import paper_2609_19242_amd as bd
import synth
from tests.serving_util import check, packed

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,KV,D", [(8, 2, 128), (6, 2, 64)])
def test_one_sequence_in_several_batches(H, KV, D, dtype):
    n, m = 130, 1700  # rows and keys of the sequence
    mine = [synth.normal((r, h, D), 91 + i, dtype) for i, (r, h) in enumerate(((n, H), (m, KV), (m, KV), (n, H)))]
    q, k, v, do = mine
    ref = packed(q, k, v, [(0, n, 0, m)], do=do)
    seen = set()
    for before, behind in (([], []), ([(700, 700)], [(1, 900)]), ([(60, 60)] * 40, [(2200, 2200)]),
                           ([(300, 1500)] * 40, []), ([(1800, 1800)] * 6, [(7, 7)])):
        qs, ks = sum(a for a, _ in before), sum(b for _, b in before)
        ql, kl = (list(x) for x in zip(*(before + [(n, m)] + behind)))
        args = [synth.normal((sum(x), t.shape[1], D), 95 + i, dtype) for i, (x, t) in enumerate(zip((ql, kl, kl, ql), mine))]
        for t, x, at in zip(args, mine, (qs, ks, ks, qs)):
            t[at:at + x.shape[0]] = x
        dev = [t.to(DEV) for t in args]
        plan = bd.packed_plan(ql, kl, heads=H, kv_heads=KV, head_dim=D, dtype=dtype)
        seen.add((plan._record.teams, plan._record.fwd.items > 0, plan._record.dq.items > 0, plan._record.n_sums > 0))
        o, lse = bd.packed_fwd(plan, *dev[:3])
        dq, dk, dv = bd.packed_bwd(plan, *dev[:3], o, lse, dev[3])
        torch.cuda.synchronize()
        for name, t, at, r in (("o", o, qs, n), ("dq", dq, qs, n), ("dk", dk, ks, m), ("dv", dv, ks, m)):
            check(name, t[at:at + r], *ref[name])
        check("lse", lse[:, qs:qs + n], *ref["lse"])
    assert dtype == torch.float32 or len(seen) >= 3  # the batches were planned in different ways
