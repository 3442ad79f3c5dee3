"""Numbers that do not fit the C ABI's integers are refused, not cut to their low bits.  Host only."""
import pytest
import torch

import paper_2609_19242_amd as bd

BF = torch.bfloat16


@pytest.mark.parametrize("kw", [
    dict(heads=(1 << 32) + 4), dict(kv_heads=(1 << 32) + 2), dict(head_dim=(1 << 32) + 64), dict(block_size=(1 << 64) + 1),
    dict(window=1 << 64), dict(ql=[(1 << 64) + 5]), dict(ql=[5], kl=[(1 << 64) + 5]), dict(ql=[5], q_starts=[1 << 64]),
    dict(ql=[5], k_starts=[1 << 64]), dict(window=-(1 << 64))])
def test_plans(kw):
    kw = dict(dict(ql=[5, 3], kl=None, heads=4, kv_heads=2, head_dim=64, dtype=BF, device="cpu"), **kw)
    with pytest.raises((ValueError, bd.BdlmError)):
        bd.packed_plan(kw.pop("ql"), kw.pop("kl"), **kw)


@pytest.mark.parametrize("layer,prefix", [(1 << 64, 0), (0, 1 << 64), (0, -(1 << 64)), ((1 << 64) + 1, 16)])
def test_attention_over_the_cache(layer, prefix, monkeypatch):
    c = bd.cache_new(2, 6, 16, 2, 64, 3, 4, BF, "cpu")
    q, seqs = torch.zeros(2, 1, 4, 64, dtype=BF), torch.zeros(2, dtype=torch.int32)
    monkeypatch.setattr(bd.cache, "_launch", lambda *a: None)
    with pytest.raises(ValueError, match="layer|prefix"):
        bd.prefix_attn(q, c, layer, seqs, prefix)
    if layer == 0:
        with pytest.raises(ValueError, match="prefix"):
            bd.prefix_attn_workspace_bytes(q, c, prefix)
    else:
        k = torch.zeros(4, 2, 64, dtype=BF)
        with pytest.raises(ValueError, match="layer"):
            bd.cache_write(c, layer, seqs[:1], seqs[:1], k, k)
