"""Refusals of attention of chunks of new tokens over a cache, by the binding and by the C ABI; the room that is made for
plans.  Host only: every call here fails before anything is launched."""
import ctypes
import math

import pytest
import torch

import paper_2609_19242_amd as bd
from paper_2609_19242_amd import cache as cm
from paper_2609_19242_amd import chunk as km
from paper_2609_19242_amd import packed as pm

BF, F32 = torch.bfloat16, torch.float32
FAKE = 0x10000  # never dereferenced: these calls fail validation first
host_only = pytest.mark.skipif(torch.cuda.device_count() > 0,
                               reason="passes unmapped pointers that validation must reject; host-only test")


def cache(**kw):
    return bd.cache_new(**dict(dict(layers=2, pages=6, page_size=16, kv_heads=2, head_dim=64, seqs=3, max_pages=4, dtype=BF,
                                    device="cpu"), **kw))


def i32(*xs):
    return torch.tensor(xs, dtype=torch.int32)


def planned(monkeypatch, **kw):
    """A plan of a cache on the CPU, with nothing launched."""
    monkeypatch.setattr(km, "_launch", lambda *a: None)
    return bd.chunk_plan(cache(), i32(0, 1), i32(3, 1), rows=6, heads=4, **kw)


@pytest.mark.parametrize("change,err,what", [
    (dict(cache=None), TypeError, "Cache"), (dict(seqs=[0]), TypeError, "seqs"), (dict(seqs=torch.tensor([0, 1])), TypeError, "int32"),
    (dict(counts=i32(1)), ValueError, "counts"), (dict(counts=i32(1, 2, 3, 4)[::2]), ValueError, "contiguous"),
    (dict(rows=1.5), TypeError, "float"), (dict(rows=1 << 70), ValueError, "rows"), (dict(heads=1 << 40), ValueError, "heads"),
    (dict(window=1 << 70), ValueError, "window"), (dict(sinks=1 << 40), ValueError, "sinks"), (dict(block_size=1 << 70), ValueError, "block_size"),
    (dict(scale=math.nan), ValueError, "scale"), (dict(out=3), TypeError, "ChunkPlan")])
def test_plans_refuse(change, err, what):
    args = dict(dict(cache=cache(), seqs=i32(0, 1), counts=i32(3, 1), rows=6, heads=4), **change)
    with pytest.raises(err, match=what):
        bd.chunk_plan(**args)


def test_plans_need_a_gpu():
    with pytest.raises(ValueError, match="GPU"):
        bd.chunk_plan(cache(), i32(0, 1), i32(3, 1), rows=6, heads=4)


def test_plans_are_used_again_for_the_same_sizes(monkeypatch):
    p = planned(monkeypatch)
    assert p.starts.shape == (2,) and p.requests == 2 and p.rows == 6
    again = bd.chunk_plan(p.cache, i32(1, 2), i32(1, 1), rows=6, heads=4, window=8, out=p)
    assert again is p and p._record.window == 8
    # room for a plan does not depend on its window, room for the calls does
    far = cache(max_pages=64)
    p2 = bd.chunk_plan(far, i32(0, 1), i32(3, 1), rows=6, heads=4, window=8)
    assert p2.workspace_bytes == 0
    bd.chunk_plan(far, i32(0, 1), i32(3, 1), rows=6, heads=4, out=p2)
    assert p2.workspace_bytes > 0 and p2._bytes >= bd.lib().bdlm_chunk_plan_bytes(far._ref, p2._ref)
    for kw in (dict(cache=cache()), dict(seqs=i32(0), counts=i32(1)), dict(rows=7), dict(heads=2)):
        with pytest.raises(ValueError, match="same"):
            bd.chunk_plan(**dict(dict(cache=p.cache, seqs=i32(0, 1), counts=i32(3, 1), rows=6, heads=4, out=p), **kw))


def test_attention_refuses_tensors(monkeypatch):
    p = planned(monkeypatch)
    q, lse = torch.zeros(6, 4, 64, dtype=BF), torch.zeros(4, 6)
    o, z = bd.chunk_attn(p, q, 0)
    assert o.shape == q.shape and z.shape == (4, 6) and z.dtype == F32
    for bad, err in ((q.float(), TypeError), (q[:5], ValueError), (torch.zeros(7, 4, 64, dtype=BF), ValueError), (q[:, :2], ValueError),
                     (q[..., :32], ValueError), (q.transpose(0, 1), ValueError), (None, TypeError)):
        with pytest.raises(err):
            bd.chunk_attn(p, bad, 0)
    with pytest.raises(TypeError, match="plan"):
        bd.chunk_attn(None, q, 0)
    with pytest.raises(TypeError, match="plan"):
        bd.chunk_attn_workspace_bytes(None)
    for out, err in (((q,), ValueError), ((q.float(), lse), TypeError), ((q, lse.t()), ValueError), ((q, lse.double()), TypeError),
                     ((q[:5], lse), ValueError)):
        with pytest.raises(err):
            bd.chunk_attn(p, q, 0, out=out)
    with pytest.raises(ValueError, match="workspace"):
        bd.chunk_attn(p, q, 0, workspace=torch.zeros(8, 8)[:, ::2])
    with pytest.raises(TypeError):
        bd.chunk_attn(p, q, 0.5)


def crec(**kw):
    r = cm._Cache(*[FAKE] * 7, 2, 6, 16, 3, 4, 2, 64, bd.BF16, 0)
    for n, x in kw.items():
        setattr(r, n, x)
    return r


def krec(**kw):
    return km._Chunk(**dict(dict(requests=2, rows=6, block_size=1, window=0, heads=4, sinks=0, scale=0.0, reserved=0), **kw))


def make_plan(c=None, k=None, seqs=FAKE, counts=FAKE, plan=FAKE, nb=1 << 30):
    return bd.lib().bdlm_chunk_plan(ctypes.byref(c or crec()), ctypes.byref(k or krec()), seqs, counts, plan, nb, None)


def attend(c=None, k=None, **kw):
    x = dict(dict(layer=0, plan=FAKE, nb=1 << 30, q=FAKE, qs=256, o=FAKE, os=256, lse=FAKE, pitch=6, fill=0, ws=FAKE, wb=1 << 30), **kw)
    return bd.lib().bdlm_chunk_attn(ctypes.byref(c or crec()), ctypes.byref(k or krec()), x["layer"], x["plan"], x["nb"],
                                    pm._Rows(x["q"], x["qs"]), pm._Rows(x["o"], x["os"]), x["lse"], x["pitch"], x["fill"], x["ws"],
                                    x["wb"], None)


@host_only
@pytest.mark.parametrize("kw,status", [
    (dict(requests=-1), -1), (dict(requests=(1 << 19) + 1), -1), (dict(rows=-1), -1), (dict(rows=1 << 24), -2), (dict(rows=1 << 60), -2),
    (dict(block_size=0), -1), (dict(block_size=1 << 40), -1), (dict(window=-1), -1), (dict(window=1 << 40), -1), (dict(heads=0), -1),
    (dict(heads=3), -1), (dict(sinks=-1), -1), (dict(sinks=1 << 29), -1), (dict(scale=math.nan), -1), (dict(scale=math.inf), -1),
    (dict(reserved=1), -1)])
def test_the_c_abi_refuses_chunks(kw, status):
    k = krec(**kw)
    assert make_plan(k=k) == status and attend(k=k) == status
    c = ctypes.byref(crec())
    assert bd.lib().bdlm_chunk_plan_bytes(c, ctypes.byref(k)) == 0 == bd.lib().bdlm_chunk_workspace_bytes(c, ctypes.byref(k))
    assert bd.lib().bdlm_last_error()


@host_only
@pytest.mark.parametrize("kw,status", [(dict(k=0), -1), (dict(head_dim=32), -2), (dict(seqs=0), -1), (dict(table=0), -1), (dict(pages=0), -1),
                                       (dict(pages=(1 << 28) + 1, page_size=64), -2)])
def test_the_c_abi_refuses_caches(kw, status):
    assert make_plan(crec(**kw)) == status and attend(crec(**kw)) == status
    assert bd.lib().bdlm_chunk_plan_bytes(ctypes.byref(crec(**kw)), ctypes.byref(krec())) == 0


@host_only
def test_the_c_abi_refuses_pointers_and_room():
    L, c, k = bd.lib(), crec(), krec()
    need = L.bdlm_chunk_plan_bytes(ctypes.byref(c), ctypes.byref(k))
    assert need > 0
    for kw in (dict(seqs=0), dict(seqs=FAKE + 2), dict(counts=0), dict(counts=FAKE + 2), dict(plan=0), dict(plan=FAKE + 8), dict(nb=need - 1)):
        assert make_plan(**kw) == -1, kw
    for kw in (dict(layer=-1), dict(layer=2), dict(plan=0), dict(plan=FAKE + 8), dict(nb=need - 1), dict(q=0), dict(q=FAKE + 8), dict(qs=255),
               dict(qs=260), dict(o=0), dict(os=128), dict(os=1 << 31), dict(lse=0), dict(lse=FAKE + 2), dict(pitch=5), dict(pitch=1 << 40),
               dict(fill=2)):
        assert attend(**kw) == -1, kw
    # (walks that no table or window lets grow past 512 keys are never cut)
    assert L.bdlm_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(k)) == 0
    far = crec(max_pages=64)
    assert L.bdlm_chunk_workspace_bytes(ctypes.byref(far), ctypes.byref(krec(window=60, sinks=4))) == 0
    need = L.bdlm_chunk_workspace_bytes(ctypes.byref(far), ctypes.byref(k))
    assert need > 0
    for kw in (dict(ws=0), dict(ws=FAKE + 128), dict(wb=need - 1)):
        assert attend(far, **kw) == -4, kw
    assert attend(k=krec(rows=0), q=0, o=0, lse=0) == 0  # nothing to do, nothing launched
    assert L.bdlm_chunk_plan(None, ctypes.byref(k), FAKE, FAKE, FAKE, 1 << 30, None) == -1
    assert L.bdlm_chunk_plan(ctypes.byref(c), None, FAKE, FAKE, FAKE, 1 << 30, None) == -1


def test_workspaces_do_not_grow_with_the_tables():
    def room(**kw):
        c, k = crec(**kw), krec(rows=512, requests=64, heads=32)
        c.kv_heads, c.head_dim = 8, 128
        return bd.lib().bdlm_chunk_workspace_bytes(ctypes.byref(c), ctypes.byref(k))

    short, far = room(max_pages=64), room(max_pages=8192)
    assert short <= far == room(max_pages=4096) and far < 256 << 20
    # (tables of a million tokens: more chunks than that may be needed where every request has so many)
    assert room(max_pages=65536) >= far


def test_new_tensors_of_a_given_stream(monkeypatch):
    """They come from that stream's memory, and results are kept for the current one too."""
    import contextlib
    at, new, kept = ["current"], [], []

    @contextlib.contextmanager
    def stream(s):
        at.append(s)
        yield
        at.pop()

    for owner, name in ((torch, "empty"), (torch.Tensor, "new_empty")):
        plain = getattr(owner, name)
        monkeypatch.setattr(owner, name, lambda *a, plain=plain, **kw: new.append((plain(*a, **kw), at[-1])) or new[-1][0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept.append((t, s)))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: at[-1])
    monkeypatch.setattr(bd, "_torch_stream", lambda s, device: s)
    monkeypatch.setattr(km, "_launch", lambda *a: None)
    c = cache(max_pages=64)  # (walks that may be cut: with a workspace)
    new.clear()
    p = bd.chunk_plan(c, i32(0, 1), i32(3, 1), rows=6, heads=4, stream="side")
    assert len(new) == 1 and new[0][1] == "side" and any(t is p._items and s == "current" for t, s in kept)
    new.clear()
    res = bd.chunk_attn(p, torch.zeros(6, 4, 64, dtype=BF), 0, stream="side")
    assert len(new) == 4 - 1 and all(s == "side" for _, s in new)  # o, lse and the workspace
    assert all(any(r is t and s == "current" for t, s in kept) for r in res)
