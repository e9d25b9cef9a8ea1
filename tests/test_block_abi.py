"""Refusals of the uniform 8-bit cache's operators and of the norms with rotation (CPU only; no call here reaches a
kernel)."""
import ctypes as C
import math
import os

import pytest
import torch

FAKE = 0x10000


@pytest.fixture(scope="module")
def dk():
    from paper_2412_03131_amd import diffkv
    if not os.path.exists(diffkv.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    diffkv.lib()
    return diffkv


def _cache(dk, a):
    return C.byref(dk.BlockCacheStruct(a["pool"], a["scale"], a["blocks"], a["table"], a["tail"], a["seq_len"], a["status"],
                                       a["seqs"], a["Hkv"], a["fmt"]))


def _args(dk, c):
    a = dict(L=dk.layout(max_seq_len=256), pool=FAKE, scale=FAKE, blocks=16, table=FAKE, tail=FAKE, seq_len=FAKE,
             status=FAKE, seqs=2, Hkv=2, fmt=0, total=10, max_new=6, new_len=FAKE, start=FAKE, Hq=8, q=FAKE, qs=8 * 128, k=FAKE,
             ks=2 * 128, v=FAKE, vs=2 * 128, sm=0.1, form=None, sinks=0, out=FAKE, lse=None, ws=FAKE, ws_bytes=0)
    a.update(c)
    return a


def append(dk, **c):
    a = _args(dk, c)
    return dk.lib().diffkv_block_append(C.byref(a["L"]), _cache(dk, a), a["total"], a["max_new"], a["new_len"], a["k"],
                                        a["ks"], a["v"], a["vs"], None)


def read(dk, **c):
    a = _args(dk, c)
    return dk.lib().diffkv_block_read(C.byref(a["L"]), _cache(dk, a), a["total"], a["max_new"], a["start"], a["new_len"],
                                      a["k"], a["ks"], a["v"], a["vs"], None)


def attention(dk, **c):
    """With valid arguments DIFFKV_E_WORKSPACE: none is given."""
    a = _args(dk, c)
    return dk.lib().diffkv_block_attention(
        C.byref(a["L"]), _cache(dk, a), a["total"], a["max_new"], a["new_len"], a["Hq"], a["q"], a["qs"], a["k"], a["ks"],
        a["v"], a["vs"], a["sm"], a["form"], a["sinks"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


SHARED = [dict(pool=0), dict(scale=0), dict(table=0), dict(tail=0), dict(seq_len=0), dict(status=0), dict(pool=FAKE + 8),
          dict(tail=FAKE + 2), dict(blocks=-1), dict(blocks=1 << 31), dict(fmt=2), dict(fmt=-1), dict(seqs=-1), dict(Hkv=0),
          dict(total=-1), dict(max_new=-1), dict(new_len=None), dict(k=None), dict(v=None), dict(k=FAKE + 2),
          dict(v=FAKE + 8), dict(ks=2 * 128 - 8), dict(vs=2 * 128 + 4), dict(ks=-1024)]


@pytest.mark.parametrize("bad", SHARED, ids=str)
def test_refused_arguments(dk, bad):
    for f in (append, read, attention):
        assert f(dk, **bad) == dk.E_INVAL


def test_refused_by_one(dk):
    assert read(dk, start=None) == dk.E_INVAL
    for bad in (dict(q=None), dict(q=FAKE + 8), dict(qs=8 * 128 - 8), dict(qs=4), dict(out=None), dict(out=FAKE + 2),
                dict(Hq=7), dict(Hq=0), dict(Hq=-8), dict(sinks=-1), dict(sm=0.0), dict(sm=-1.0), dict(sm=math.nan),
                dict(sm=math.inf), dict(sm=65537.0)):
        assert attention(dk, **bad) == dk.E_INVAL
    for cap, window in ((-1.0, 0), (math.nan, 0), (math.inf, 0), (0.0, -1), (1e-35, 0)):
        assert attention(dk, form=C.byref(dk.ScoreForm(cap, window, None))) == dk.E_INVAL
    need = dk.workspace_size(dk.OP_BLOCK_ATTENTION, dk.layout(), 2, 8, 2, 10)
    assert attention(dk, ws=FAKE + 8, ws_bytes=need) == dk.E_INVAL
    assert attention(dk, ws=None, ws_bytes=need) == dk.E_WORKSPACE


def test_not_implemented(dk):
    for f in (append, read, attention):
        assert f(dk, L=dk.layout(head_dim=64)) == dk.E_UNSUPPORTED
        assert f(dk, L=dk.layout(max_seq_len=(1 << 30) + 1)) == dk.E_UNSUPPORTED
        assert f(dk, total=(1 << 24) + 1) == dk.E_UNSUPPORTED
        assert f(dk, seqs=(1 << 21) + 1) == dk.E_UNSUPPORTED
    assert attention(dk, Hq=130, qs=130 * 128) == dk.E_UNSUPPORTED
    assert attention(dk, Hq=128, qs=128 * 128) == dk.E_WORKSPACE
    assert attention(dk, total=(1 << 23) + 1) == dk.E_UNSUPPORTED  # (its units of work would pass 64 bits)
    assert attention(dk, total=1 << 23) == dk.E_WORKSPACE


def test_nothing_to_do(dk):
    for none in (dict(seqs=0), dict(total=0), dict(max_new=0)):
        none = dict(none, q=None, k=None, v=None, new_len=None, start=None, out=None, ws=None)
        for f in (append, read, attention):
            assert f(dk, **none) == dk.OK
    assert attention(dk, blocks=0, pool=0, scale=0) == dk.E_WORKSPACE  # (a cache of tails alone)


@pytest.mark.parametrize("stride", [-1, 0, 3, 1 << 40])
def test_a_single_row_has_any_stride(dk, stride):
    assert attention(dk, total=1, max_new=1, qs=stride, ks=stride, vs=stride) == dk.E_WORKSPACE


def test_workspace(dk):
    L = dk.layout(max_seq_len=8192)
    for G, Hkv in ((1, 1), (4, 8), (8, 8), (64, 2)):
        need = [dk.workspace_size(dk.OP_BLOCK_ATTENTION, L, 64, G * Hkv, Hkv, rows) for rows in (0, 1, 64, 500, 4000, 1 << 23)]
        assert need == sorted(need) and need[-1] < 192 << 20  # (one for more rows serves fewer)
        for seqs in (1, 1000):
            assert dk.workspace_size(dk.OP_BLOCK_ATTENTION, L, seqs, G * Hkv, Hkv, 500) == need[3]
    for bad in ((0, 1, 1), (4, 0, 1), (4, 8, 1), (8, 2, -1), (8, 2, (1 << 23) + 1)):
        with pytest.raises(dk.DiffKVError) as e:
            dk.workspace_size(dk.OP_BLOCK_ATTENTION, L, 1, *bad)
        assert e.value.code == dk.E_INVAL


def test_binding_checks_its_tensors(dk):
    L = dk.layout(max_seq_len=256)
    c = dk.BlockCache(L, 16, 2, 2, device="cpu")
    assert c.table.shape == (2, 8) and c.pool.shape == (16, 2, 2, 4096)
    q, kv = torch.zeros((3, 8, 128), dtype=torch.float16), torch.zeros((3, 2, 128), dtype=torch.float16)
    nl, ws = torch.tensor([2, 1], dtype=torch.int32), torch.zeros(1 << 26, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        dk.block_append(c, nl, kv, kv, max_new=2)
    with pytest.raises(ValueError, match="GPU"):
        dk.block_read(c, nl, nl, 3, max_count=2)
    with pytest.raises(ValueError, match="GPU"):
        dk.block_attention(c, nl, q, kv, kv, 0.1, max_new=2, ws=ws)
    freq, _ = dk.rope_frequencies(128)
    with pytest.raises(ValueError, match="GPU"):
        dk.norm_rotate(L, torch.zeros(3, dtype=torch.int32), freq, q, kv)
    with pytest.raises(ValueError):
        dk.norm_rotate(L, torch.zeros(3, dtype=torch.int32), freq, q, kv, q_weight=torch.ones(64))
    for bad in (nl.long(), nl[:1], torch.zeros(4, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="lengths"):
            dk.block_append(c, bad, kv, kv, max_new=2)
    with pytest.raises(ValueError):
        dk.block_append(c, nl, kv, kv[:2], max_new=2)
    with pytest.raises(ValueError):
        dk.block_append(c, nl, kv[:, :1], kv[:, :1], max_new=2)
    with pytest.raises(ValueError):
        dk.block_attention(c, nl, q[:2], kv, kv, 0.1, max_new=2, ws=ws)
    with pytest.raises(ValueError):
        dk.block_read(c, nl, nl, 3, max_count=2, k_out=kv[:2], v_out=kv)
    t = list(c.tensors())
    for i, bad in ((0, t[0][:8]), (0, t[0].int()), (1, t[1][:8]), (2, t[2][:, :4]), (3, t[3].float()), (4, t[4].long()),
                   (5, t[5].long())):
        with pytest.raises(ValueError):
            dk.BlockCache(L, 16, 2, 2, buffers=t[:i] + [bad] + t[i + 1:])
    c.seq_len += 3  # (in place: the same tensor)
    assert c.seq_len.tolist() == [3, 3] and c.seq_len is t[4]
    with pytest.raises(AttributeError):
        c.seq_len = torch.zeros(2, dtype=torch.int32)


def norm_rotate(dk, **c):
    a = dict(L=dk.layout(), rows=5, pos=FAKE, freq=FAKE, rot=64, style=0, scale=1.0, eps=1e-6, Hq=4, q=FAKE, qs=512, qw=FAKE,
             qo=FAKE, qos=512, Hkv=1, k=FAKE, ks=128, kw=FAKE, ko=FAKE, kos=128)
    a.update(c)
    return dk.lib().diffkv_norm_rotate(C.byref(a["L"]), a["rows"], a["pos"], a["freq"], a["rot"], a["style"], a["scale"],
                                       a["eps"], a["Hq"], a["q"], a["qs"], a["qw"], a["qo"], a["qos"], a["Hkv"], a["k"],
                                       a["ks"], a["kw"], a["ko"], a["kos"], None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(pos=None), dict(freq=None), dict(freq=FAKE + 4), dict(rot=0),
                                 dict(rot=33), dict(rot=144), dict(style=2), dict(Hq=0), dict(Hkv=-1), dict(Hkv=0),
                                 dict(k=None), dict(ko=None), dict(q=None), dict(qo=None), dict(q=FAKE + 2),
                                 dict(qs=504), dict(qs=516), dict(kos=64), dict(qos=1024), dict(kos=256), dict(eps=0.0),
                                 dict(eps=-1e-6), dict(eps=1e-39), dict(eps=math.nan), dict(eps=math.inf), dict(qw=FAKE + 4), dict(kw=FAKE + 8)],
                         ids=str)
def test_refused_norms(dk, bad):
    assert norm_rotate(dk, **bad) == dk.E_INVAL


def test_norms_not_implemented(dk):
    assert norm_rotate(dk, rot=40) == dk.E_UNSUPPORTED
    assert norm_rotate(dk, L=dk.layout(head_dim=64)) == dk.E_UNSUPPORTED
    assert norm_rotate(dk, rows=0) == dk.OK
