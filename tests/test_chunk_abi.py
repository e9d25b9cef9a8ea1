"""Refusals of the chunk operators and the frequency tables of rotary positions (CPU only; no call
here reaches a kernel)."""
import ctypes as C
import math
import os

import numpy as np
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


def attention(dk, **c):
    """diffkv_chunk_attention with valid arguments but those given."""
    a = dict(L=dk.layout(max_seq_len=256), pool=FAKE, seq_len=FAKE, seqs=2, Hkv=2, total=10, max_new=6, new_len=FAKE,
             Hq=8, q=FAKE, qs=8 * 128, k=FAKE, ks=2 * 128, v=FAKE, vs=2 * 128, scale=0.1, form=None, out=FAKE,
             lse=None, ws=FAKE, ws_bytes=0)
    a.update(c)
    st = dk.CacheStruct(a["pool"], 16, FAKE, FAKE, FAKE, a["seq_len"], FAKE, FAKE, FAKE, a["seqs"], a["Hkv"])
    return dk.lib().diffkv_chunk_attention(
        C.byref(a["L"]), C.byref(st), a["total"], a["max_new"], a["new_len"], a["Hq"], a["q"], a["qs"], a["k"], a["ks"],
        a["v"], a["vs"], a["scale"], a["form"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


def significance(dk, **c):
    a = dict(L=dk.layout(max_seq_len=256), pool=FAKE, seq_len=FAKE, seqs=2, Hkv=2, total=10, max_new=6, new_len=FAKE,
             Hq=8, q=FAKE, qs=8 * 128, k=FAKE, ks=2 * 128, scale=0.1, form=None, lse=FAKE, score=FAKE)
    a.update(c)
    st = dk.CacheStruct(a["pool"], 16, FAKE, FAKE, FAKE, a["seq_len"], FAKE, FAKE, FAKE, a["seqs"], a["Hkv"])
    return dk.lib().diffkv_chunk_significance(
        C.byref(a["L"]), C.byref(st), a["total"], a["max_new"], a["new_len"], a["Hq"], a["q"], a["qs"], a["k"], a["ks"],
        a["scale"], a["form"], a["lse"], a["score"], FAKE, 0, None)


SHARED = [dict(pool=0), dict(seq_len=0), dict(total=-1), dict(max_new=-1), dict(total=1 << 30), dict(Hq=7), dict(Hq=0),
          dict(new_len=None), dict(q=None), dict(k=None), dict(q=FAKE + 8), dict(k=FAKE + 2), dict(qs=8 * 128 - 8),
          dict(ks=2 * 128 + 4), dict(qs=-1024), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
          dict(scale=math.inf)]


@pytest.mark.parametrize("bad", SHARED, ids=str)
def test_refused_arguments(dk, bad):
    assert attention(dk, **bad) == dk.E_INVAL
    assert significance(dk, **bad) == dk.E_INVAL


@pytest.mark.parametrize("form", [(-1.0, 0), (math.nan, 0), (math.inf, 0), (0.0, -1), (1e-35, 0)], ids=str)
def test_refused_forms(dk, form):
    f = C.byref(dk.ScoreForm(form[0], form[1], None))
    assert attention(dk, form=f) == dk.E_INVAL
    assert significance(dk, form=f) == dk.E_INVAL


def test_refused_by_one(dk):
    for bad in (dict(v=None), dict(v=FAKE + 4), dict(vs=128), dict(out=None), dict(out=FAKE + 2)):
        assert attention(dk, **bad) == dk.E_INVAL
    for bad in (dict(lse=None), dict(score=None)):
        assert significance(dk, **bad) == dk.E_INVAL


def test_unsupported_layouts_and_group_sizes(dk):
    L = dk.layout(tokens_per_page=(16, 64), max_seq_len=64)
    for f in (attention, significance):
        assert f(dk, L=L) == dk.E_UNSUPPORTED
        assert f(dk, Hq=18, qs=18 * 128) == dk.E_UNSUPPORTED
        assert f(dk, L=dk.layout(head_dim=64), Hq=8) == dk.E_UNSUPPORTED


def test_nothing_to_do(dk):
    for none in (dict(seqs=0), dict(total=0), dict(max_new=0)):
        none = dict(none, q=None, k=None, new_len=None)
        assert attention(dk, v=None, out=None, ws=None, **none) == dk.OK
        assert significance(dk, lse=None, score=None, **none) == dk.OK


def test_workspace(dk):
    L = dk.layout(max_seq_len=8192)
    for seqs, Hq, Hkv, rows in ((1, 32, 8, 1), (64, 32, 8, 64), (8, 64, 8, 4000), (1, 8, 8, 1), (24, 28, 4, 100)):
        need = dk.workspace_size(dk.OP_CHUNK_ATTENTION, L, seqs, Hq, Hkv, rows)
        assert need < 144 << 20
        assert attention(dk, L=L, seqs=seqs, Hq=Hq, Hkv=Hkv, total=rows, max_new=1, qs=Hq * 128, ks=Hkv * 128,
                         vs=Hkv * 128, ws_bytes=need - 1) == (dk.E_WORKSPACE if need else dk.E_INVAL) or need == 0
    for op in (dk.OP_CHUNK_ATTENTION, dk.OP_CHUNK_SIGNIFICANCE):
        with pytest.raises(dk.DiffKVError):
            dk.workspace_size(op, L, 1, 0, 1, 1)
        with pytest.raises(dk.DiffKVError):
            dk.workspace_size(op, L, 1, 4, 0, 1)


def rotate(dk, **c):
    a = dict(L=dk.layout(), rows=5, pos=FAKE, freq=FAKE, rot=64, style=0, scale=1.0, Hq=4, q=FAKE, qs=512, qo=FAKE,
             qos=512, Hkv=1, k=FAKE, ks=128, ko=FAKE, kos=128)
    a.update(c)
    return dk.lib().diffkv_rotate(C.byref(a["L"]), a["rows"], a["pos"], a["freq"], a["rot"], a["style"], a["scale"],
                                  a["Hq"], a["q"], a["qs"], a["qo"], a["qos"], a["Hkv"], a["k"], a["ks"], a["ko"],
                                  a["kos"], None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(pos=None), dict(freq=None), dict(freq=FAKE + 4), dict(rot=0),
                                 dict(rot=33), dict(rot=144), dict(style=2), dict(Hq=0), dict(Hkv=-1), dict(Hkv=0),
                                 dict(k=None), dict(ko=None), dict(q=None), dict(qo=None), dict(q=FAKE + 2),
                                 dict(qs=504), dict(qs=516), dict(kos=64), dict(qos=1024), dict(kos=256)], ids=str)
def test_refused_rotations(dk, bad):
    assert rotate(dk, **bad) == dk.E_INVAL


def test_rotations_not_implemented(dk):
    assert rotate(dk, rot=40) == dk.E_UNSUPPORTED
    assert rotate(dk, L=dk.layout(head_dim=64)) == dk.E_UNSUPPORTED
    assert rotate(dk, rows=0, pos=None, freq=None, q=None, qo=None, Hkv=0, k=None, ko=None) == dk.OK


def test_frequencies(dk):
    i = np.arange(32)
    plain = 10000.0 ** (-2.0 * i / 64)
    f, scale = dk.rope_frequencies(64)
    assert scale == 1.0 and np.array_equal(f.numpy(), plain.astype(np.float32))
    f, _ = dk.rope_frequencies(64, 10000.0, dk.ROPE_LINEAR, 4.0)
    assert np.array_equal(f.numpy(), (plain / 4.0).astype(np.float32))
    f, _ = dk.rope_frequencies(64, 10000.0, dk.ROPE_BASE, 4.0)
    want = (10000.0 * 4.0 ** (64 / 62)) ** (-2.0 * i / 64)
    assert np.allclose(f.numpy(), want, rtol=2.0 ** -23, atol=0)
    # the last frequency is stretched by the whole factor, the first not at all
    assert abs(f[-1].item() / (plain[-1] / 4.0) - 1) < 1e-6 and f[0].item() == 1.0
    f, scale = dk.rope_frequencies(64, 10000.0, dk.ROPE_BY_PARTS, 8.0, trained_len=2048, slow=1.0, fast=32.0)
    turns = 2048 * plain / (2 * math.pi)
    assert np.array_equal(f.numpy()[turns >= 32], plain.astype(np.float32)[turns >= 32])
    assert np.array_equal(f.numpy()[turns <= 1], (plain / 8).astype(np.float32)[turns <= 1])
    mid = (turns > 1) & (turns < 32)
    g = (turns[mid] - 1) / 31
    assert np.allclose(f.numpy()[mid], plain[mid] * (g + (1 - g) / 8), rtol=2.0 ** -23, atol=0)
    assert abs(scale - (0.1 * math.log(8.0) + 1)) < 1e-6


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=7), dict(base=0.0), dict(base=math.nan), dict(factor=0.5),
                                 dict(factor=math.inf), dict(scaling=4), dict(scaling=2, rot_dim=2),
                                 dict(scaling=3), dict(scaling=3, trained_len=100, slow=4.0, fast=4.0),
                                 dict(scaling=3, trained_len=100, slow=-1.0)], ids=str)
def test_refused_frequencies(dk, bad):
    with pytest.raises(dk.DiffKVError) as e:
        dk.rope_frequencies(**dict(dict(rot_dim=64), **bad))
    assert e.value.code == dk.E_INVAL


def test_binding_refuses_rows_that_are_not_packed(dk):
    class Nothing:
        num_kv_heads, num_seqs, L = 2, 1, dk.layout()
    x = torch.zeros((3, 8, 128), dtype=torch.float16)
    kv = torch.zeros((3, 2, 128), dtype=torch.float16)
    nl = torch.tensor([3], dtype=torch.int32)
    for q, k in ((x[:, ::2], kv), (x.float(), kv), (x[..., :64], kv), (x, kv[:2]), (x, x)):
        with pytest.raises(ValueError):
            dk.chunk_attention(Nothing, nl, q, k, kv, 0.1, out=x, lse=x, max_new=3, ws=x)
    with pytest.raises(ValueError):
        dk.rotate(dk.layout(), torch.zeros(3, dtype=torch.int64), torch.zeros(32), x)
    with pytest.raises(ValueError):
        dk.rotate(dk.layout(), torch.zeros(2, dtype=torch.int32), torch.zeros(32), x)


def test_binding_refuses_types_and_shapes(dk):
    class Nothing:
        num_kv_heads, num_seqs, L = 2, 1, dk.layout()
    q = torch.zeros((3, 8, 128), dtype=torch.float16)
    kv = torch.zeros((3, 2, 128), dtype=torch.float16)
    nl = torch.tensor([3], dtype=torch.int32)
    lse = torch.zeros((3, 8))
    good = dict(q=q, k=kv, v=kv, new_len=nl, out=q.clone(), lse=lse, slopes=None)
    for bad in (dict(q=q.bfloat16()), dict(k=kv.bfloat16()), dict(v=kv[..., :64].contiguous()), dict(new_len=nl.long()),
                dict(new_len=torch.zeros(2, dtype=torch.int32)), dict(out=q.float()), dict(out=q[:2]), dict(lse=lse.double()),
                dict(lse=lse[:, :7]), dict(slopes=torch.zeros(7)), dict(slopes=torch.zeros(8, dtype=torch.float64)),
                dict(q=q[..., :64].contiguous(), out=q[..., :64].contiguous())):
        a = dict(good, **bad)
        with pytest.raises(ValueError):
            dk.chunk_attention(Nothing, a["new_len"], a["q"], a["k"], a["v"], 0.1, slopes=a["slopes"], out=a["out"],
                               lse=a["lse"], max_new=3, ws=q)
    for bad in (dict(lse=lse.half()), dict(score=torch.zeros((3, 3))), dict(k=kv.float())):
        a = dict(good, score=torch.zeros((3, 2)), **bad) if "score" not in bad else dict(good, **bad)
        with pytest.raises(ValueError):
            dk.chunk_significance(Nothing, nl, a["q"], a["k"], 0.1, a["lse"], score=a["score"], max_new=3, ws=q)


def test_misaligned_workspaces(dk):
    L = dk.layout(max_seq_len=256)
    need = dk.workspace_size(dk.OP_CHUNK_ATTENTION, L, 2, 8, 2, 10)
    assert attention(dk, ws=FAKE + 8, ws_bytes=need) == dk.E_INVAL


@pytest.mark.parametrize("seqs,Hq,Hkv", [(1, 32, 8), (1, 8, 1), (128, 32, 8), (127, 32, 8), (1024, 4, 1), (3, 5, 5),
                                         (16, 64, 8), (2000, 8, 8)])
def test_a_workspace_for_more_rows_serves_fewer(dk, seqs, Hq, Hkv):
    L = dk.layout(max_seq_len=4096)
    rows = sorted(set(list(range(1, 700)) + [seqs - 1, seqs, seqs + 1, 1023, 1024, 1025, 5000, 70000]) - {0})
    need = [dk.workspace_size(dk.OP_CHUNK_ATTENTION, L, seqs, Hq, Hkv, r) for r in rows]
    assert need == sorted(need)
