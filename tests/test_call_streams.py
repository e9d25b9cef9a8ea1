"""A call that is given a stream and no buffers takes its buffers from that stream: the current one would hand their
bytes on while the call's kernels still use them.  CPU only: the library and torch's streams are stood in for."""
import contextlib

import pytest
import torch

from paper_2412_03131_amd import diffkv as dk

HERE, OTHER = 0x10, 0x20


class Stream:
    def __init__(self, address):
        self.cuda_stream, self.device = address, torch.device("cuda", 0)


@pytest.fixture
def calls(monkeypatch):
    """The binding over a library that only counts calls; what it allocates, with the stream that was current then."""
    try:
        real = dk.lib()
    except OSError:
        import __graft_entry__
        __graft_entry__.build()
        real = dk.lib()
    seen = dict(current=[HERE], allocated=[], launched=[])

    class Library:
        def __getattr__(self, name):
            if name in ("diffkv_workspace_size", "diffkv_status_str", "diffkv_layout_init", "diffkv_rope_frequencies"):
                return getattr(real, name)
            return lambda *args: seen["launched"].append(name) or dk.OK

    @contextlib.contextmanager
    def on(stream):
        seen["current"].append(stream.cuda_stream)
        yield
        seen["current"].pop()

    empty = torch.empty
    monkeypatch.setattr(dk, "lib", Library)
    monkeypatch.setattr(dk, "_on_one_gpu", lambda *args: None)
    monkeypatch.setattr(dk, "_stream_at", lambda what, stream, t: dk._stream(stream))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: seen["current"][-1], raising=False)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: seen["allocated"].append(seen["current"][-1]) or empty(*a, **k))
    return seen


def operators():
    """Name -> a call without buffers, its lengths given, and how many buffers it takes."""
    L = dk.layout(max_seq_len=256)
    f16, i32, f32 = torch.float16, torch.int32, torch.float32
    q, kv = torch.zeros((3, 4, 128), dtype=f16), torch.zeros((3, 2, 128), dtype=f16)
    lens, score, lse = torch.tensor([2, 1], dtype=i32), torch.zeros((3, 2), dtype=f32), torch.zeros((3, 4), dtype=f32)
    pos, freq = torch.zeros(3, dtype=i32), torch.zeros(64, dtype=f32)
    c, u = dk.Cache(L, 8, 2, 2, device="cpu"), dk.BlockCache(L, 8, 2, 2, device="cpu")
    return {
        "quantize_append": (lambda s: dk.quantize_append(c, lens, kv, kv, score, total_new=3, max_new=2, stream=s), 1),
        "decode_attention": (lambda s: dk.decode_attention(c, q[:2], 0.1, stream=s), 3),
        "prompt_significance": (lambda s: dk.prompt_significance(L, lens, q, kv, 0.1, max_new=2, stream=s), 2),
        "rotate": (lambda s: dk.rotate(L, pos, freq, q, kv, stream=s), 2),
        "norm_rotate": (lambda s: dk.norm_rotate(L, pos, freq, q, kv, stream=s), 2),
        "chunk_attention": (lambda s: dk.chunk_attention(c, lens, q, kv, kv, 0.1, max_new=2, stream=s), 3),
        "chunk_significance": (lambda s: dk.chunk_significance(c, lens, q, kv, 0.1, lse, max_new=2, stream=s), 2),
        "block_read": (lambda s: dk.block_read(u, lens, lens, 3, max_count=2, stream=s), 2),
        "block_attention": (lambda s: dk.block_attention(u, lens, q, kv, kv, 0.1, max_new=2, stream=s), 3),
        "compact_free_list": (lambda s: dk.compact_free_list(c, torch.zeros((4, L.p_max), dtype=torch.uint8), stream=s), 1),
        "alloc_pages": (lambda s: dk.alloc_pages(c, torch.zeros((4, 2), dtype=i32), stream=s), 1),
        "generation_step": (lambda s: dk.generation_step(c, 1.0, 0.1, 64, stream=s), 1),
    }


@pytest.mark.parametrize("name", ["quantize_append", "decode_attention", "prompt_significance", "rotate", "norm_rotate",
                                  "chunk_attention", "chunk_significance", "block_read", "block_attention",
                                  "compact_free_list", "alloc_pages", "generation_step"])
@pytest.mark.parametrize("given", [None, HERE, OTHER], ids=["none", "current", "other"])
def test_buffers_come_from_the_stream_of_the_call(calls, name, given):
    call, buffers = operators()[name]
    calls["allocated"].clear()
    call(None if given is None else Stream(given))
    assert calls["launched"] == ["diffkv_" + name]
    assert calls["allocated"] == [HERE if given is None else given] * buffers
    assert calls["current"] == [HERE]


@pytest.mark.parametrize("name", ["quantize_append", "prompt_significance", "chunk_attention", "chunk_significance",
                                  "block_append", "block_read", "block_attention"])
@pytest.mark.parametrize("given", [None, HERE, OTHER], ids=["none", "current", "other"])
def test_lengths_are_read_on_the_stream_of_the_call(calls, monkeypatch, name, given):
    """A program may still be writing them there."""
    L = dk.layout(max_seq_len=256)
    f16, i32, f32 = torch.float16, torch.int32, torch.float32
    q, kv, lens = torch.zeros((3, 4, 128), dtype=f16), torch.zeros((3, 2, 128), dtype=f16), torch.tensor([2, 1], dtype=i32)
    score, lse = torch.zeros((3, 2), dtype=f32), torch.zeros((3, 4), dtype=f32)
    c, u = dk.Cache(L, 8, 2, 2, device="cpu"), dk.BlockCache(L, 8, 2, 2, device="cpu")
    s = None if given is None else Stream(given)
    call = {
        "quantize_append": lambda: dk.quantize_append(c, lens, kv, kv, score, stream=s),
        "prompt_significance": lambda: dk.prompt_significance(L, lens, q, kv, 0.1, stream=s),
        "chunk_attention": lambda: dk.chunk_attention(c, lens, q, kv, kv, 0.1, stream=s),
        "chunk_significance": lambda: dk.chunk_significance(c, lens, q, kv, 0.1, lse, stream=s),
        "block_append": lambda: dk.block_append(u, lens, kv, kv, stream=s),
        "block_read": lambda: dk.block_read(u, lens, lens, 3, stream=s),
        "block_attention": lambda: dk.block_attention(u, lens, q, kv, kv, 0.1, stream=s),
    }[name]
    read, real_max, real_cpu = [], torch.Tensor.max, torch.Tensor.cpu
    monkeypatch.setattr(torch.Tensor, "max", lambda t, *a: read.append(calls["current"][-1]) or real_max(t, *a))
    monkeypatch.setattr(torch.Tensor, "cpu", lambda t, *a: read.append(calls["current"][-1]) or real_cpu(t, *a))
    call()
    assert calls["launched"] == ["diffkv_" + name]
    # (quantize_append copies them to the host first: what it does there is no matter)
    assert read[0] == (HERE if given is None else given)
    assert calls["current"] == [HERE]
