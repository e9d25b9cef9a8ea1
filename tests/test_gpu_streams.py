"""Calls on streams that are not the current one, with buffers that they take themselves: results as on one stream."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import block_ref as ref  # noqa: E402
from block_ref import D  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402

DEV = "cuda"
SCALE = 1.0 / np.sqrt(128.0)


def test_two_streams_without_buffers():
    """A layer's step on two streams by turns, while the current one fills what it allocates."""
    rng = np.random.default_rng(31)
    half = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float16)).to(DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    plain = ref.Plain(2, 2, dk.BLOCK_INT8)
    plain.append([900, 300], *(rng.standard_normal((1200, 2, D)).astype(np.float16) for _ in (0, 1)))
    c = ref.filled(dk, plain, 1200, DEV)
    freq = dk.rope_frequencies(D)[0].to(DEV)
    sizes = (1, 150)
    rows = [(half(2 * n, 8, D), half(2 * n, 2, D), half(2 * n, 2, D)) for n in sizes]
    lens, pos = [ints([n, n]) for n in sizes], [ints(list(range(2 * n))) for n in sizes]
    start, count = ints([3, 40]), ints([800, 200])

    def step(i, s):
        q, k, v = rows[i]
        qr, kr = dk.norm_rotate(c.L, pos[i], freq, q, k, stream=s)
        kb, vb = dk.block_read(c, start, count, 1000, max_count=800, stream=s)
        out, lse = dk.block_attention(c, lens[i], qr, kr, v, SCALE, max_new=sizes[i], stream=s)
        return qr, kr, kb, vb, out, lse

    want = [step(i, None) for i in (0, 1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(6):
        for i, s in enumerate(streams):
            got.append((i, step(i, s)))
        torch.empty(1 << 20, dtype=torch.uint8, device=DEV).fill_(0x7f)
    torch.cuda.synchronize()
    for i, results in got:
        assert all(torch.equal(x, y) for x, y in zip(results, want[i]))


def test_lengths_written_on_the_stream_of_the_call():
    """Without max_new the lengths are read where the call runs, behind what writes them there."""
    rng = np.random.default_rng(32)
    plain = ref.Plain(2, 1, dk.BLOCK_E4M3)
    plain.append([70, 40], *(rng.standard_normal((110, 1, D)).astype(np.float16) for _ in (0, 1)))
    c = ref.filled(dk, plain, 300, DEV)
    q, k, v = (torch.from_numpy(rng.standard_normal((90, h, D)).astype(np.float16)).to(DEV) for h in (4, 1, 1))
    lens = torch.tensor([80, 10], dtype=torch.int32, device=DEV)
    want = dk.block_attention(c, lens, q, k, v, SCALE)
    a = torch.randn((4096, 4096), device=DEV)
    late = torch.zeros_like(lens)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            a = a @ a
            a = a / a.abs().max()
        late.copy_(lens)
    got = dk.block_attention(c, late, q, k, v, SCALE, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
