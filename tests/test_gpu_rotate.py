"""Rotary positions against the 64-bit definition.

Tolerance: the products a cos t, b sin t and their sum in fp32, sine and cosine to about
2^-20 absolute: |err| <= (|a| + |b|) scale 2^-19, then one rounding to fp16 (2^-11 relative, 2^-25
where the result is an fp16 denormal).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from chunk_ref import D, rotated  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402

DEV = "cuda"
L = dk.layout()


def check(x, y, pos, freq, style, scale, what):
    want = rotated(x, pos, freq, style, scale)
    a = np.abs(x.cpu().numpy().astype(np.float64))
    half = len(freq)
    i = np.arange(half)
    lo, hi = (i, i + half) if style == 0 else (2 * i, 2 * i + 1)
    size = np.zeros_like(a)
    size[..., lo] = size[..., hi] = a[..., lo] + a[..., hi]
    tol = size * scale * 2.0 ** -19 + np.abs(want) * 2.0 ** -11 + 2.0 ** -25
    got = y.cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d wrong, first %s: %r, expected %r" % (
        what, bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0])
    rest = 2 * half
    assert torch.equal(x[..., rest:].contiguous().view(torch.int16), y[..., rest:].contiguous().view(torch.int16))


@pytest.mark.parametrize("style", [dk.ROPE_HALF, dk.ROPE_INTERLEAVED])
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("rows,Hq,Hkv", [(1, 1, 1), (5, 7, 1), (130, 32, 8), (2500, 9, 3)])
def test_rotate(style, rot, rows, Hq, Hkv):
    print("case: style %d, rot %d, %d rows, %d / %d heads" % (style, rot, rows, Hq, Hkv), flush=True)
    rng = np.random.default_rng(rot + rows)
    x = torch.from_numpy(rng.standard_normal((rows, Hq + 2 * Hkv, D)).astype(np.float16)).to(DEV)
    q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    pos = rng.integers(0, 1 << 20, rows).astype(np.int32)
    pos[0] = 0 if rows > 1 else 2 ** 31 - 1
    freq, scale = dk.rope_frequencies(rot, 10000.0, dk.ROPE_BY_PARTS, 8.0, trained_len=4096)
    assert scale > 1.0
    before = x.clone()
    qo, ko = dk.rotate(L, torch.from_numpy(pos).to(DEV), freq.to(DEV), q, k, style=style, scale=scale)
    torch.cuda.synchronize()
    check(q, qo, pos, freq, style, scale, "q")
    check(k, ko, pos, freq, style, scale, "k")
    assert torch.equal(x, before)


@pytest.mark.parametrize("style", [dk.ROPE_HALF, dk.ROPE_INTERLEAVED])
def test_in_place_in_a_fused_projection(style):
    """Turned inside the projection's output: the values and everything else stay as they were."""
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.standard_normal((77, 12, D)).astype(np.float16)).to(DEV)
    want = x.clone()
    pos = torch.arange(1000, 1077, dtype=torch.int32, device=DEV)
    freq, _ = dk.rope_frequencies(96)
    want[:, :8], want[:, 8:10] = dk.rotate(L, pos, freq.to(DEV), want[:, :8], want[:, 8:10], style=style)
    dk.rotate(L, pos, freq.to(DEV), x[:, :8], x[:, 8:10], style=style, q_out=x[:, :8], k_out=x[:, 8:10])
    torch.cuda.synchronize()
    assert torch.equal(x.view(torch.int16), want.view(torch.int16))


def test_queries_alone_and_no_rows():
    rng = np.random.default_rng(4)
    q = torch.from_numpy(rng.standard_normal((9, 4, D)).astype(np.float16)).to(DEV)
    pos = torch.full((9,), -5, dtype=torch.int32, device=DEV)
    freq, _ = dk.rope_frequencies(128, 500000.0)
    y, none = dk.rotate(L, pos, freq.to(DEV), q)
    torch.cuda.synchronize()
    assert none is None
    check(q, y, [-5] * 9, freq, dk.ROPE_HALF, 1.0, "q alone")
    dk.rotate(L, pos[:0], freq.to(DEV), q[:0])
