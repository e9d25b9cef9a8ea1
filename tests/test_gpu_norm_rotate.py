"""Norms of queries and keys with their rotary positions against the 64-bit definition.

Tolerance: the sum of squares (128 terms), its root and inverse and two products in fp32: 24 roundings, 2^-19.4 relative;
sine and cosine to about 2^-20 absolute: |err| <= size 2^-18 (size: |a| + |b| of the pair, or |y|), then one rounding to fp16 (2^-11
relative, 2^-25 where the result is an fp16 denormal).
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from block_ref import D, norm_rotated  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402

DEV = "cuda"
L = dk.layout()


def check(x, y, weight, eps, pos, freq, style, scale, what):
    want, size = norm_rotated(x.cpu().numpy(), weight, eps, pos, freq, style, scale)
    tol = size * 2.0 ** -18 + np.abs(want) * 2.0 ** -11 + 2.0 ** -25
    got = y.cpu().numpy().astype(np.float64)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d wrong, first %s: %r, expected %r" % (
        what, bad.sum(), np.argwhere(bad)[0], got[bad][0], want[bad][0])


def to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.mark.parametrize("style", [dk.ROPE_HALF, dk.ROPE_INTERLEAVED])
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("rows,Hq,Hkv", [(1, 1, 1), (5, 7, 1), (130, 32, 8), (2500, 9, 3)])
def test_norm_rotate(style, rot, rows, Hq, Hkv):
    print("case: style %d, rot %d, %d rows, %d / %d heads" % (style, rot, rows, Hq, Hkv), flush=True)
    rng = np.random.default_rng(rot + rows)
    x = rng.standard_normal((rows, Hq + 2 * Hkv, D)) * np.exp(2 * rng.standard_normal((rows, Hq + 2 * Hkv, 1)))
    x = to(x.astype(np.float16))
    q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    pos = rng.integers(0, 1 << 20, rows).astype(np.int32)
    pos[0] = 0 if rows > 1 else 2 ** 31 - 1
    freq, scale = dk.rope_frequencies(rot, 10000.0, dk.ROPE_BY_PARTS, 8.0, trained_len=4096)
    wq, wk = ((1 + 0.5 * rng.standard_normal(D)).astype(np.float32) for _ in (0, 1))
    before = x.clone()
    qo, ko = dk.norm_rotate(L, to(pos), freq.to(DEV), q, k, to(wq), to(wk), eps=1e-5, style=style, scale=scale)
    torch.cuda.synchronize()
    check(q, qo, wq, 1e-5, pos, freq, style, scale, "q")
    check(k, ko, wk, 1e-5, pos, freq, style, scale, "k")
    assert torch.equal(x, before)
    # one side's weights, queries alone, in place
    qo, ko = dk.norm_rotate(L, to(pos), freq.to(DEV), q, k, None, to(wk), eps=1e-5, style=style, scale=scale)
    check(q, qo, None, 1e-5, pos, freq, style, scale, "q without weights")
    only, none = dk.norm_rotate(L, to(pos), freq.to(DEV), q, q_weight=to(wq), eps=1e-5, style=style, scale=scale)
    assert none is None
    check(q, only, wq, 1e-5, pos, freq, style, scale, "q alone")
    dk.norm_rotate(L, to(pos), freq.to(DEV), q, k, None, to(wk), eps=1e-5, style=style, scale=scale, q_out=q, k_out=k)
    assert torch.equal(q, qo) and torch.equal(k, ko)
    assert torch.equal(x[:, Hq + Hkv:], before[:, Hq + Hkv:])


def test_heads_of_all_sizes():
    """Heads of zeros, of the smallest and the largest halfs, of one large value; values that are not finite."""
    x = np.zeros((1, 8, D), np.float16)
    x[0, 1] = 2.0 ** -24
    x[0, 2] = 65504
    x[0, 3, 9] = 65504
    x[0, 4] = np.linspace(-1, 1, D) * 2.0 ** -14
    x[0, 5] = 1
    x[0, 6, 3] = np.inf
    x[0, 7, 3] = np.nan
    freq = dk.rope_frequencies(32)[0]
    for eps in (1e-12, 1e-6, 1e6):
        y, _ = dk.norm_rotate(L, to(np.array([3], np.int32)), freq.to(DEV), to(x), eps=eps)
        torch.cuda.synchronize()
        check(to(x[:, :6]), y[:, :6], None, np.float32(eps), [3], freq, 0, 1.0, "sizes")
        assert torch.isnan(y[0, 7]).all() and torch.isnan(y[0, 6]).any()
