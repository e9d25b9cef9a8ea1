"""Chunks of new tokens over the compressed cache: attention and scores against 64-bit definitions.

Tolerances, from the arithmetic.  A logit is an fp32 sum of exact products (codes times
halfs, group sums weighted by their scale): its error is at most a few dozen roundings of
the sum of its terms' magnitudes, delta = 64 * 2^-24 * sm_scale * sum |q||k| + 2^-20.
  out    weights and values are rounded to fp16 (half a step each, 2^-11), the result once
         more; weights below 2^-14 of the largest are fp16 denormals (2^-25 each):
         |err| <= 2^-11 (2 A + |out|) + 2 delta A + keys * 2^-25 * max|v|, A = sum p |v|;
  lse    delta + 2^-22 |lse|;
  score  relative 2 delta + 2^-20 (exp2, sums), of the mean before as well.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from chunk_ref import D, filled, kept_tokens, logits, score_at, softmax  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402

DEV = "cuda"
SCALE = 1.0 / np.sqrt(128.0)
LAYOUTS = [dict(), dict(v_bits=(8, 2)), dict(v_bits=(2, 1)), dict(tokens_per_page=(16, 16))]
H16 = 2.0 ** -11


def fused(rng, rows, Hq, Hkv, kscale=1.0):
    x = rng.standard_normal((rows, Hq + 2 * Hkv, D))
    x[:, Hq:Hq + Hkv] *= kscale
    x = torch.from_numpy(x.astype(np.float16)).to(DEV)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def delta(size):
    return 64 * 2.0 ** -24 * size.max(-1) + 2.0 ** -20


def check_attention(cache, new_len, q, k, v, out, lse, what="", **form):
    kept = kept_tokens(cache)
    got, got_lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    vv = v.cpu().numpy().astype(np.float64)
    G = q.shape[1] // cache.num_kv_heads
    for b, h, row, n, x, size in logits(cache, kept, new_len, q, k, SCALE, **form):
        vals = np.concatenate([kept[b * cache.num_kv_heads + h][1], vv[row:row + n, h]])
        p, want_lse = softmax(x)
        want = p @ vals
        A = p @ np.abs(vals)
        d = delta(size)
        tol = H16 * (2 * A + np.abs(want)) + 2 * d[..., None] * A + vals.shape[0] * 2.0 ** -25 * np.abs(vals).max()
        g = got[row:row + n, h * G:(h + 1) * G].transpose(1, 0, 2)
        bad = ~(np.abs(g - want) <= tol)
        assert not bad.any(), "%s b=%d h=%d: %d wrong, first %s: %r, expected %r" % (
            what, b, h, bad.sum(), np.argwhere(bad)[0], g[bad][0], want[bad][0])
        gl = got_lse[row:row + n, h * G:(h + 1) * G].T
        bad = ~(np.abs(gl - want_lse) <= d + 2.0 ** -22 * np.abs(want_lse))
        assert not bad.any(), "%s b=%d h=%d lse: %d wrong: %r, expected %r" % (
            what, b, h, bad.sum(), gl[bad][0], want_lse[bad][0])


def check_scores(cache, before, new_len, q, k, lse, score, what="", **form):
    """`before`: kept_tokens of the cache before the call."""
    H = cache.num_kv_heads
    G = q.shape[1] // H
    seen = cache.seq_len.cpu().numpy()
    lse = lse.cpu().numpy().astype(np.float64)
    got_own = score.cpu().numpy().astype(np.float64)
    touched = set()
    for b, h, row, n, x, size in logits(cache, before, new_len, q, k, SCALE, **form):
        _, _, pos, old, where = before[b * H + h]
        P = np.exp(x - lse[row:row + n, h * G:(h + 1) * G].T[..., None]).max(0)
        rel = 2 * delta(size).max() + 2.0 ** -20
        X = P.sum(0)
        m = len(pos)
        want = old + (X[:m] - n * old) / (seen[b] + n - pos)
        got = score_at(cache, where)
        tol = rel * (np.abs(old) * (1 + n / (seen[b] + n - pos)) + X[:m] / (seen[b] + n - pos)) + 1e-30
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), "%s b=%d h=%d: %d of %d wrong: %r, expected %r" % (
            what, b, h, bad.sum(), m, got[bad][0], want[bad][0])
        want = X[m:] / np.arange(n, 0, -1)
        g = got_own[row:row + n, h]
        bad = ~(np.abs(g - want) <= rel * want + 1e-30)
        assert not bad.any(), "%s own b=%d h=%d: %d wrong: %r, expected %r" % (
            what, b, h, bad.sum(), g[bad][0], want[bad][0])
        touched.add(b)
    for b in set(range(cache.num_seqs)) - touched:
        for h in range(H):
            _, _, _, old, where = before[b * H + h]
            assert np.array_equal(score_at(cache, where), old), "%s: scores of sequence %d changed" % (what, b)


def both(cache, new_len, q, k, v, what, **form):
    print("case:", what, flush=True)
    before = kept_tokens(cache)
    nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
    args = dict(form)
    if form.get("slopes") is not None:
        args["slopes"] = torch.tensor(form["slopes"], dtype=torch.float32, device=DEV)
    out, lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=max(new_len), **args)
    torch.cuda.synchronize()
    check_attention(cache, new_len, q, k, v, out, lse, what, **form)
    score = dk.chunk_significance(cache, nl, q, k, SCALE, lse, max_new=max(new_len), **args)
    torch.cuda.synchronize()
    check_scores(cache, before, new_len, q, k, lse, score, what, **form)


@pytest.mark.parametrize("layout", range(4))
@pytest.mark.parametrize("G", [1, 4, 7])
def test_layouts_and_group_sizes(layout, G):
    """Ragged chunks (none, one token, several tiles) over ragged caches (empty, partial pages)."""
    rng = np.random.default_rng(100 * layout + G)
    lens, new_len = [0, 1, 37, 300, 129, 64], [3, 1, 0, 40, 17, 1]
    cache = filled(dk, LAYOUTS[layout], 6, 2, lens, seed=layout)
    q, k, v = fused(rng, sum(new_len), 2 * G, 2)
    both(cache, new_len, q, k, v, "layout %d, G %d" % (layout, G))


@pytest.mark.parametrize("G", range(1, 9))
def test_single_tokens(G):
    rng = np.random.default_rng(G)
    lens = [0, 5, 16, 33, 700, 1500]
    cache = filled(dk, {}, 6, 2, lens, seed=G)
    q, k, v = fused(rng, 6, 2 * G, 2, kscale=3.0)
    both(cache, [1] * 6, q, k, v, "single tokens, G %d" % G)


@pytest.mark.parametrize("form", [dict(cap=20.0), dict(window=1), dict(window=45), dict(slopes=True),
                                  dict(cap=5.0, window=130, slopes=True)], ids=str)
@pytest.mark.parametrize("n", [1, 6, 70])
def test_score_forms(form, n):
    rng = np.random.default_rng(n)
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = (2.0 ** -np.arange(1, 7)).astype(np.float32)
    cache = filled(dk, {}, 3, 2, [200, 0, 431], seed=7)
    q, k, v = fused(rng, 2 * n + 1, 6, 2, kscale=2.0)
    both(cache, [n, 1, n], q, k, v, "form %s, n %d" % (form, n), **form)


@pytest.mark.parametrize("layout", range(1, 4))
def test_score_forms_in_other_layouts(layout):
    rng = np.random.default_rng(layout)
    slopes = (2.0 ** -np.arange(1, 11)).astype(np.float32)
    cache = filled(dk, LAYOUTS[layout], 2, 2, [333, 90], seed=9)
    q, k, v = fused(rng, 31, 10, 2)
    both(cache, [9, 22], q, k, v, "forms, layout %d" % layout, cap=10.0, window=100, slopes=slopes)


def test_long_chunk():
    rng = np.random.default_rng(3)
    cache = filled(dk, {}, 2, 1, [1100, 30], seed=5, max_len=2048)
    q, k, v = fused(rng, 700, 4, 1)
    both(cache, [699, 1], q, k, v, "a long chunk beside one token")


def test_peaked_and_large_scores():
    """Queries up to the fp16 range's end and rows of zeros: exponents of the row scaling."""
    rng = np.random.default_rng(11)
    cache = filled(dk, {}, 1, 1, [200], seed=6)
    q, k, v = fused(rng, 6, 2, 1)
    q = q.contiguous()
    q[0] *= 100.0
    q[1] = 0.0
    q[2] *= 1e-4
    q[3] *= 6e-8
    q[4, :, 0] = 60000.0
    both(cache, [6], q, k, v, "scales of q")
