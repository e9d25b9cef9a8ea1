"""The uniform 8-bit cache's attention where its operands are not finite, and its ends: against the 64-bit definitions of
block_ref.  Tolerances as test_gpu_block derives them."""
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
E4M3, INT8 = dk.BLOCK_E4M3, dk.BLOCK_INT8
FORMS = {"plain": {}, "windowed": dict(window=45, sinks=5), "formed": dict(cap=20.0, slopes=True),
         "all": dict(cap=5.0, slopes=True, window=45, sinks=5)}


def halves(rng, *shape, size=1.0):
    return (rng.standard_normal(shape) * size).astype(np.float16)


def to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def plain_of(rng, lens, H, fmt):
    p = ref.Plain(len(lens), H, fmt)
    p.append(lens, halves(rng, sum(lens), H, D), halves(rng, sum(lens), H, D))
    return p


def form_of(name, heads):
    form = dict(FORMS[name])
    if form.get("slopes"):
        form["slopes"] = (2.0 ** -np.arange(1, heads + 1)).astype(np.float32)
    return form


def attend(plain, new, q, k, v, scale=SCALE, room=0, drop=(), **form):
    """Outputs and normalizers of new's rows as numpy; `room` rows more are in the call than the sequences have."""
    c = ref.filled(dk, plain, max(len(r[0]) for r in plain.rows) + max(new), DEV, drop=drop)
    if form.get("slopes") is not None:
        form["slopes"] = to(form["slopes"])
    q, k, v = (to(np.concatenate([x, np.zeros((room,) + x.shape[1:], x.dtype)])) for x in (q, k, v))
    out, lse = dk.block_attention(c, ints(new), q, k, v, scale, max_new=max(new) + room, **form)
    torch.cuda.synchronize()
    return out.cpu().numpy()[:sum(new)].astype(np.float64), lse.cpu().numpy()[:sum(new)].astype(np.float64)


def check(plain, new, q, k, v, got, what, scale=SCALE, measure=None, drop=(), **form):
    """Values within their tolerances, and what is not finite as it should be.  `measure`: (plain, k) whose products say
    how far the scores may be off, where those of plain and k are infinite."""
    kept = lambda b, i: (b, i) not in drop
    G = q.shape[1] // plain.H
    with np.errstate(all="ignore"):
        sizes = [x[6:] for x in ref.attention((measure or (plain, k))[0], new, q, (measure or (plain, k))[1],
                                              np.nan_to_num(v, posinf=0, neginf=0), scale, kept, **form)]
        for (b, h, row, n, want, want_lse, *_), (A, size, keys, V) in zip(ref.attention(plain, new, q, k, v, scale, kept, **form), sizes):
            A, V = np.nan_to_num(A), float(np.nan_to_num(V))
            size = np.nan_to_num(size)
            d = 64 * 2.0 ** -24 * size + 2.0 ** -20
            tol = 2.0 ** -11 * np.abs(want) + (2 * d[..., None] + 2.0 ** -20 + keys * 2.0 ** -28) * A + \
                keys * 2.0 ** -31 * V * max(1.0, V) + 2.0 ** -25
            g = got[0][row:row + n, h * G:(h + 1) * G].transpose(1, 0, 2)
            fine = np.isfinite(want)
            odd = np.isfinite(g) != fine
            assert not odd.any(), "%s b=%d h=%d: %d that should (not) be finite" % (what, b, h, odd.sum())
            bad = fine & ~(np.abs(g - want) <= tol)
            assert not bad.any(), "%s b=%d h=%d: %d wrong, first %s: %r, expected %r" % (
                what, b, h, bad.sum(), np.argwhere(bad)[0], g[bad][0], want[bad][0])
            gl = got[1][row:row + n, h * G:(h + 1) * G].T
            fine = np.isfinite(want_lse)
            odd = np.isfinite(gl) != fine
            assert not odd.any(), "%s b=%d h=%d: %d lse that should (not) be finite" % (what, b, h, odd.sum())
            bad = fine & ~(np.abs(gl - want_lse) <= d + 2.0 ** -22 * np.abs(want_lse))
            assert not bad.any(), "%s b=%d h=%d lse: %r, expected %r" % (what, b, h, gl[bad][0], want_lse[bad][0])


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("n", [6, 200])  # (few rows, many)
def test_a_block_whose_values_read_nan(fmt, form, n):
    """The outputs of the rows that see one of its tokens are NaN; their normalizers know no values."""
    rng = np.random.default_rng(41)
    form = form_of(form, 4)
    lens, new = [100, 64], [n, n]
    plain = plain_of(rng, lens, 1, fmt)
    plain.rows[0][1][40, 0, 17] = np.nan
    q, k, v = halves(rng, 2 * n, 4, D), halves(rng, 2 * n, 1, D), halves(rng, 2 * n, 1, D)
    got = attend(plain, new, q, k, v, **form)
    assert np.isfinite(got[1]).all() and np.isnan(got[0][0]).all() and np.isfinite(got[0][n:]).all()
    check(plain, new, q, k, v, got, "values", **form)


@pytest.mark.parametrize("scale", [1e-30, 1e-38, 1e-42, 1.5e-45])
@pytest.mark.parametrize("n", [6, 200])
def test_scales_of_scores_down_to_zero(scale, n):
    """Hidden tokens stay hidden where a score's scale rounds to nothing."""
    rng = np.random.default_rng(42)
    plain = plain_of(rng, [100, 0], 1, E4M3)
    plain.rows[0][0][:] *= np.float16(2.0 ** -12)
    new = [n, n]
    q, k, v = halves(rng, 2 * n, 4, D), halves(rng, 2 * n, 1, D), halves(rng, 2 * n, 1, D)
    got = attend(plain, new, q, k, v, scale=scale, window=45, sinks=5)
    check(plain, new, q, k, v, got, "scale %g" % scale, scale=scale, window=45, sinks=5)


# ---- forms over both formats -----------------------------------------------------------------


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("form", [dict(cap=20.0), dict(slopes=True), dict(cap=5.0, window=130, sinks=2, slopes=True),
                                  dict(cap=30.0, window=64, sinks=300), dict(window=64, sinks=300)], ids=str)
@pytest.mark.parametrize("n,G", [(1, 3), (9, 7), (70, 2), (300, 4)])
def test_forms_of_both_formats(fmt, form, n, G):
    """Few rows and many, two KV heads, first tokens that reach past the window among them."""
    print("case: fmt %d %s n %d G %d" % (fmt, form, n, G), flush=True)
    rng = np.random.default_rng(43 + n)
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = (2.0 ** -np.arange(1, 2 * G + 1)).astype(np.float32)
    lens, new = [431, 0, 200, 96], [n, n, 1, n + 3]
    plain = plain_of(rng, lens, 2, fmt)
    q, k, v = (halves(rng, sum(new), h, D) for h in (2 * G, 2, 2))
    check(plain, new, q, k, v, attend(plain, new, q, k, v, **form), "forms", **form)


# ---- operands that are not finite ------------------------------------------------------------


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n", [6, 200])
def test_operands_that_are_not_finite(fmt, form, bad, n):
    """Every value and normalizer of every row, the rows that see the token and those that do not: a key of a capped form may be
    infinite, an infinite score without one is NaN or hides its token, a block reads NaN whatever it met."""
    form = form_of(form, 4)
    for where in ("own k", "own v", "tail k", "tail v", "block k", "block v"):
        rng = np.random.default_rng(44)
        lens, new = [100, 64], [n, n]
        clean = plain_of(rng, lens, 1, fmt)
        plain = ref.Plain(2, 1, fmt)
        plain.rows = [[x.copy() for x in r] for r in clean.rows]
        q, k, v = halves(rng, 2 * n, 4, D), halves(rng, 2 * n, 1, D), halves(rng, 2 * n, 1, D)
        k0 = k.copy()
        if where == "own k":
            k[3, 0, 17], k0[3, 0, 17] = bad, 0
        elif where == "own v":
            v[3, 0, 17] = bad
        else:
            plain.rows[0][1 if where[-1] == "v" else 0][98 if where[0] == "t" else 40, 0, 17] = bad
            clean.rows[0][0][98, 0, 17] = 0
        got = attend(plain, new, q, k, v, **form)
        if where[:5] == "block":
            assert np.isnan(got[0][0]).all() and np.isfinite(got[0][n:]).all()
        check(plain, new, q, k, v, got, where, measure=(clean, k0), **form)


# ---- weights -----------------------------------------------------------------------------


@pytest.mark.parametrize("room", [0, 400], ids=["few", "many"])  # (a lone sequence of a padded call goes to the many-row kernel)
@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_small_weights_behind_large_ones(fmt, room):
    """In every block one token of no value with a weight 2^26.5 times that of the others, which carry all of it."""
    n = 4096
    plain = ref.Plain(1, 1, fmt)
    k, v = np.zeros((n, 1, D), np.float16), np.zeros((n, 1, D), np.float16)
    k[:, :, 0], v[:, :, 0] = -1.0, 1024.0
    k[::32, :, 0], v[::32] = 1.0, 0.0
    plain.append([n], k, v)
    q, own_k, own_v = (np.zeros((1, 1, D), np.float16) for _ in range(3))
    q[:, :, 0] = 26.5 * np.log(2.0) / SCALE / 2
    own_k[:, :, 0] = 1.0
    out, lse = attend(plain, [1], q, own_k, own_v, room=room)
    _, _, _, _, want, want_lse, A, size, _, V = next(ref.attention(plain, [1], q, own_k, own_v, SCALE, lambda b, i: True))
    # A block's large token has u = 2^12 and the others' u is off by half an fp16 denormal's step, 2^-25, at most: with one scale
    # for all blocks 32 of them to a large one, 32 2^-37 V of the result.  The scores as test_gpu_block has them.
    d = 64 * 2.0 ** -24 * float(size[0, 0]) + 2.0 ** -20
    tol = 2.0 ** -11 * abs(want[0, 0, 0]) + 32 * 2.0 ** -37 * V + (2 * d + 2.0 ** -20) * A[0, 0, 0] + 2.0 ** -25
    assert want[0, 0, 0] > 2.0 ** -12 and tol < 2.0 ** -20
    assert abs(out[0, 0, 0] - want[0, 0, 0]) <= tol
    assert abs(lse[0, 0] - want_lse[0, 0]) <= d + 2.0 ** -22 * abs(want_lse[0, 0])


@pytest.mark.parametrize("room", [0, 400], ids=["few", "many"])
@pytest.mark.parametrize("fmt,stored", [(INT8, True), (E4M3, True), (E4M3, False)])
def test_weights_in_two_parts(fmt, stored, room):
    """Two tokens of opposite values and nearly equal weights, stored and own: to 2^-20 of their sum."""
    lens = 64 if stored else 1
    plain = ref.Plain(1, 1, fmt)
    k, v = np.zeros((lens, 1, D), np.float16), np.zeros((lens, 1, D), np.float16)
    k[:, :, 1] = -100.0 if stored else 0.0
    k[0, 0, 1] = 0.0
    v[0] = 1.0
    plain.append([lens], k, v)
    for eps in (2.0 ** -9, 3 * 2.0 ** -11, 2.0 ** -6):
        q, own_k, own_v = np.zeros((1, 1, D), np.float16), np.zeros((1, 1, D), np.float16), np.full((1, 1, D), -1.0, np.float16)
        q[:, :, 0], q[:, :, 1], own_k[:, :, 0] = 1.0, 64.0, eps
        out, _ = attend(plain, [1], q, own_k, own_v, room=room)
        held, x = plain.read(0, 0, 1, lambda i: True)[0][0, 0], eps * SCALE
        want = (held - np.exp(x)) / (1 + np.exp(x))
        assert abs(out[0, 0, 0] - want) <= 2.0 ** -20 + 2.0 ** -11 * abs(want), eps
