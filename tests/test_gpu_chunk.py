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


@pytest.mark.parametrize("B,Hkv,G", [(20, 8, 4), (130, 2, 3), (200, 8, 5)])
def test_many_tables(B, Hkv, G):
    """160 and 260 tables (cut into pieces by a workgroup's scan) and 1600 (none is cut)."""
    rng = np.random.default_rng(B)
    lens = rng.integers(0, 90, B)
    lens[B // 2] = 700
    new_len = rng.integers(0, 3, B)
    new_len[0] = 1
    cache = filled(dk, {}, B, Hkv, lens, seed=B, max_len=1400)
    q, k, v = fused(rng, int(new_len.sum()), Hkv * G, Hkv)
    both(cache, new_len.tolist(), q, k, v, "%d tables" % (B * Hkv))


def test_mixture_of_lengths():
    """One token, a few, tens and hundreds side by side: every kernel of a call has some of the rows."""
    rng = np.random.default_rng(17)
    lens, new_len = [900, 0, 431, 64, 1200, 5], [1, 300, 8, 0, 30, 2]
    cache = filled(dk, {}, 6, 2, lens, seed=3, max_len=2048)
    q, k, v = fused(rng, sum(new_len), 10, 2)
    both(cache, new_len, q, k, v, "mixture")
    slopes = (2.0 ** -np.arange(10)).astype(np.float32)
    both(cache, new_len, q, k, v, "mixture, forms", cap=15.0, window=250, slopes=slopes)


@pytest.mark.parametrize("n", [1, 9, 80])
def test_pages_outside_the_pool_count_no_tokens(n):
    """Page IDs that the caller has lost (-1, too large): their tokens are not attended to, their scores not
    written, and nothing outside the pool is read."""
    rng = np.random.default_rng(n)
    cache = filled(dk, {}, 2, 1, [400, 300], seed=12)
    L = cache.L
    cache.page_table[0, 1] = -1
    cache.page_table[0, 4] = cache.num_pages
    cache.page_table[0, L.p_max - 2] = 2 ** 31 - 1
    cache.page_table[1, L.p_max - 1] = -7
    q, k, v = fused(rng, 2 * n, 4, 1)
    both(cache, [n, n], q, k, v, "lost pages, n %d" % n)


@pytest.mark.parametrize("n", [6, 90])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_non_finite_own_values_stay_with_their_token(n, bad):
    """A chunk's infinite or NaN key or value reaches the rows that see its token, and no other."""
    rng = np.random.default_rng(n)
    cache = filled(dk, {}, 2, 1, [100, 50], seed=8)
    q, k, v = (x.contiguous() for x in fused(rng, 2 * n, 4, 1))
    nl = torch.tensor([n, n], dtype=torch.int32, device=DEV)
    at = n // 2
    want, want_lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=n)
    v[at, 0, 77] = bad
    k[n + at, 0, 5] = float("nan")
    print("case: non-finite own values, n %d" % n, flush=True)
    out, lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=n)
    torch.cuda.synchronize()
    assert torch.equal(out[:at], want[:at]) and torch.equal(lse[:n], want_lse[:n])
    assert not torch.isfinite(out[at:n, :, 77]).any()
    others = torch.arange(D, device=DEV) != 77
    assert torch.equal(out[at:n][..., others], want[at:n][..., others])
    assert torch.equal(out[n:n + at], want[n:n + at]) and torch.isnan(out[n + at:]).all()
    assert torch.isnan(lse[n + at:]).all()


def test_rows_of_no_sequence_and_workspace_bounds():
    """Rows that no sequence owns stay as they were; nothing behind a workspace of the exact size is written."""
    rng = np.random.default_rng(5)
    cache = filled(dk, {}, 3, 2, [300, 40, 0], seed=2)
    for new_len in ([1, 1, 0], [5, 0, 2], [90, 20, 1]):
        rows = sum(new_len) + 7
        q, k, v = fused(rng, rows, 8, 2)
        nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
        out = torch.full((rows, 8, D), 7.0, dtype=torch.float16, device=DEV)
        lse = torch.full((rows, 8), 7.0, device=DEV)
        score = torch.full((rows, 2), 7.0, device=DEV)
        print("case: rows of no sequence, %s" % new_len, flush=True)
        for op in (dk.OP_CHUNK_ATTENTION, dk.OP_CHUNK_SIGNIFICANCE):
            need = dk.workspace_size(op, cache.L, 3, 8, 2, rows)
            ws = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=DEV)
            if op == dk.OP_CHUNK_ATTENTION:
                dk.chunk_attention(cache, nl, q, k, v, SCALE, out=out, lse=lse, max_new=max(new_len), ws=ws[:need])
            else:
                dk.chunk_significance(cache, nl, q, k, SCALE, lse, score=score, max_new=max(new_len), ws=ws[:need])
            torch.cuda.synchronize()
            assert bool((ws[need:] == 0x5A).all())
            with pytest.raises(ValueError):
                if op == dk.OP_CHUNK_ATTENTION:
                    dk.chunk_attention(cache, nl, q, k, v, SCALE, out=out, lse=lse, max_new=max(new_len),
                                       ws=ws[:need - 1])
                else:
                    dk.chunk_significance(cache, nl, q, k, SCALE, lse, score=score, max_new=max(new_len),
                                          ws=ws[:need - 1])
        n = sum(new_len)
        check_attention(cache, new_len, q[:n], k[:n], v[:n], out[:n], lse[:n], "rows")
        for t in (out, lse, score):
            assert bool((t[n:] == 7.0).all())


def test_strides_and_dense_rows_agree():
    """The same rows as slices of a wider projection and dense: bit for bit the same."""
    rng = np.random.default_rng(6)
    cache = filled(dk, {}, 2, 2, [500, 33], seed=4)
    for new_len in ([1, 1], [40, 3]):
        wide = torch.from_numpy(rng.standard_normal((sum(new_len), 30, D)).astype(np.float16)).to(DEV)
        q, k, v = wide[:, 3:13], wide[:, 20:22], wide[:, 25:27]
        nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
        a = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=max(new_len))
        b = dk.chunk_attention(cache, nl, q.contiguous(), k.contiguous(), v.contiguous(), SCALE, max_new=max(new_len))
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_pool_beyond_32_bits():
    """Pages more than 2^32 bytes into the pool."""
    rng = np.random.default_rng(9)
    cache = filled(dk, {}, 2, 1, [300, 70], seed=1, before=(1 << 32) // 4352 + 10)
    q, k, v = fused(rng, 41, 4, 1)
    both(cache, [1, 40], q, k, v, "a pool of over 4 GiB")


def test_captured_and_replayed():
    """A step's calls captured into a graph: every replay, with eager calls and new inputs between, equals
    the eager result bit for bit (the workspace's arrival words carry each call's own tag)."""
    rng = np.random.default_rng(21)
    for new_len in ([1, 1, 1], [60, 1, 9]):
        cache = filled(dk, {}, 3, 2, [900, 40, 333], seed=5)
        rows, longest = sum(new_len), max(new_len)
        nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
        draws = [fused(rng, rows, 8, 2) for _ in range(3)]
        q, k, v = (x.contiguous() for x in draws[0])
        pos = torch.arange(rows, dtype=torch.int32, device=DEV) + 1000
        freq = dk.rope_frequencies(128)[0].to(DEV)
        qr, kr = torch.empty_like(q), torch.empty_like(k)
        out = torch.empty((rows, 8, D), dtype=torch.float16, device=DEV)
        lse = torch.empty((rows, 8), device=DEV)
        score = torch.empty((rows, 2), device=DEV)
        ws = [torch.empty(dk.workspace_size(op, cache.L, 3, 8, 2, rows), dtype=torch.uint8, device=DEV)
              for op in (dk.OP_CHUNK_ATTENTION, dk.OP_CHUNK_SIGNIFICANCE)]

        def step():
            dk.rotate(cache.L, pos, freq, q, k, q_out=qr, k_out=kr)
            dk.chunk_attention(cache, nl, qr, kr, v, SCALE, out=out, lse=lse, max_new=longest, ws=ws[0])
            dk.chunk_significance(cache, nl, qr, kr, SCALE, lse, score=score, max_new=longest, ws=ws[1])

        pool = cache.pool.clone()
        want = []
        for d in draws:
            for x, y in zip((q, k, v), d):
                x.copy_(y)
            cache.pool.copy_(pool)
            step()
            want.append([x.clone() for x in (out, lse, score, cache.pool)])
        torch.cuda.synchronize()
        print("case: captured, %s" % new_len, flush=True)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for i in (0, 2, 1, 0, 1):
            for x, y in zip((q, k, v), draws[i]):
                x.copy_(y)
            cache.pool.copy_(pool)
            g.replay()
            for x, y in zip((out, lse, score, cache.pool), want[i]):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            torch.cuda.synchronize()
            cache.pool.copy_(pool)
            step()  # eager, with the same workspaces
            assert torch.equal(out, want[i][0])


def test_two_streams():
    """Calls that may overlap, on streams of their own with workspaces of their own."""
    rng = np.random.default_rng(31)
    caches = [filled(dk, {}, 2, 2, lens, seed=s) for s, lens in ((1, [900, 100]), (2, [50, 700]))]
    new = [[1, 1], [70, 5]]
    args = [fused(rng, sum(n), 8, 2) for n in new]
    lens = [torch.tensor(n, dtype=torch.int32, device=DEV) for n in new]
    want = [dk.chunk_attention(c, l, *a, SCALE, max_new=max(n)) for c, l, a, n in zip(caches, lens, args, new)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [[torch.empty_like(x) for x in w] for w in want]
    ws = [torch.empty(dk.workspace_size(dk.OP_CHUNK_ATTENTION, c.L, 2, 8, 2, sum(n)), dtype=torch.uint8, device=DEV)
          for c, n in zip(caches, new)]
    torch.cuda.synchronize()
    for _ in range(8):
        for i in (0, 1):
            dk.chunk_attention(caches[i], lens[i], *args[i], SCALE, out=got[i][0], lse=got[i][1], max_new=max(new[i]),
                               ws=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w[0], g[0]) and torch.equal(w[1], g[1])


def test_prompt_in_parts_then_decoding():
    """The operators as they are used: a prompt in three parts, then decoded tokens, each step rotated,
    attended, scored and appended; every step against its definition on the cache as it then is."""
    rng = np.random.default_rng(41)
    B, Hkv, G = 2, 2, 4
    L = dk.layout(max_seq_len=1024)
    cache = dk.Cache(L, 4 * 2 * 80, B, Hkv, device=DEV)
    freq, scale = dk.rope_frequencies(64, 10000.0, dk.ROPE_LINEAR, 2.0)
    freq = freq.to(DEV)
    seen = np.zeros(B, np.int64)
    for step, new_len in enumerate(([90, 40], [70, 0], [33, 120], [1, 1], [1, 1], [4, 1])):
        rows = sum(new_len)
        q, k, v = fused(rng, rows, G * Hkv, Hkv)
        pos = np.concatenate([seen[b] + np.arange(n) for b, n in enumerate(new_len)]).astype(np.int32)
        qr, kr = dk.rotate(L, torch.from_numpy(pos).to(DEV), freq, q, k, style=dk.ROPE_INTERLEAVED, scale=scale)
        nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
        print("case: step %d, %s" % (step, new_len), flush=True)
        before = kept_tokens(cache)
        out, lse = dk.chunk_attention(cache, nl, qr, kr, v, SCALE, max_new=max(new_len), window=200)
        torch.cuda.synchronize()
        check_attention(cache, new_len, qr, kr, v, out, lse, "step %d" % step, window=200)
        score = dk.chunk_significance(cache, nl, qr, kr, SCALE, lse, max_new=max(new_len), window=200)
        torch.cuda.synchronize()
        check_scores(cache, before, new_len, qr, kr, lse, score, "step %d" % step, window=200)
        dk.quantize_append(cache, nl, kr, v.contiguous(), score, alpha_h=1.0, alpha_l=0.2, window=16, total_new=rows,
                           max_new=max(new_len))
        torch.cuda.synchronize()
        assert int(cache.status.cpu()[0]) == 0
        seen += new_len
        assert cache.seq_len.cpu().tolist() == seen.tolist()


def test_a_prompt_without_a_cache_scores_as_the_prompt_operator():
    """On an empty cache the chunk's scores are the prompt's."""
    rng = np.random.default_rng(51)
    cache = filled(dk, {}, 2, 2, [0, 0], seed=1)
    new_len = [150, 37]
    q, k, v = (x.contiguous() for x in fused(rng, sum(new_len), 8, 2))
    nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
    _, lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=150)
    score = dk.chunk_significance(cache, nl, q, k, SCALE, lse, max_new=150)
    want = dk.prompt_significance(cache.L, nl, q, k, SCALE, max_new=150)
    torch.cuda.synchronize()
    # both within 5e-5 of the definition
    assert torch.allclose(score, want, rtol=1e-4, atol=1e-30)


def test_a_single_token_scores_as_the_step_operator():
    """One new token: the cached scores move as the one-query update moves them once its softmax counts
    the token too (same lse, same N)."""
    rng = np.random.default_rng(52)
    cache = filled(dk, {}, 3, 2, [200, 31, 90], seed=6)
    q, k, v = (x.contiguous() for x in fused(rng, 3, 8, 2))
    nl = torch.ones(3, dtype=torch.int32, device=DEV)
    _, lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=1)
    pool = cache.pool.clone()
    dk.chunk_significance(cache, nl, q, k, SCALE, lse, max_new=1)
    kept = kept_tokens(cache)
    got = [t[3] for t in kept]
    cache.pool.copy_(pool)
    cache.seq_len += 1
    dk.update_significance(cache, q, SCALE, lse)
    torch.cuda.synchronize()
    for g, t in zip(got, kept_tokens(cache)):
        assert np.allclose(g, t[3], rtol=5e-5, atol=1e-30)


@pytest.mark.parametrize("n", [1, 6, 90])
def test_values_at_the_ends_of_fp16(n):
    """Cached groups whose largest value s c + z rounds past the largest finite half."""
    rng = np.random.default_rng(n)
    L = dk.layout(max_seq_len=512)
    cache = dk.Cache(L, 64, 1, 1, device=DEV)
    v = torch.from_numpy(np.where(rng.random((96, 1, D)) < 0.5, 65504.0, -65504.0).astype(np.float16)).to(DEV)
    v[::3] = torch.from_numpy(rng.uniform(-65000, 65504, (32, 1, D)).astype(np.float16)).to(DEV)
    k = torch.from_numpy(rng.standard_normal((96, 1, D)).astype(np.float16)).to(DEV)
    one = torch.tensor([96], dtype=torch.int32, device=DEV)
    quota = torch.tensor([[[48, 48]]], dtype=torch.int32, device=DEV)
    dk.quantize_append(cache, one, k, v, torch.rand((96, 1), device=DEV), quota=quota, total_new=96, max_new=96)
    q, k, v = fused(rng, n, 4, 1)
    both(cache, [n], q, k, v, "large values, n %d" % n)


@pytest.mark.parametrize("new_len,want", [([5, 9, 200], [5, 9, 6]), ([1, 1, 4], [1, 1, 0]), ([40, 300, 300], [40, 300, 10])],
                         ids=str)
def test_lengths_past_the_rows_are_clamped(new_len, want):
    """Lengths that sum to more rows than there are: the rows that are there are those of the clamped
    lengths; nothing behind them, or behind the workspace, is written."""
    rng = np.random.default_rng(sum(new_len))
    cache = filled(dk, {}, 3, 2, [300, 40, 700], seed=2)
    rows = sum(want)
    q, k, v = fused(rng, rows, 8, 2)
    nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
    before = kept_tokens(cache)
    out = torch.full((rows + 5, 8, D), 7.0, dtype=torch.float16, device=DEV)
    lse = torch.full((rows + 5, 8), 7.0, device=DEV)
    score = torch.full((rows + 5, 2), 7.0, device=DEV)
    ws = []
    for op in (dk.OP_CHUNK_ATTENTION, dk.OP_CHUNK_SIGNIFICANCE):
        need = dk.workspace_size(op, cache.L, 3, 8, 2, rows)
        ws.append((torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device=DEV), need))
    print("case: lengths %s for %d rows" % (new_len, rows), flush=True)
    dk.chunk_attention(cache, nl, q, k, v, SCALE, out=out[:rows], lse=lse[:rows], max_new=max(new_len), ws=ws[0][0][:ws[0][1]])
    torch.cuda.synchronize()
    check_attention(cache, want, q, k, v, out[:rows], lse[:rows], "clamped")
    dk.chunk_significance(cache, nl, q, k, SCALE, lse[:rows], score=score[:rows], max_new=max(new_len),
                          ws=ws[1][0][:ws[1][1]])
    torch.cuda.synchronize()
    check_scores(cache, before, want, q, k, lse[:rows], score[:rows], "clamped")
    for t in (out, lse, score):
        assert bool((t[rows:] == 7.0).all())
    for w, need in ws:
        assert bool((w[need:] == 0x5A).all())


@pytest.mark.parametrize("G,n", [(4, 4), (4, 5), (4, 16), (4, 20), (4, 32), (4, 33), (8, 2), (8, 3), (8, 16), (8, 17),
                                 (1, 16), (1, 17), (1, 128), (1, 129)])
def test_both_sides_of_the_row_borders(G, n):
    """16, 17, 128 and 129 rows of a sequence and those around: every kernel and its number of row tiles."""
    rng = np.random.default_rng(10 * G + n)
    cache = filled(dk, {}, 3, 1, [333, 0, 90], seed=n)
    q, k, v = fused(rng, 2 * n + 1, G, 1)
    both(cache, [n, 1, n], q, k, v, "G %d, n %d" % (G, n))


@pytest.mark.parametrize("layout", range(4))
@pytest.mark.parametrize("G", [1, 3, 4, 8])
def test_calls_of_many_rows(layout, G):
    """More rows than the few-row kernel takes altogether: tiles and shares, beside short chunks."""
    rng = np.random.default_rng(200 * layout + G)
    lens, new_len = [0, 333, 130, 64, 17], [1100 if G == 1 else 330, 1, 0, 140, 17]
    assert sum(new_len) * 2 * G > 2048
    cache = filled(dk, LAYOUTS[layout], 5, 2, lens, seed=layout)
    q, k, v = fused(rng, sum(new_len), 2 * G, 2)
    both(cache, new_len, q, k, v, "many rows, layout %d, G %d" % (layout, G))


@pytest.mark.parametrize("form", [dict(cap=20.0), dict(window=45), dict(slopes=True), dict(cap=5.0, window=130, slopes=True)],
                         ids=str)
def test_score_forms_of_many_rows(form):
    rng = np.random.default_rng(5)
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = (2.0 ** -np.arange(1, 7)).astype(np.float32)
    cache = filled(dk, {}, 3, 2, [700, 0, 90], seed=9)
    q, k, v = fused(rng, 401, 6, 2, kscale=2.0)
    both(cache, [200, 1, 200], q, k, v, "many rows, form %s" % form, **form)


@pytest.mark.parametrize("rows", [256, 257])
def test_both_sides_of_the_border_of_all_rows(rows):
    rng = np.random.default_rng(rows)
    cache = filled(dk, {}, 1, 1, [900], seed=rows)
    q, k, v = fused(rng, rows, 8, 1)
    both(cache, [rows], q, k, v, "%d tokens" % rows)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_lost_pages_and_non_finite_values_of_many_rows(bad):
    rng = np.random.default_rng(3)
    n, at = 300, 77
    cache = filled(dk, {}, 2, 1, [400, 50], seed=8)
    cache.page_table[0, 1] = -1
    cache.page_table[0, cache.L.p_max - 2] = 2 ** 31 - 1
    q, k, v = (x.contiguous() for x in fused(rng, 2 * n, 4, 1))
    nl = torch.tensor([n, n], dtype=torch.int32, device=DEV)
    want, want_lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=n)
    torch.cuda.synchronize()
    check_attention(cache, [n, n], q, k, v, want, want_lse, "lost pages")
    v[at, 0, 77] = bad
    k[n + at, 0, 5] = float("nan")
    out, lse = dk.chunk_attention(cache, nl, q, k, v, SCALE, max_new=n)
    torch.cuda.synchronize()
    assert torch.equal(out[:at], want[:at]) and torch.equal(lse[:n], want_lse[:n])
    assert not torch.isfinite(out[at:n, :, 77]).any()
    others = torch.arange(D, device=DEV) != 77
    assert torch.equal(out[at:n][..., others], want[at:n][..., others])
    assert torch.equal(out[n:n + at], want[n:n + at]) and torch.isnan(out[n + at:]).all()
    assert torch.isnan(lse[n + at:]).all()


def test_many_rows_captured_and_repeated():
    """Tiles in equal shares, replayed: bit-equal every time."""
    rng = np.random.default_rng(61)
    new_len = [300, 1, 25]
    cache = filled(dk, {}, 3, 2, [900, 40, 333], seed=5)
    q, k, v = fused(rng, sum(new_len), 8, 2)
    nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
    out = torch.empty((sum(new_len), 8, D), dtype=torch.float16, device=DEV)
    lse = torch.empty((sum(new_len), 8), device=DEV)
    ws = torch.empty(dk.workspace_size(dk.OP_CHUNK_ATTENTION, cache.L, 3, 8, 2, sum(new_len)), dtype=torch.uint8, device=DEV)
    call = lambda: dk.chunk_attention(cache, nl, q, k, v, SCALE, out=out, lse=lse, max_new=300, ws=ws)
    call()
    torch.cuda.synchronize()
    want = out.clone(), lse.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(4):
        for f in (g.replay, call):
            out.fill_(0.0)
            f()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
