"""Chunk operators where a cache, a batch or its values are out of the ordinary: lengths past a table's row,
padded batches, values that are not finite, scores far apart.  Definitions and tolerances are those of
test_gpu_chunk.py unless a test derives its own."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

from chunk_ref import D, filled, kept_tokens, logits, score_at, softmax  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402
from test_gpu_chunk import DEV, H16, LAYOUTS, SCALE, check_attention, check_scores, delta, fused  # noqa: E402

# Chunks that reach every kernel with eight query heads on two KV heads: single tokens (blocks of one row tile,
# short scores), a few (two row tiles), tens (scores of long chunks), and more rows than the few-row kernel takes
CHUNKS = [[1, 1, 1], [6, 1, 4], [30, 2, 9], [300, 2, 40]]


def run(cache, new_len, q, k, v, rows=None, max_new=None, **form):
    """Attention, then scores; rows beyond the lengths' sum hold 7."""
    rows = q.shape[0] if rows is None else rows
    max_new = max(new_len) if max_new is None else max_new
    nl = torch.tensor(new_len, dtype=torch.int32, device=DEV)
    out = torch.full((rows, q.shape[1], D), 7.0, dtype=torch.float16, device=DEV)
    lse = torch.full((rows, q.shape[1]), 7.0, device=DEV)
    score = torch.full((rows, k.shape[1]), 7.0, device=DEV)
    dk.chunk_attention(cache, nl, q, k, v, SCALE, out=out, lse=lse, max_new=max_new, **form)
    torch.cuda.synchronize()
    dk.chunk_significance(cache, nl, q, k, SCALE, lse, score=score, max_new=max_new, **form)
    torch.cuda.synchronize()
    return out, lse, score


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("layout", [0, 3])
@pytest.mark.parametrize("new_len", CHUNKS, ids=str)
def test_lengths_past_the_table_stay_in_its_row(layout, new_len):
    """Section lengths of more pages than the row has slots, or below zero: the high section ends with the row,
    the low one where the high one begins.  Everything is as with those lengths, byte for byte; the
    neighbouring tables' page IDs are neither read nor their scores moved a second time."""
    rng = np.random.default_rng(layout)
    cache = filled(dk, LAYOUTS[layout], 3, 2, [300, 70, 200], seed=layout)
    P, Tl = cache.L.p_max, cache.L.tokens_per_page[1]
    assert Tl == (16 if layout == 3 else 32)
    q, k, v = fused(rng, sum(new_len), 8, 2)
    lens, pool = cache.len.clone(), cache.pool.clone()
    for t, hi, lo in ((2, 16 * 5000, 0), (1, 0, 2 ** 31 - 1), (3, 50, 40000), (4, 2 ** 31 - 1, 2 ** 31 - 1), (0, -5, -70)):
        bounded = (min(max(hi, 0), P * 16), min(max(lo, 0), max(P - -(-max(hi, 0) // 16), 0) * Tl))
        print("case: layout %d, %s, table %d of lengths %d, %d" % (layout, new_len, t, hi, lo), flush=True)
        got = []
        for pair in (bounded, (hi, lo)):
            cache.len.copy_(lens)
            cache.len[t] = torch.tensor(pair, dtype=torch.int32, device=DEV)
            cache.pool.copy_(pool)
            got.append(run(cache, new_len, q, k, v) + (cache.pool.clone(),))
        assert same(*got)


@pytest.mark.parametrize("new_len", [[1, 0, 1], [0, 1, 0], [0] * 40 + [1] * 60 + [0, 1] * 20, [0, 1, 1] * 500], ids=len)
def test_single_tokens_of_a_padded_batch(new_len):
    """As many rows as sequences, one token at most each, but some sequences have none: every token goes with its
    own sequence's cache, rows that no sequence owns stay as they were, and so do the scores of sequences without
    new tokens.  (few tables, tables found by a workgroup's scan, tables that are not split)"""
    rng = np.random.default_rng(len(new_len))
    B, n = len(new_len), sum(new_len)
    lens = rng.integers(0, 120, B)
    cache = filled(dk, {}, B, 1, lens, seed=B, max_len=256)
    q, k, v = fused(rng, B, 4, 1)
    print("case: a padded batch of %d" % B, flush=True)
    before = kept_tokens(cache)
    out, lse, score = run(cache, new_len, q, k, v)
    check_attention(cache, new_len, q[:n], k[:n], v[:n], out[:n], lse[:n], "padded")
    check_scores(cache, before, new_len, q[:n], k[:n], lse[:n], score[:n], "padded")
    for x in (out, lse, score):
        assert bool((x[n:] == 7.0).all())


@pytest.mark.parametrize("Hq", [16, 6])
@pytest.mark.parametrize("max_new,new_len", [(100, [100, 1]), (300, [300, 1]), (300, [2, 16, 0, 300, 17]), (300, [0, 3]),
                                             (300, [3]), (300, [90]), (16, [16, 3, 0])], ids=str)
def test_rows_padded_to_the_longest_chunk(max_new, new_len, Hq):
    """As many rows as sequences times the longest chunk, with shorter and empty chunks among them: the short
    ones' outputs and scores are there, rows that no sequence owns stay as they were."""
    rng = np.random.default_rng(len(new_len))
    B, n = len(new_len), sum(new_len)
    cache = filled(dk, {}, B, 2, [300, 70, 0, 150, 40][:B], seed=B)
    q, k, v = fused(rng, B * max_new, Hq, 2)
    print("case: %s padded to %d" % (new_len, max_new), flush=True)
    before = kept_tokens(cache)
    out, lse, score = run(cache, new_len, q, k, v, max_new=max_new)
    check_attention(cache, new_len, q[:n], k[:n], v[:n], out[:n], lse[:n], "padded")
    check_scores(cache, before, new_len, q[:n], k[:n], lse[:n], score[:n], "padded")
    for x in (out, lse, score):
        assert bool((x[n:] == 7.0).all())


def cache_of(layout, keys, values, high, scores=None, max_len=None):
    """One table that holds the given tokens' keys and values [n, D], the `high` of the largest scores high."""
    n = len(keys)
    cache = dk.Cache(dk.layout(max_seq_len=max_len or n + 512, **layout), 2 * (n // 16 + 4), 1, 1, device=DEV)
    to = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).to(DEV)
    score = np.random.default_rng(n).random((n, 1)) if scores is None else np.asarray(scores)[:, None]
    dk.quantize_append(cache, to([n], np.int32), to(keys[:, None], np.float16), to(values[:, None], np.float16),
                       to(score, np.float32), quota=to([[[high, n - high]]], np.int32), total_new=n, max_new=n)
    torch.cuda.synchronize()
    assert int(cache.status.cpu()[0]) == 0 and cache.len.cpu().tolist() == [[high, n - high]]
    return cache


def attention_bounds(cache, new_len, q, k, v, small, **form):
    """Per (sequence, KV head): rows, expected outputs, and bounds where a weight's error is at most `small` of its
    row's largest weight besides its relative error (half a step of fp16) and the values' (the same)."""
    kept, G = kept_tokens(cache), q.shape[1] // cache.num_kv_heads
    vv = v.cpu().numpy().astype(np.float64)
    for b, h, row, n, x, size in logits(cache, kept, new_len, q, k, SCALE, **form):
        vals = np.concatenate([kept[b * cache.num_kv_heads + h][1], vv[row:row + n, h]])
        p, _ = softmax(x)
        want, A = p @ vals, p @ np.abs(vals)
        tol = H16 * (2 * A + np.abs(want)) + 2 * delta(size)[..., None] * A + 2.0 ** -25
        tol += small * p.max(-1)[..., None] * np.abs(vals).sum(0)
        yield slice(row, row + n), slice(h * G, (h + 1) * G), want, tol


@pytest.mark.parametrize("n,G", [(1, 4), (6, 4), (300, 8)])
def test_many_small_weights_count(n, G):
    """Tokens 2^-26.5 of their row's largest each, and fifteen of them for each large one, carry all of the value.
    A weight is at most 2^-25 / 2^7 of its row's largest off (it is an fp16 number, 2^7 for the running max,
    which a row's largest passes by at most 2^8)."""
    rng = np.random.default_rng(n)
    keys, values = np.zeros((2048, D)), np.full((2048, D), 1000.0)
    keys[::16, 3] = 26.5 * np.log(2) / SCALE / 8.0
    values[::16] = 0.0
    cache = cache_of({}, keys, values, 900)
    q, k, v = (torch.zeros((n, heads, D), dtype=torch.float16, device=DEV) for heads in (G, 1, 1))
    q[:, :, 3] = 8.0
    v.fill_(1000.0)
    print("case: small weights, n %d" % n, flush=True)
    out = run(cache, [n], q, k, v)[0].cpu().numpy().astype(np.float64)
    for rows, heads, want, tol in attention_bounds(cache, [n], q, k, v, 2.0 ** -32):
        assert want.min() > 1e-4 and tol.max() < 0.1 * want.min()
        assert (np.abs(out[rows, heads].transpose(1, 0, 2) - want) <= tol).all()


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("n,G", [(2, 4), (4, 4), (30, 4), (300, 8)])
def test_weights_enter_whole(n, G, own):
    """Two tokens of nearly the same weight and opposite values, and nothing else that counts: what is left of them
    shows their weights' error.  Values are whole in fp16, weights 2^-22 off at most (two parts), products and
    sums of fp32 far below 2^-20 of the two; with each weight rounded once it would be 2^-12."""
    print("case: whole weights, n %d, own %s" % (n, own), flush=True)
    a, b = 1.0, 0.94
    if own:  # the chunk's first two tokens, over an empty cache; the others' logits are 200 below
        cache = filled(dk, {}, 1, 1, [0], seed=1)
    else:    # one kept high, one low
        cache = cache_of({}, np.array([[a], [b]]) * (np.arange(D) == 3), np.array([[1.0], [-1.0]]) * np.ones(D), 1, [2.0, 1.0])
    q, k, v = (torch.zeros((n, heads, D), dtype=torch.float16, device=DEV) for heads in (G, 1, 1))
    q[:, :, 3] = torch.linspace(4.0, 12.0, n * G, device=DEV).reshape(n, G).half()
    k[:, :, 3] = -6000.0
    v.fill_(1.0)
    if own:
        k[0, 0, 3], k[1, 0, 3] = a, b
        v[1] = -1.0
    out, lse, _ = run(cache, [n], q, k, v)
    got = out.cpu().numpy().astype(np.float64)
    for b, h, row, _, x, size in logits(cache, kept_tokens(cache), [n], q, k, SCALE):
        vals = np.concatenate([kept_tokens(cache)[0][1], v[:, 0].cpu().numpy().astype(np.float64)])
        p, _ = softmax(x)
        want = p @ vals
        # (the others have no weight, and their logits no part in the error)
        d = 64 * 2.0 ** -24 * np.where(p > 0, size, 0.0).max(-1) + 2.0 ** -20
        tol = H16 * np.abs(want) + (2 * d + 2.0 ** -20)[..., None] + 2.0 ** -25
        first = 1 if own else 0  # (from the row that sees both)
        assert (p[:, first:] > 1e-30).sum(-1).max() == 2 and tol[:, first:].max() < 2.0 ** -14
        assert (np.abs(got.transpose(1, 0, 2) - want) <= tol)[:, first:].all()


def poke(cache, t, sec, u, group, pair, section="vmeta"):
    """{s, z} of token u of a section of table t, as fp16."""
    L = cache.L
    T = L.tokens_per_page[sec]
    page = int(cache.page_table[t, u // T if sec == 0 else L.p_max - 1 - u // T])
    at = L.off_vmeta[sec] + (group * T + u % T) * 4 if section == "vmeta" else L.off_kmeta[sec] + (u % T * 4 + group) * 4
    raw = torch.tensor(pair, dtype=torch.float16).view(torch.uint8).to(DEV)
    cache.pool[page, at:at + 4] = raw


NOT_FINITE = [(float("inf"), 0.5), (float("nan"), 0.5), (0.25, float("inf")), (0.25, float("-inf")), (0.25, float("nan"))]


@pytest.mark.parametrize("window", [0, 150, 330], ids=lambda w: "window%d" % w)
@pytest.mark.parametrize("layout", range(4))
@pytest.mark.parametrize("new_len", CHUNKS, ids=str)
def test_cached_values_that_are_not_finite(layout, new_len, window):
    """Cached groups whose scale or zero is infinite or NaN: the rows that see such a token are not finite in that
    group's dims, all other rows and dims are as ever."""
    rng = np.random.default_rng(10 * layout + len(new_len))
    cache = filled(dk, LAYOUTS[layout], 3, 2, [300, 70, 200], seed=layout)
    lens = cache.len.cpu().numpy()
    for i, pair in enumerate(NOT_FINITE):
        for t in (0, 1, 5):
            sec = int(rng.integers(2))
            poke(cache, t, sec, int(rng.integers(lens[t, sec])), (i + t) % 4, pair)
    q, k, v = fused(rng, sum(new_len), 8, 2)
    form = dict(window=window) if window else {}
    print("case: not finite, layout %d, %s, window %d" % (layout, new_len, window), flush=True)
    with np.errstate(invalid="ignore"):
        kept = kept_tokens(cache)
    out, lse, _ = run(cache, new_len, q, k, v, **form)
    got, got_lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    vv = v.cpu().numpy().astype(np.float64)
    mixed = False  # whether some rows see such a token and others do not
    for b, h, row, n, x, size in logits(cache, kept, new_len, q, k, SCALE, **form):
        vals = np.concatenate([kept[b * 2 + h][1], vv[row:row + n, h]])
        p, want_lse = softmax(x)
        lost = (np.isfinite(x).astype(float) @ ~np.isfinite(vals)) > 0
        mixed |= bool((lost.any((0, 1)) & ~lost.all((0, 1))).any())
        vals = np.where(np.isfinite(vals), vals, 0.0)
        want, A = p @ vals, p @ np.abs(vals)
        tol = H16 * (2 * A + np.abs(want)) + 2 * delta(size)[..., None] * A + vals.shape[0] * 2.0 ** -25 * np.abs(vals).max()
        g = got[row:row + n, h * 4:(h + 1) * 4].transpose(1, 0, 2)
        assert np.array_equal(np.isfinite(g), ~lost)
        assert (np.abs(g - want) <= tol)[~lost].all()
        assert (np.abs(got_lse[row:row + n, h * 4:(h + 1) * 4].T - want_lse) <= delta(size) + 2.0 ** -22 * np.abs(want_lse)).all()
    assert mixed or not window or new_len[0] < 300


@pytest.mark.parametrize("n", [1, 6, 300])
def test_an_infinite_value_appended(n):
    """An overflowed value at the append: its group is not finite here and in diffkv_decode_attention alike."""
    rng = np.random.default_rng(n)
    keys, values = rng.standard_normal((2, 200, D))
    values[20, 40] = np.inf
    values[150, 70] = -np.inf
    values[151, 100:103] = np.nan
    with np.errstate(invalid="ignore"):
        cache = cache_of({}, keys, values, 90)
    q, k, v = (x.contiguous() for x in fused(rng, n, 8, 1))
    out, lse, _ = run(cache, [n], q, k, v)
    dec, _ = dk.decode_attention(cache, q[:1].contiguous(), SCALE)
    torch.cuda.synchronize()
    dims = ~torch.isfinite(dec[0])
    assert dims.any() and not dims.all() and torch.isfinite(lse).all()
    assert torch.equal(~torch.isfinite(out), dims[:1].expand(8, -1)[None].expand(n, -1, -1))


@pytest.mark.parametrize("form", [{}, dict(window=100), dict(cap=10.0)], ids=str)
@pytest.mark.parametrize("new_len", CHUNKS, ids=str)
def test_what_lies_behind_a_section_reaches_nothing(new_len, form):
    """Slots of a page behind its section's end full of bits that are no numbers: the results are those of clean
    pages, bit for bit."""
    rng = np.random.default_rng(5)
    cache = filled(dk, {}, 3, 2, [301, 70, 203], seed=3)
    L, lens = cache.L, cache.len.cpu().numpy()
    q, k, v = fused(rng, sum(new_len), 8, 2)
    pool = cache.pool.clone()
    want = run(cache, new_len, q, k, v, **form)
    behind = pool.clone()
    for t in range(6):
        for sec in (0, 1):
            T, n = L.tokens_per_page[sec], int(lens[t, sec])
            if n % T == 0:
                continue
            page = int(cache.page_table[t, n // T if sec == 0 else L.p_max - 1 - n // T])
            for off, groups in ((L.off_kmeta[sec], None), (L.off_vmeta[sec], 4)):
                meta = behind[page, off:off + 16 * T]
                if groups:
                    meta.view(4, T, 4)[:, n % T:] = 0xFF
                else:
                    meta.view(T, 16)[n % T:] = 0xFF
    cache.pool.copy_(behind)
    print("case: behind the sections, %s, %s" % (new_len, form), flush=True)
    assert same(run(cache, new_len, q, k, v, **form), want)


@pytest.mark.parametrize("form", [{}, dict(window=1000)], ids=str)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("n", [1, 6, 300])
def test_scores_at_the_end_of_their_range(n, sign, form):
    """Scores of 4.1e6 in magnitude, all alike: a mean of the values seen."""
    cache = filled(dk, {}, 1, 1, [0], seed=1)
    q, k, v = (torch.zeros((n, heads, D), dtype=torch.float16, device=DEV) for heads in (8, 1, 1))
    rng = np.random.default_rng(n)
    q[:, :, 3], k[:, :, 3] = 1.0, sign * 62.5
    v.copy_(torch.from_numpy(rng.standard_normal((n, 1, D)).astype(np.float16)))
    nl = torch.tensor([n], dtype=torch.int32, device=DEV)
    print("case: large scores, n %d, sign %g, %s" % (n, sign, form), flush=True)
    out, lse = dk.chunk_attention(cache, nl, q, k, v, 65536.0, max_new=n, **form)
    torch.cuda.synchronize()
    vals = v[:, 0].cpu().numpy().astype(np.float64)
    count = np.arange(1, n + 1)[:, None]
    want, A = np.cumsum(vals, 0) / count, np.cumsum(np.abs(vals), 0) / count
    tol = (H16 * np.abs(want) + 2.0 ** -20 * A + 2.0 ** -25)[:, None]
    assert (np.abs(out.cpu().numpy().astype(np.float64) - want[:, None]) <= tol).all()
    x = sign * 62.5 * 65536.0
    assert np.allclose(lse.cpu().numpy(), x, rtol=2.0 ** -18, atol=0)


def test_host_tensors_beside_device_ones_are_refused():
    cache = filled(dk, {}, 1, 1, [50], seed=1)
    q, k, v = fused(np.random.default_rng(1), 3, 4, 1)
    nl = torch.tensor([3], dtype=torch.int32, device=DEV)
    pos = torch.arange(3, dtype=torch.int32, device=DEV)
    freq, _ = dk.rope_frequencies(128)
    for bad in ((pos, freq), (pos.cpu(), freq.to(DEV))):
        with pytest.raises(ValueError, match="GPU"):
            dk.rotate(cache.L, *bad, q, k)
    for bad in ((nl.cpu(), v, None), (nl, v.cpu(), None), (nl, v, torch.zeros(4))):
        with pytest.raises(ValueError, match="GPU"):
            dk.chunk_attention(cache, bad[0], q, k, bad[1], SCALE, max_new=3, slopes=bad[2])
    with pytest.raises(ValueError, match="GPU"):
        dk.chunk_significance(cache, nl, q, k, SCALE, torch.zeros((3, 4)), max_new=3)


@pytest.mark.parametrize("form", [{}, dict(window=200)], ids=str)
@pytest.mark.parametrize("n", [6, 60, 300])
def test_scores_beside_nan_count_the_other_rows(n, form):
    """A NaN key of the chunk's own, a NaN query: the rows that meet them have no part in any score."""
    rng = np.random.default_rng(n)
    cache = filled(dk, {}, 1, 1, [250], seed=8)
    q, k, v = (x.contiguous() for x in fused(rng, n, 8, 1))
    q[1, 3, 50] = float("nan")
    k[n // 2, 0, 5] = float("nan")
    print("case: scores beside NaN, n %d, %s" % (n, form), flush=True)
    before = kept_tokens(cache)
    _, lse, score = run(cache, [n], q, k, v, **form)
    norm = lse.cpu().numpy().astype(np.float64)
    pos, old, where = before[0][2:]
    for b, h, row, _, x, size in logits(cache, before, [n], q, k, SCALE, **form):
        rel = 2 * delta(np.nan_to_num(size)).max() + 2.0 ** -20
        P = np.nan_to_num(np.exp(x - norm.T[..., None])).max(0)
        assert np.isnan(norm[n // 2:]).any() and np.isfinite(norm[0]).all()
        X, m = P.sum(0), len(pos)
        left = cache.seq_len.cpu().numpy()[0] + n - pos
        got, want = score_at(cache, where), old + (X[:m] - n * old) / left
        assert (np.abs(got - want) <= rel * (np.abs(old) * (1 + n / left) + X[:m] / left) + 1e-30).all()
        got, want = score.cpu().numpy().astype(np.float64)[:, 0], X[m:] / np.arange(n, 0, -1)
        assert (np.abs(got - want) <= rel * want + 1e-30).all()


@pytest.mark.parametrize("B,Hkv,Hq,most", [(140, 8, 32, 20), (130, 8, 8, 128), (1100, 1, 8, 9)])
def test_many_tables_of_several_blocks(B, Hkv, Hq, most):
    """Over 1024 tables, so none is split, with up to eight row blocks each; empty chunks and padded rows among them."""
    rng = np.random.default_rng(B)
    new_len = rng.integers(0, most + 1, B)
    new_len[rng.integers(0, B, B // 3)] = 0
    new_len[B // 2] = most
    new_len, n = new_len.tolist(), int(new_len.sum())
    cache = filled(dk, {}, B, Hkv, rng.integers(0, 60, B), seed=B, max_len=256)
    q, k, v = fused(rng, n + 5, Hq, Hkv)
    print("case: %d tables, %d rows" % (B * Hkv, n), flush=True)
    before = kept_tokens(cache)
    out, lse, score = run(cache, new_len, q, k, v)
    check_attention(cache, new_len, q[:n], k[:n], v[:n], out[:n], lse[:n], "many tables")
    check_scores(cache, before, new_len, q[:n], k[:n], lse[:n], score[:n], "many tables")
    for x in (out, lse, score):
        assert bool((x[n:] == 7.0).all())


@pytest.mark.parametrize("new_len", [[1, 1, 1], [3, 0, 9], [70, 1, 2]], ids=str)
def test_a_longest_chunk_that_is_none(new_len):
    """A program that captured its step for longer chunks than the batch now has: the results are those of the call
    with the chunks' own length."""
    rng = np.random.default_rng(sum(new_len))
    cache = filled(dk, {}, 3, 2, [300, 70, 200], seed=5)
    n = sum(new_len)
    q, k, v = fused(rng, 600, 8, 2)
    before, pool = kept_tokens(cache), cache.pool.clone()
    for max_new in (max(new_len), 128, 200, 600):
        cache.pool.copy_(pool)
        print("case: %s of at most %d" % (new_len, max_new), flush=True)
        out, lse, score = run(cache, new_len, q, k, v, max_new=max_new)
        check_attention(cache, new_len, q[:n], k[:n], v[:n], out[:n], lse[:n], "at most %d" % max_new)
        check_scores(cache, before, new_len, q[:n], k[:n], lse[:n], score[:n], "at most %d" % max_new)
        for x in (out, lse, score):
            assert bool((x[n:] == 7.0).all())
