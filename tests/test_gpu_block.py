"""The uniform 8-bit cache: what is stored (exactly), reading back, attention over it against 64-bit definitions.

Tolerances of attention, from the arithmetic.  A score is an fp32 sum of exact products (codes times halfs) times fp32
scales: its error is at most a few dozen roundings of its terms' magnitudes, delta = 64 * 2^-24 * size + 2^-20 (a score of
a form as well: a bias enters by one rounding, a sixteenth of those dozens).
  out  weights in two fp16 parts (2^-22; the second's last step 2^-32 of the row's largest weight, which the value
       scale weighs), sums in fp32 over keys / 32 products and their joins, one rounding to fp16:
       |err| <= 2^-11 |out| + (2 delta + 2^-20 + keys 2^-28) A + keys 2^-31 V max(1, V) + 2^-25, A = sum p |v|, V = max |v|
       (the last step's part: a smaller one, 2^-37, where the weights' reference is twelve below the largest);
  lse  delta + 2^-22 |lse|.
"""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("needs a GPU", allow_module_level=True)

import block_ref as ref  # noqa: E402
from block_ref import D, T  # noqa: E402
from paper_2412_03131_amd import diffkv as dk  # noqa: E402

DEV = "cuda"
SCALE = 1.0 / np.sqrt(128.0)
E4M3, INT8 = dk.BLOCK_E4M3, dk.BLOCK_INT8


def halves(rng, *shape, size=1.0):
    return (rng.standard_normal(shape) * size).astype(np.float16)


def keys_of(rng, rows, H):
    k = rng.standard_normal((rows, H, D))
    k[:, :, [3, 40, 77, 120]] *= 10.0
    return k.astype(np.float16)


def to(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def plain_of(rng, lens, H, fmt):
    p = ref.Plain(len(lens), H, fmt)
    p.append(lens, keys_of(rng, sum(lens), H), halves(rng, sum(lens), H, D))
    return p


def same_cache(c, plain, what, untouched=None):
    """Every whole block that has an ID and every tail row, exactly; blocks without one as they were."""
    pool, scale, tail, table = (t.cpu().numpy() for t in (c.pool, c.scale, c.tail, c.table))
    owned = set()
    for b, (rows, _) in enumerate(plain.rows):
        n = len(rows)
        for i in range(n // T):
            p = int(table[b, i])
            if not 0 <= p < c.num_blocks:
                continue
            owned.add(p)
            for h in range(c.num_kv_heads):
                for side in (0, 1):
                    codes, s = plain.block(b, i, h, side)
                    got = ref.numbers(pool[p, h, side], plain.fmt)[ref.AT[side]]
                    assert np.array_equal(got, codes), "%s: codes of %d/%d/%d/%d" % (what, b, i, h, side)
                    assert np.array_equal(np.float32(s), scale[p, h, side], equal_nan=True), (what, b, i, h, side)
        rest = n % T
        for side in (0, 1):
            want = plain.rows[b][side][n - rest:].transpose(1, 0, 2)
            assert np.array_equal(tail[b, :, side, :rest].view(np.int16), want.view(np.int16)), "%s: tail of %d" % (what, b)
    if untouched is not None:
        others = [p for p in range(c.num_blocks) if p not in owned]
        assert np.array_equal(pool[others], untouched[0][others]) and np.array_equal(scale[others], untouched[1][others]), what


def new_cache(lens, H, fmt, max_len=None, spare=2):
    """An empty cache with blocks assigned for lens[b] tokens."""
    B = len(lens)
    L = dk.layout(max_seq_len=max_len or max(max(lens), 1))
    need = [n // T for n in lens]
    c = dk.BlockCache(L, sum(need) + spare, B, H, fmt=fmt, device=DEV)
    ids = np.random.default_rng(5).permutation(c.num_blocks)
    table = np.full(c.table.shape, -1, np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = ids[at:at + n]
        at += n
    c.table.copy_(to(table))
    c.pool.fill_(7)
    c.tail.fill_(float("nan"))
    return c


# ---- append --------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("calls", [
    [[0, 1, 31, 32, 33, 64, 100]], [[5, 0, 40, 31, 1, 32, 63], [27, 1, 24, 2, 31, 64, 1], [1, 70, 0, 96, 33, 5, 200]],
    [[1] * 7] * 34, [[700, 0, 0, 0, 0, 0, 3]]], ids=["once", "thrice", "singles", "long"])
def test_append(fmt, calls):
    print("case: append fmt %d, %d calls" % (fmt, len(calls)), flush=True)
    rng = np.random.default_rng(len(calls))
    B, H = 7, 3
    total = np.array(calls).sum(0).tolist()
    c = new_cache(total, H, fmt)
    before = c.pool.cpu().numpy(), c.scale.cpu().numpy()
    plain = ref.Plain(B, H, fmt)
    for new in calls:
        x = to(np.concatenate([keys_of(rng, sum(new), H), halves(rng, sum(new), H, D)], 1))  # slices of one projection
        k, v = x[:, :H], x[:, H:]
        dk.block_append(c, ints(new), k, v, max_new=max(new))
        plain.append(new, k.cpu().numpy(), v.cpu().numpy())
        c.seq_len += ints(new)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    same_cache(c, plain, "append", before)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_append_values_at_the_borders(fmt):
    """Ties between codes, the largest and the smallest halfs, zeros, a block's largest at a border of its scale."""
    rng = np.random.default_rng(3)
    blocks = []
    n = np.arange(-127, 127) + 0.5
    for s in (2.0 ** -3, 1.0, 1.5, 129 / 128, 255 / 128, 2.0 ** -20):
        x = np.zeros((T, D))
        flat = x.reshape(-1)
        flat[:254] = n * s
        flat[254] = 127 * s
        flat[300:2300] = rng.uniform(-127, 127, 2000) * s
        blocks.append(x)
    for top in (65504.0, 2.0 ** -24, 448.0, 448.5, 449.0, 2.0 ** -14, 2.0 ** -10 * 1.75, 1e-6):
        x = rng.uniform(-1, 1, (T, D)) * top
        x[4, 5] = -top
        x[7] *= 2.0 ** -9
        blocks.append(x)
    blocks.append(np.zeros((T, D)))
    blocks.append(-np.zeros((T, D)))
    # every half that e4m3 can meet below 448: ties to even among its normal and subnormal values
    x = (np.arange(T * D) % 448) + (np.arange(T * D) // 448) / 16
    x[0] = 448
    blocks.append(np.minimum(x, 448).reshape(T, D))
    x = (np.arange(T * D) - T * D / 2) * 2.0 ** -11
    x[0] = 448
    blocks.append(x.reshape(T, D))
    with np.errstate(over="ignore"):
        k = np.concatenate(blocks).astype(np.float16)[:, None]
    c = new_cache([len(k)], 1, fmt)
    plain = ref.Plain(1, 1, fmt)
    dk.block_append(c, ints([len(k)]), to(k), to(k[::-1].copy()), max_new=len(k))
    plain.append([len(k)], k, k[::-1])
    torch.cuda.synchronize()
    same_cache(c, plain, "borders")


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_append_values_that_are_not_finite(fmt, bad):
    rng = np.random.default_rng(4)
    k, v = halves(rng, 96, 2, D), halves(rng, 96, 2, D)
    k[40, 1, 99] = bad
    v[31, 0, 0] = bad
    c = new_cache([96], 2, fmt)
    plain = ref.Plain(1, 2, fmt)
    dk.block_append(c, ints([96]), to(k), to(v))
    plain.append([96], k, v)
    torch.cuda.synchronize()
    same_cache(c, plain, "not finite")
    assert torch.isnan(c.scale).sum() == 2


def test_append_drops_blocks_without_ids():
    rng = np.random.default_rng(6)
    lens = [100, 64, 300]
    c = new_cache(lens, 2, E4M3)
    c.table[0, 1], c.table[2, 0], c.table[2, 4], c.table[1, 1] = -1, -7, c.num_blocks, 2 ** 31 - 1
    before = c.pool.cpu().numpy(), c.scale.cpu().numpy()
    k, v = keys_of(rng, sum(lens), 2), halves(rng, sum(lens), 2, D)
    plain = ref.Plain(3, 2, E4M3)
    plain.append(lens, k, v)
    dk.block_append(c, ints(lens), to(k), to(v))
    torch.cuda.synchronize()
    assert int(c.status) == 0
    same_cache(c, plain, "dropped", before)


@pytest.mark.parametrize("new,most,seen,status", [
    ([40, 3, 40], 40, [0, 0, 0], dk.ST_BAD_INPUT),       # more rows than there are
    ([40, -1, 0], 40, [0, 0, 0], dk.ST_BAD_INPUT),
    ([40, 0, 1], 39, [0, 0, 0], dk.ST_BAD_INPUT),        # longer than max_new
    ([10, 0, 40], 40, [0, 0, 65], dk.ST_TABLE_OVERFLOW),  # past max_seq_len
    ([10, 10, 10], 40, [-1, 0, 5], dk.ST_TABLE_OVERFLOW),
    ([10, 10, 10], 40, [0, 2 ** 31 - 1, 5], dk.ST_TABLE_OVERFLOW)], ids=str)
def test_append_that_changes_nothing(new, most, seen, status):
    rng = np.random.default_rng(7)
    c = new_cache([96, 96, 96], 2, E4M3, max_len=104)
    c.seq_len.copy_(ints(seen))
    before = [t.clone() for t in c.tensors()]
    dk.block_append(c, ints(new), to(halves(rng, 60, 2, D)), to(halves(rng, 60, 2, D)), max_new=most)
    torch.cuda.synchronize()
    assert int(c.status) == status
    for t, u in list(zip(c.tensors(), before))[:-1]:
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))


def test_append_of_a_padded_batch_up_to_the_last_position():
    rng = np.random.default_rng(8)
    c = new_cache([96, 96], 1, INT8, max_len=96)
    plain = ref.Plain(2, 1, INT8)
    for new in ([50, 96], [46, 0]):
        k, v = halves(rng, 200, 1, D), halves(rng, 200, 1, D)
        dk.block_append(c, ints(new), to(k), to(v), max_new=200)
        plain.append(new, k, v)
        c.seq_len += ints(new)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    same_cache(c, plain, "padded")


def test_append_to_many_sequences():
    """More sequences than a wave's lanes, most of them idle."""
    rng = np.random.default_rng(9)
    new = [int(n) for n in rng.integers(0, 3, 1500)]
    new[777], new[1400] = 64, 33
    c = new_cache([n + 31 for n in new], 2, E4M3)
    plain = plain_of(rng, [30] * 1500, 2, E4M3)
    start = ref.filled(dk, plain, c.L.max_seq_len, DEV)
    c.tail.copy_(start.tail)
    c.seq_len.fill_(30)
    k, v = keys_of(rng, sum(new), 2), halves(rng, sum(new), 2, D)
    dk.block_append(c, ints(new), to(k), to(v))
    plain.append(new, k, v)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    same_cache(c, plain, "many sequences")


# ---- read ----------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_read(fmt):
    print("case: read fmt %d" % fmt, flush=True)
    rng = np.random.default_rng(10)
    lens = [0, 31, 32, 100, 256, 517]
    plain = plain_of(rng, lens, 3, fmt)
    plain.rows[3][1][40:50] *= np.float16(3e3)
    drop = {(4, 2), (5, 0)}
    c = ref.filled(dk, plain, 544, DEV, drop=drop)
    for start, count in (([0] * 6, lens), ([0, 5, 31, 64, 63, 500], [0, 26, 1, 33, 70, 17]),
                         ([-3, 30, 32, 90, 250, -1], [9, 5, 4, 200, 10, 1]), ([7, -2 ** 31, 2 ** 31 - 1, 99, 0, 515], [1] * 6)):
        total = sum(count)
        out = torch.full((total + 5, 8, D), 123.0, dtype=torch.float16, device=DEV)  # wider rows, five that are nobody's
        dk.block_read(c, ints(start), ints(count), total + 5, k_out=out[:, 1:4], v_out=out[:, 4:7])
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        assert (got[:, [0, 7]] == 123).all() and (got[total:] == 123).all()
        row = 0
        for b in range(6):
            for h in range(3):
                for side in (0, 1):
                    x, _ = plain.read(b, h, side, lambda i: (b, i) not in drop)
                    pos = np.arange(count[b], dtype=np.int64) + start[b]
                    inside = (pos >= 0) & (pos < lens[b])
                    want = np.zeros((count[b], D))
                    want[inside] = x[pos[inside]]
                    want = np.clip(want, -65504, 65504).astype(np.float16)
                    assert np.array_equal(got[row:row + count[b], 1 + 3 * side + h], want), (start, b, h, side)
            row += count[b]


def test_read_of_the_largest_halfs():
    """A code times its scale can lie beyond the largest half."""
    k = np.full((32, 1, D), 65504, np.float16)
    k[1] = -k[1]
    c = new_cache([32], 1, E4M3)
    dk.block_append(c, ints([32]), to(k), to(k))
    c.seq_len.fill_(32)
    got, _ = dk.block_read(c, ints([0]), ints([32]), 32)
    assert torch.equal(got, to(k))


def test_read_clamps_counts():
    rng = np.random.default_rng(11)
    plain = plain_of(rng, [64, 64, 64], 1, INT8)
    c = ref.filled(dk, plain, 64, DEV)
    out = torch.zeros((40, 1, D), dtype=torch.float16, device=DEV)
    dk.block_read(c, ints([0, 8, 0]), ints([30, -5, 64]), 40, max_count=20, k_out=out, v_out=torch.zeros_like(out))
    torch.cuda.synchronize()
    want = [plain.read(b, 0, 0, lambda i: True)[0][:20].astype(np.float16) for b in (0, 2)]
    assert np.array_equal(out[:, 0].cpu().numpy(), np.concatenate(want))


# ---- attention -------------------------------------------------------------------------------


def check(plain, c, new, q, k, v, out, lse, what, drop=(), **form):
    got, got_lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    G = q.shape[1] // plain.H
    q, k, v = (x.cpu().numpy() for x in (q, k, v))
    for b, h, row, n, want, want_lse, A, size, keys, V in ref.attention(
            plain, new, q, k, v, SCALE, lambda b, i: (b, i) not in drop, **form):
        d = 64 * 2.0 ** -24 * size + 2.0 ** -20
        tol = 2.0 ** -11 * np.abs(want) + (2 * d[..., None] + 2.0 ** -20 + keys * 2.0 ** -28) * A + \
            keys * 2.0 ** -31 * V * max(1.0, V) + 2.0 ** -25
        g = got[row:row + n, h * G:(h + 1) * G].transpose(1, 0, 2)
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(g), fine), "%s b=%d h=%d: what is finite" % (what, b, h)
        bad = ~(np.abs(g - want) <= tol) & fine
        assert not bad.any(), "%s b=%d h=%d: %d wrong, first %s: %r, expected %r" % (
            what, b, h, bad.sum(), np.argwhere(bad)[0], g[bad][0], want[bad][0])
        gl = got_lse[row:row + n, h * G:(h + 1) * G].T
        bad = ~(np.abs(gl - want_lse) <= d + 2.0 ** -22 * np.abs(want_lse)) & np.isfinite(want_lse)
        assert not bad.any(), "%s b=%d h=%d lse: %d wrong: %r, expected %r" % (
            what, b, h, bad.sum(), gl[bad][0], want_lse[bad][0])


def rows_of(rng, rows, Hq, H, size=1.0):
    x = to(np.concatenate([halves(rng, rows, Hq, D, size=size), keys_of(rng, rows, H), halves(rng, rows, H, D)], 1))
    return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]


def attend(plain, new, G, what, seed=0, drop=(), size=1.0, max_len=None, **form):
    print("case:", what, flush=True)
    rng = np.random.default_rng(1000 + seed)
    H = plain.H
    c = ref.filled(dk, plain, max_len or max(len(r[0]) for r in plain.rows) + max(new), DEV, seed=seed, drop=drop)
    q, k, v = rows_of(rng, sum(new), H * G, H, size)
    args = dict(form)
    if form.get("slopes") is not None:
        args["slopes"] = torch.tensor(form["slopes"], dtype=torch.float32, device=DEV)
    before = [t.clone() for t in c.tensors()]
    out, lse = dk.block_attention(c, ints(new), q, k, v, SCALE, max_new=max(new), **args)
    torch.cuda.synchronize()
    check(plain, c, new, q, k, v, out, lse, what, drop, **form)
    for t, u in zip(c.tensors(), before):
        assert torch.equal(t.view(torch.uint8), u.view(torch.uint8))
    return c, q, k, v, out, lse


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("G", [1, 4, 7, 16, 33])
def test_ragged_chunks(fmt, G):
    """Chunks of none, one and several tokens over caches that are empty, all tail, all blocks."""
    rng = np.random.default_rng(G)
    lens, new = [0, 1, 37, 300, 129, 64, 31], [3, 1, 0, 40, 17, 1, 2]
    attend(plain_of(rng, lens, 2, fmt), new, G, "fmt %d, G %d" % (fmt, G), seed=G)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("G", [1, 2, 5, 8])
def test_single_tokens(fmt, G):
    rng = np.random.default_rng(G)
    attend(plain_of(rng, [0, 5, 16, 32, 700, 1500], 2, fmt), [1] * 6, G, "single tokens, G %d" % G, seed=G, size=3.0)


@pytest.mark.parametrize("form", [
    dict(window=1), dict(window=1, sinks=4), dict(window=45), dict(window=45, sinks=1), dict(window=64, sinks=33),
    dict(window=200, sinks=100), dict(window=10 ** 9, sinks=3), dict(window=33, sinks=10 ** 9), dict(sinks=5), dict(cap=20.0),
    dict(cap=5.0, window=130, sinks=2, slopes=True), dict(slopes=True), dict(window=2 ** 31 - 1, sinks=2 ** 31 - 1)], ids=str)
@pytest.mark.parametrize("n", [1, 6, 70, 300])
def test_forms(form, n):
    form = dict(form)
    if form.get("slopes"):
        form["slopes"] = (2.0 ** -np.arange(1, 7)).astype(np.float32)
    rng = np.random.default_rng(n)
    attend(plain_of(rng, [200, 0, 431, 96], 2, E4M3), [n, 1, n, n + 3], 3, "form %s, n %d" % (form, n), seed=n, **form)


@pytest.mark.parametrize("fmt", [E4M3, INT8])
@pytest.mark.parametrize("B,n,L,G", [(1, 1, 9000, 4), (1, 300, 2100, 8), (2, 513, 0, 4), (1, 700, 1000, 1), (3, 9, 3000, 7)])
def test_long(fmt, B, n, L, G):
    rng = np.random.default_rng(n)
    lens = [max(0, L - 37 * b) for b in range(B)]
    attend(plain_of(rng, lens, 1, fmt), [max(1, n - 3 * b) for b in range(B)], G, "long %d %d %d %d" % (B, n, L, G), seed=n)


@pytest.mark.parametrize("window,sinks", [(500, 4), (1000, 130), (64, 0)])
def test_long_windows(window, sinks):
    """Blocks that no row sees have no ID; those that some rows see are cut by both ends of the window."""
    rng = np.random.default_rng(window)
    lens, new = [3001, 1500, 777], [300, 1, 40]
    drop = {(b, i) for b, L in enumerate(lens) for i in range(L // T) if i * T + T <= L - window + 1 and i * T >= sinks}
    assert drop
    attend(plain_of(rng, lens, 1, INT8), new, 4, "windows %d %d" % (window, sinks), seed=window, drop=drop, window=window, sinks=sinks)


def test_blocks_that_are_not_there():
    rng = np.random.default_rng(12)
    drop = {(0, 0), (0, 3), (1, 0), (1, 1), (1, 2)}
    attend(plain_of(rng, [200, 96, 64], 2, E4M3), [5, 3, 40], 4, "missing blocks", drop=drop)


def test_many_sequences():
    rng = np.random.default_rng(13)
    lens = [int(n) for n in rng.integers(0, 90, 700)]
    new = [int(n) for n in rng.integers(0, 4, 700)]
    attend(plain_of(rng, lens, 1, E4M3), new, 4, "many sequences")


@pytest.mark.parametrize("B", [64, 65, 256, 257, 4096, 4097, 8300])
def test_numbers_of_sequences(B):
    """Both sides of the numbers of sequences that a wave reads at once, and keeps the starts of: attention, append, read."""
    rng = np.random.default_rng(27 + B)
    lens = [int(n) for n in rng.integers(0, 40, B)]
    new = [int(n) for n in (rng.random(B) < 0.4) * rng.integers(1, 4, B)]
    idle = min(128, B // 4)  # (in large calls a whole 64 of them)
    new[B // 3:B // 3 + idle] = [0] * idle
    new[B // 2], new[B - 1] = 70, 1
    plain = plain_of(rng, lens, 1, INT8)
    c, q, k, v, _, _ = attend(plain, new, 4, "%d sequences" % B)
    free = sorted(set(range(c.num_blocks)) - set(c.table.cpu().numpy().ravel().tolist()))
    table = c.table.cpu().numpy()
    for b in range(B):  # (blocks that the call fills and that find no ID are dropped)
        for i in range(lens[b] // T, (lens[b] + new[b]) // T):
            if free:
                table[b, i] = free.pop()
    c.table.copy_(to(table))
    dk.block_append(c, ints(new), k, v)
    plain.append(new, k.cpu().numpy(), v.cpu().numpy())
    c.seq_len += ints(new)
    same_cache(c, plain, "append to %d sequences" % B)
    start, count = [len(r[0]) // T * T for r in plain.rows], [len(r[0]) % T for r in plain.rows]
    kb, vb = dk.block_read(c, ints(start), ints(count), sum(count))
    torch.cuda.synchronize()
    assert int(c.status) == 0
    for side, x in enumerate((kb, vb)):
        want = np.concatenate([r[side][s:] for r, s in zip(plain.rows, start)])
        assert np.array_equal(x.cpu().numpy().view(np.int16), want.view(np.int16))


def test_one_long_among_single_tokens():
    rng = np.random.default_rng(14)
    new = [1] * 20
    new[7] = 260
    attend(plain_of(rng, [int(n) for n in rng.integers(100, 900, 20)], 2, E4M3), new, 4, "mixed")


def test_scales_of_all_sizes():
    """Blocks whose values differ by powers of two from each other, small keys beside large ones."""
    rng = np.random.default_rng(15)
    for fmt in (E4M3, INT8):
        plain = plain_of(rng, [512, 170], 1, fmt)
        for rows in plain.rows:
            for i in range(len(rows[0]) // T):
                rows[1][i * T:i * T + T] = rows[1][i * T:i * T + T].astype(np.float64) * 2.0 ** (int(rng.integers(-8, 6)))
                rows[0][i * T:i * T + T] = rows[0][i * T:i * T + T].astype(np.float64) * 2.0 ** (int(rng.integers(-6, 2)))
        attend(plain, [3, 20], 4, "scales, fmt %d" % fmt)
    zero = plain_of(rng, [96], 1, INT8)
    zero.rows[0][1][32:64] = 0
    zero.rows[0][0][:32] = 0
    attend(zero, [2], 2, "blocks of zeros")


def test_many_small_weights():
    """Tokens 2^-26.5 of the largest weight that carry all of the value."""
    plain = ref.Plain(1, 1, INT8)
    n = 4096
    k, v = np.zeros((n, 1, D), np.float16), np.zeros((n, 1, D), np.float16)
    v[:, :, 0] = 1.0
    k[:, :, 0] = -1.0
    plain.append([n], k, v)
    c = ref.filled(dk, plain, n + 1, DEV)
    q = torch.zeros((1, 1, D), dtype=torch.float16, device=DEV)
    q[:, :, 0] = 26.5 * np.log(2.0) / SCALE / 2
    own_k, own_v = torch.zeros((2, 1, 1, D), dtype=torch.float16, device=DEV)
    own_k[:, :, 0] = 1.0
    out, lse = dk.block_attention(c, ints([1]), q, own_k, own_v, SCALE)
    torch.cuda.synchronize()
    x = float(q[0, 0, 0]) * SCALE * 2
    want = plain.read(0, 0, 1, lambda i: True)[0][0, 0] * n * np.exp(-x) / (1 + n * np.exp(-x))
    # Rounding of the result: 2^-11, or as an fp16 denormal 2^-25.  A stored token's weight enters as u = p s 2^12 with its
    # value's scale s = 32 / 127 (the own token has the row's largest u, 2^12), whose second part is off by half an fp16
    # denormal's step, 2^-25, times a code of 127 / 32: n 2^-25 2^-12 4 = 2^-23 of the sum.
    assert abs(float(out[0, 0, 0]) - want) <= 2.0 ** -11 * want + 2.0 ** -25 + 2.0 ** -23


def test_weights_of_two_parts():
    """Two tokens of opposite values and nearly equal weights, stored and own: to 2^-20 of their sum."""
    for fmt, stored in ((INT8, True), (E4M3, True), (E4M3, False)):
        lens = 64 if stored else 1
        plain = ref.Plain(1, 1, fmt)
        k, v = np.zeros((lens, 1, D), np.float16), np.zeros((lens, 1, D), np.float16)
        k[:, :, 1] = -100.0 if stored else 0.0
        k[0, 0, 1] = 0.0
        v[0] = 1.0
        plain.append([lens], k, v)
        for eps in (2.0 ** -9, 3 * 2.0 ** -11, 2.0 ** -6):
            c = ref.filled(dk, plain, lens + 1, DEV)
            q = torch.zeros((1, 1, D), dtype=torch.float16, device=DEV)
            q[:, :, 0], q[:, :, 1] = 1.0, 64.0
            own_k, own_v = torch.zeros((1, 1, D), dtype=torch.float16, device=DEV), torch.full((1, 1, D), -1.0, dtype=torch.float16, device=DEV)
            own_k[:, :, 0] = eps
            out, _ = dk.block_attention(c, ints([1]), q, own_k, own_v, SCALE)
            x = eps * SCALE
            held = plain.read(0, 0, 1, lambda i: True)[0][0, 0]  # (1 as it is stored)
            want = (held - np.exp(x)) / (1 + np.exp(x))
            assert abs(float(out[0, 0, 0]) - want) <= 2.0 ** -20 + 2.0 ** -11 * abs(want), (fmt, stored, eps)


@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("n", [6, 200])
def test_values_that_are_not_finite(bad, n):
    """Own and tail values and keys reach the rows that see their token; a block's, those that see one of its tokens."""
    rng = np.random.default_rng(16)
    lens = [75, 64]
    for where in ("own v", "own k", "tail v", "block v", "block k"):
        plain = plain_of(rng, lens, 1, E4M3)
        c = ref.filled(dk, plain, 400, DEV)
        q, k, v = (x.clone() for x in rows_of(rng, 2 * n, 4, 1))
        win = 0
        if where == "own v":
            v[3, 0, 17] = bad
        elif where == "own k":
            k[3, 0, 17] = bad
        else:
            win = 8
            at = 70 if where[:4] == "tail" else 63
            side = 1 if where[-1] == "v" else 0
            if where[:4] == "tail":
                c.tail[0, 0, side, at % T, 17] = bad
            else:
                c.scale[int(c.table[0, at // T]), 0, side] = float("nan")
        out, lse = dk.block_attention(c, ints([n, n]), q, k, v, SCALE, window=win)
        out0, _ = dk.block_attention(ref.filled(dk, plain, 400, DEV), ints([n, n]), q.nan_to_num(0, 0, 0),
                                     k.nan_to_num(0, 0, 0), v.nan_to_num(0, 0, 0), SCALE, window=win)
        torch.cuda.synchronize()
        p = 75 + np.arange(n)
        if where[:3] == "own":
            hit = p >= 78
        elif where[:4] == "tail":
            hit = (p >= 70) & (p - 70 < win)
        else:
            hit = p - 63 < win  # the nearest of the block's tokens
        rows = ~torch.isfinite(out).all(-1).cpu().numpy()  # [2 n, heads]
        if where == "own k" or where[:5] == "block":
            # (an infinite key's score may be -inf: its token then has no weight)
            assert not rows[:n][~hit].any() and (bad is np.inf or rows[:n][hit].all()), where
        else:
            assert np.array_equal(rows[:n].any(1), hit) and np.array_equal(rows[:n].all(1), hit), where
            clean = ~(np.arange(D) == 17)
            assert torch.isfinite(out[..., torch.from_numpy(clean).to(DEV)]).all(), where
        assert not rows[n:].any(), where
        free = torch.from_numpy(~hit).to(DEV)
        assert torch.equal(out[:n][free], out0[:n][free]) and torch.equal(out[n:], out0[n:]), where


@pytest.mark.parametrize("n", [6, 200])
def test_queries_that_are_not_finite(n):
    """A NaN or infinite query is its own row's alone."""
    rng = np.random.default_rng(23)
    plain = plain_of(rng, [75, 64], 1, INT8)
    c = ref.filled(dk, plain, 400, DEV)
    q, k, v = (x.clone() for x in rows_of(rng, 2 * n, 4, 1))
    want, want_lse = dk.block_attention(c, ints([n, n]), q, k, v, SCALE)
    q[3, 1, 5], q[n + 1, 0, 9] = float("nan"), float("inf")
    out, lse = dk.block_attention(c, ints([n, n]), q, k, v, SCALE)
    torch.cuda.synchronize()
    hit = torch.zeros((2 * n, 4), dtype=torch.bool, device=DEV)
    hit[3, 1] = hit[n + 1, 0] = True
    assert torch.isnan(out[hit]).all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


def test_nothing_to_do_and_nothing_kept():
    """No rows, no blocks, a sequence's tail alone, no lse."""
    c = dk.BlockCache(dk.layout(max_seq_len=100), 0, 2, 1, device=DEV)
    rng = np.random.default_rng(25)
    plain = ref.Plain(2, 1, E4M3)
    q, k, v = rows_of(rng, 5, 2, 1)
    dk.block_append(c, ints([4, 1]), k, v)
    plain.append([4, 1], k.cpu().numpy(), v.cpu().numpy())
    c.seq_len += ints([4, 1])
    kb, vb = dk.block_read(c, ints([0, 0]), ints([4, 1]), 5)
    out, lse = dk.block_attention(c, ints([2, 3]), q, k, v, SCALE)
    alone, none = dk.block_attention(c, ints([2, 3]), q, k, v, SCALE, want_lse=False)
    torch.cuda.synchronize()
    assert torch.equal(kb, k) and torch.equal(vb, v) and none is None and torch.equal(alone, out)
    check(plain, c, [2, 3], q, k, v, out, lse, "tails")
    out, lse = dk.block_attention(c, ints([0, 0]), q[:0], k[:0], v[:0], SCALE)
    assert out.shape == (0, 2, D) and lse.shape == (0, 2)
    dk.block_append(c, ints([0, 0]), k, v)
    kb, _ = dk.block_read(c, ints([3, 0]), ints([0, 0]), 0)
    torch.cuda.synchronize()
    assert kb.shape == (0, 1, D) and int(c.status) == 0 and c.seq_len.tolist() == [4, 1]


def test_two_calls_at_once():
    """Attention on two streams, each with its own workspace, over one cache."""
    rng = np.random.default_rng(26)
    plain = plain_of(rng, [900, 300], 2, E4M3)
    c = ref.filled(dk, plain, 1200, DEV)
    rows = [rows_of(rng, 2 * n, 8, 2) for n in (1, 150)]
    want = [dk.block_attention(c, ints([n, n]), *x, SCALE) for n, x in zip((1, 150), rows)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in rows]
    lens = [ints([1, 1]), ints([150, 150])]
    sizes = [dk.workspace_size(dk.OP_BLOCK_ATTENTION, c.L, 2, 8, 2, len(x[0])) for x in rows]
    ws = [torch.zeros(s, dtype=torch.uint8, device=DEV) for s in sizes]
    got = [[], []]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            out, lse = torch.empty_like(want[i][0]), torch.empty_like(want[i][1])
            dk.block_attention(c, lens[i], *rows[i], SCALE, out=out, lse=lse, max_new=(1, 150)[i], ws=ws[i], stream=s)
            got[i].append((out, lse))
    torch.cuda.synchronize()
    for i in (0, 1):
        assert all(torch.equal(o, want[i][0]) and torch.equal(e, want[i][1]) for o, e in got[i])


@pytest.mark.parametrize("n", [2, 150])  # (few rows, many)
def test_addresses_past_32_bits(n):
    """Blocks behind 4 GiB of pool, rows 2^24 elements apart: as near ones, bit for bit."""
    rng = np.random.default_rng(28)
    H, lens = 8, [150, 64]
    L = dk.layout(max_seq_len=300)
    k0, v0 = to(keys_of(rng, sum(lens), H)), to(halves(rng, sum(lens), H, D))
    q, k, v = (x.contiguous() for x in rows_of(rng, 2 * n, 2 * H, H))
    far = torch.empty((2 * n - 1) * (1 << 24) + 4 * H * D, dtype=torch.float16, device=DEV)
    apart = [far[at * D:].as_strided(x.shape, (1 << 24, D, 1)) for x, at in ((q, 0), (k, 2 * H), (v, 3 * H))]
    for to_, x in zip(apart, (q, k, v)):
        to_.copy_(x)
    got = []
    for blocks, rows in ((40, (q, k, v)), (66000, apart)):
        c = dk.BlockCache(L, blocks, 2, H, fmt=INT8, device=DEV)
        c.table.copy_(blocks - 1 - torch.arange(c.table.numel(), dtype=torch.int32, device=DEV).view(c.table.shape))
        dk.block_append(c, ints(lens), k0, v0)
        c.seq_len += ints(lens)
        out, lse = dk.block_attention(c, ints([n, n]), *rows, SCALE)
        dk.block_append(c, ints([n, n]), *rows[1:])
        c.seq_len += n
        total = sum(lens) + 2 * n
        got.append((out, lse, *dk.block_read(c, ints([0, 0]), ints([x + n for x in lens]), total), c.scale[-1]))
        assert int(c.status) == 0
    torch.cuda.synchronize()
    for x, y in zip(*got):
        assert torch.equal(x, y)
    assert got[0][2][:150].abs().sum() > 0
    freq = dk.rope_frequencies(128)[0].to(DEV)
    pos = torch.arange(2 * n, dtype=torch.int32, device=DEV)
    near = dk.norm_rotate(L, pos, freq, q, k)
    dk.norm_rotate(L, pos, freq, apart[0], apart[1], q_out=apart[0], k_out=apart[1])
    assert torch.equal(near[0], apart[0]) and torch.equal(near[1], apart[1])


def test_a_stream_of_another_gpu_is_refused():
    c = dk.BlockCache(dk.layout(max_seq_len=64), 4, 1, 1, device=DEV)
    k = torch.zeros((1, 1, D), dtype=torch.float16, device=DEV)

    class Elsewhere:
        device, cuda_stream = torch.device("cuda", 1), 0

    freq = dk.rope_frequencies(128)[0].to(DEV)
    for call in (lambda s: dk.block_append(c, ints([1]), k, k, stream=s),
                 lambda s: dk.block_read(c, ints([0]), ints([1]), 1, stream=s),
                 lambda s: dk.block_attention(c, ints([1]), k, k, k, SCALE, stream=s),
                 lambda s: dk.norm_rotate(c.L, ints([1]), freq, k, stream=s)):
        with pytest.raises(ValueError, match="stream"):
            call(Elsewhere())


def test_padded_batch_and_strides():
    """Rows behind the last sequence's are left as they were; a single row has any stride."""
    rng = np.random.default_rng(17)
    for n in (2, 150):
        plain = plain_of(rng, [100, 40], 2, E4M3)
        c = ref.filled(dk, plain, 400, DEV)
        q, k, v = rows_of(rng, 2 * n + 60, 8, 2)
        out = torch.full((2 * n + 60, 8, D), 5.0, dtype=torch.float16, device=DEV)
        lse = torch.full((2 * n + 60, 8), 5.0, device=DEV)
        dk.block_attention(c, ints([n, n]), q, k, v, SCALE, out=out, lse=lse, max_new=n + 60)
        torch.cuda.synchronize()
        check(plain, c, [n, n], q[:2 * n], k[:2 * n], v[:2 * n], out[:2 * n], lse[:2 * n], "padded")
        assert (out[2 * n:] == 5).all() and (lse[2 * n:] == 5).all()


@pytest.mark.parametrize("n", [0, 1, 5, 63, 64, 65])
def test_a_lone_sequence_with_less_rows_than_max_new(n):
    rng = np.random.default_rng(24)
    plain = plain_of(rng, [100], 2, INT8)
    c = ref.filled(dk, plain, 800, DEV)
    q, k, v = rows_of(rng, 400, 8, 2)
    out = torch.full((400, 8, D), 5.0, dtype=torch.float16, device=DEV)
    lse = torch.full((400, 8), 5.0, device=DEV)
    dk.block_attention(c, ints([n]), q, k, v, SCALE, out=out, lse=lse, max_new=400)
    torch.cuda.synchronize()
    if n:
        check(plain, c, [n], q[:n], k[:n], v[:n], out[:n], lse[:n], "padded")
    assert (out[n:] == 5).all() and (lse[n:] == 5).all()


def test_lengths_out_of_range_are_clamped():
    rng = np.random.default_rng(18)
    plain = plain_of(rng, [70, 40, 33], 2, INT8)
    c = ref.filled(dk, plain, 128, DEV)
    q, k, v = rows_of(rng, 12, 4, 2)
    out = torch.full((12, 4, D), 5.0, dtype=torch.float16, device=DEV)
    dk.block_attention(c, ints([100, -4, 9]), q, k, v, SCALE, out=out, max_new=8)
    torch.cuda.synchronize()
    want, _ = dk.block_attention(c, ints([8, 0, 4]), q, k, v, SCALE, max_new=8)
    assert torch.equal(out, want)


def test_results_do_not_change_from_run_to_run():
    rng = np.random.default_rng(19)
    lens, new = [5000, 31, 1200, 64], [1, 140, 33, 2]
    plain = plain_of(rng, lens, 2, E4M3)
    c, q, k, v, out, lse = attend(plain, new, 4, "again", max_len=6000)
    ws = torch.randint(0, 255, (dk.workspace_size(dk.OP_BLOCK_ATTENTION, c.L, 4, 8, 2, sum(new)),), dtype=torch.uint8, device=DEV)
    for _ in range(5):
        again, lse2 = dk.block_attention(c, ints(new), q, k, v, SCALE, ws=ws, max_new=140)
        assert torch.equal(out, again) and torch.equal(lse, lse2)


# ---- streams, graphs, together ---------------------------------------------------------------


def test_another_stream():
    rng = np.random.default_rng(20)
    plain = plain_of(rng, [333], 2, E4M3)
    c = ref.filled(dk, plain, 600, DEV)
    q, k, v = rows_of(rng, 40, 8, 2)
    nl = ints([40])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    out, lse = dk.block_attention(c, nl, q, k, v, SCALE, stream=s)
    s.synchronize()
    check(plain, c, [40], q, k, v, out, lse, "stream")
    with torch.cuda.stream(s):
        out2, _ = dk.block_attention(c, nl, q, k, v, SCALE)
        kb, _ = dk.block_read(c, ints([3]), ints([300]), 300)
    s.synchronize()
    assert torch.equal(out, out2)
    x, _ = plain.read(0, 1, 0, lambda i: True)
    assert np.array_equal(kb[:, 1].cpu().numpy(), x[3:303].astype(np.float16))


def test_captured_step():
    """A decode step of norms, attention and append, captured once and replayed with lengths that grow."""
    rng = np.random.default_rng(21)
    B, H, Hq = 3, 2, 8
    plain = plain_of(rng, [60, 31, 300], H, INT8)
    c = ref.filled(dk, plain, 400, DEV, spare=40)
    free = sorted(set(range(c.num_blocks)) - set(c.table.cpu().numpy().ravel().tolist()))
    for b, n in enumerate((60, 31, 300)):
        for i in range(n // T, n // T + 3):
            c.table[b, i] = free.pop()
    freq = dk.rope_frequencies(128)[0].to(DEV)
    w = torch.rand(128, device=DEV) + 0.5
    x = torch.zeros((B, Hq + 2 * H, D), dtype=torch.float16, device=DEV)
    one = ints([1] * B)
    qr, kr = torch.zeros((B, Hq, D), dtype=torch.float16, device=DEV), torch.zeros((B, H, D), dtype=torch.float16, device=DEV)
    out, lse = torch.zeros_like(qr), torch.zeros((B, Hq), device=DEV)
    ws = torch.zeros(dk.workspace_size(dk.OP_BLOCK_ATTENTION, c.L, B, Hq, H, B), dtype=torch.uint8, device=DEV)

    def step():
        dk.norm_rotate(c.L, c.seq_len, freq, x[:, :Hq], x[:, Hq:Hq + H], w, None, q_out=qr, k_out=kr)
        dk.block_attention(c, one, qr, kr, x[:, Hq + H:], SCALE, window=128, sinks=4, out=out, lse=lse, max_new=1, ws=ws)
        dk.block_append(c, one, kr, x[:, Hq + H:], max_new=1)

    step()  # (at the same position as the first replay)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(40):
        x.copy_(to(halves(rng, B, Hq + 2 * H, D)))
        g.replay()
        torch.cuda.synchronize()
        check(plain, c, [1] * B, qr, kr, x[:, Hq + H:], out, lse, "replay %d" % i, window=128, sinks=4)
        plain.append([1] * B, kr.cpu().numpy(), x[:, Hq + H:].cpu().numpy())
        c.seq_len += 1
    assert int(c.status) == 0
    same_cache(c, plain, "replays")


@pytest.mark.parametrize("fmt", [E4M3, INT8])
def test_together(fmt):
    """A prompt in parts, drafts, single tokens: attended, appended, read back and appended to a differentiated cache."""
    rng = np.random.default_rng(22)
    B, H, G = 2, 2, 4
    calls = [[70, 33], [128, 0], [5, 8], [1, 1], [1, 1], [64, 3]]
    total = np.array(calls).sum(0).tolist()
    c = new_cache(total, H, fmt)
    plain = ref.Plain(B, H, fmt)
    freq = dk.rope_frequencies(64)[0].to(DEV)
    for new in calls:
        q, k, v = rows_of(rng, sum(new), H * G, H)
        pos = np.concatenate([len(plain.rows[b][0]) + np.arange(n) for b, n in enumerate(new)]).astype(np.int32)
        qr, kr = dk.norm_rotate(c.L, to(pos), freq, q, k, eps=1e-5, style=dk.ROPE_INTERLEAVED)
        kr = (kr * 4).half()
        out, lse = dk.block_attention(c, ints(new), qr, kr, v, SCALE, window=100, sinks=3)
        torch.cuda.synchronize()
        check(plain, c, new, qr, kr, v, out, lse, "together %s" % new, window=100, sinks=3)
        dk.block_append(c, ints(new), kr, v)
        plain.append(new, kr.cpu().numpy(), v.cpu().numpy())
        c.seq_len += ints(new)
    torch.cuda.synchronize()
    assert int(c.status) == 0
    same_cache(c, plain, "together")
    k, v = dk.block_read(c, ints([0] * B), ints(total), sum(total))
    d = dk.Cache(dk.layout(max_seq_len=512), 200, B, H, device=DEV)
    dk.quantize_append(d, ints(total), k, v, torch.ones((sum(total), H), device=DEV), total_new=sum(total), max_new=max(total))
    torch.cuda.synchronize()
    assert int(d.status) == 0 and d.len.cpu()[:, 0].tolist() == [n for n in total for _ in range(H)]
