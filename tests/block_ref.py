"""Plain 64-bit definitions of the uniform 8-bit cache's operators, for their tests: blocks quantized and packed value by
value, attention with windows and first tokens, norms."""
import numpy as np
import torch

D, T = 128, 32


def e4m3(x):
    """The nearest e4m3 values (ties to the even one) of |x| <= 448."""
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 4, -9))
    return np.rint(x / step) * step


def quantized(x, fmt):
    """x [T, D] -> codes [T, D] as numbers, the scale; both exactly (64 bits hold every step)."""
    x = np.asarray(x, np.float64)
    if not np.isfinite(x).all():
        return np.zeros_like(x), np.nan
    top = np.abs(x).max()
    if top == 0:
        return x * 0.0, 1.0
    if fmt == 0:
        s = 2.0 ** -60
        while top > 448 * s:
            s *= 2.0
        return e4m3(x / s), s
    m, e = np.frexp(top / 127)
    s = np.ldexp(np.ceil(m * 256), e - 8)
    return np.rint(x / s), s


def code_bytes(codes, fmt):
    t = torch.from_numpy(codes)
    return t.to(torch.float8_e4m3fn if fmt == 0 else torch.int8).view(torch.uint8).numpy()


def numbers(b, fmt):
    return torch.from_numpy(np.ascontiguousarray(b)).view(torch.float8_e4m3fn if fmt == 0 else torch.int8).double().numpy()


_t, _d = np.meshgrid(np.arange(T), np.arange(D), indexing="ij")
KEY_AT = _t // 16 * 2048 + _d // 16 * 256 + _t % 16 * 16 + _d % 16
VALUE_AT = _d // 32 * 1024 + _t % 16 // 4 * 256 + _d % 16 * 16 + _d // 16 % 2 * 8 + _t // 16 * 4 + _t % 4
AT = (KEY_AT, VALUE_AT)


class Plain:
    """What a cache should hold: every token appended, [B][side] lists of [tokens, H, D] fp16."""

    def __init__(self, B, H, fmt):
        self.H, self.fmt = H, fmt
        self.rows = [[np.zeros((0, H, D), np.float16) for _ in (0, 1)] for _ in range(B)]

    def append(self, new_len, k, v):
        row = 0
        for b, n in enumerate(new_len):
            for side, x in enumerate((k, v)):
                self.rows[b][side] = np.concatenate([self.rows[b][side], x[row:row + n]])
            row += n

    def block(self, b, i, h, side):
        """Codes as numbers and scale of a whole block."""
        return quantized(self.rows[b][side][i * T:i * T + T, h], self.fmt)

    def read(self, b, h, side, kept):
        """[tokens, D] in 64 bits as the cache gives them, and which are there; kept(i): block i is stored."""
        x = self.rows[b][side][:, h].astype(np.float64)
        there = np.ones(len(x), bool)
        for i in range(len(x) // T):
            if kept(i):
                c, s = self.block(b, i, h, side)
                x[i * T:i * T + T] = c * s
            else:
                x[i * T:i * T + T] = 0.0
                there[i * T:i * T + T] = False
        return x, there


def filled(dk, plain, max_len, device, seed=0, drop=(), spare=3):
    """A cache that holds plain's tokens (packed here, not by the library); `drop`: (b, i) blocks not kept."""
    B, H = len(plain.rows), plain.H
    L = dk.layout(max_seq_len=max_len)
    lens = [len(r[0]) for r in plain.rows]
    used = [(b, i) for b in range(B) for i in range(lens[b] // T)]
    N = len(used) + spare
    c = dk.BlockCache(L, N, B, H, fmt=plain.fmt, device=device)
    rng = np.random.default_rng(seed)
    ids = rng.permutation(N)
    table = np.full(c.table.shape, -1, np.int32)
    pool = rng.integers(0, 120, (N, H, 2, T * D), dtype=np.uint8)  # (a block that nothing wrote holds anything)
    scale = np.ones((N, H, 2), np.float32)
    tail = np.full((B, H, 2, T, D), np.nan, np.float16)
    for (b, i), p in zip(used, ids):
        table[b, i] = -1 if (b, i) in drop else p
        for h in range(H):
            for side in (0, 1):
                codes, s = plain.block(b, i, h, side)
                pool[p, h, side][AT[side]] = code_bytes(codes, plain.fmt)
                scale[p, h, side] = s
    for b in range(B):
        rest = lens[b] % T
        for side in (0, 1):
            tail[b, :, side, :rest] = plain.rows[b][side][lens[b] - rest:].transpose(1, 0, 2)
    for t, a in ((c.pool, pool), (c.scale, scale), (c.table, table), (c.tail, tail), (c.seq_len, np.array(lens, np.int32))):
        t.copy_(torch.from_numpy(a))
    return c


def seen(L, n, tokens, window, sinks):
    """[n, tokens]: which keys (positions 0 ..) the new tokens L .. L + n - 1 see."""
    p, c = np.arange(L, L + n)[:, None], np.arange(tokens)[None]
    ok = c <= p
    if window:
        ok &= (p - c < window) | (c < sinks)
    return ok


def attention(plain, new_len, q, k, v, sm_scale, kept, cap=0.0, window=0, sinks=0, slopes=None):
    """Per sequence and KV head: (b, h, first row, n, out [G, n, D], lse [G, n], A = sum p |v|, size of the scores'
    products, keys, largest |v|)."""
    H = plain.H
    G = q.shape[1] // H
    row = 0
    q = q.astype(np.float64)
    for b, n in enumerate(new_len):
        for h in range(H if n else 0):
            (ck, there), (cv, _) = (plain.read(b, h, side, lambda i: kept(b, i)) for side in (0, 1))
            keys = np.concatenate([ck, k[row:row + n, h].astype(np.float64)])
            vals = np.concatenate([cv, v[row:row + n, h].astype(np.float64)])
            L = len(ck)
            ok = seen(L, n, L + n, window, sinks)
            ok[:, :L] &= there[None]
            qq = q[row:row + n, h * G:(h + 1) * G].transpose(1, 0, 2)
            with np.errstate(invalid="ignore", over="ignore"):
                x = qq @ keys.T * sm_scale
                size = np.abs(qq) @ np.abs(keys.T) * sm_scale
                if cap:
                    x = cap * np.tanh(x / cap)
                if slopes is not None:
                    away = np.arange(L, L + n)[:, None] - np.arange(L + n)[None]
                    bias = np.asarray(slopes, np.float64)[h * G:(h + 1) * G, None, None] * away
                    x, size = x - bias, size + np.abs(bias) / 16
                x = np.where(ok[None], x, -np.inf)
                size = np.where(ok[None], size, 0.0)
                top = x.max(-1, keepdims=True)
                p = np.where(ok[None], np.exp(x - top), 0.0)
                total = p.sum(-1, keepdims=True)
                p /= total
                shown = ok.any(0)
                vals = np.where(shown[:, None], vals, 0.0)
                out = np.stack([np.where(ok[j][:, None], vals, 0.0).T @ p[:, j].T for j in range(n)]).transpose(2, 0, 1)
                A = p @ np.abs(np.where(np.isfinite(vals), vals, 0.0))
                lse = (top + np.log(total))[..., 0]
            yield b, h, row, n, out, lse, A, size.max(-1), L + n, np.abs(vals[np.isfinite(vals)]).max(initial=0.0)
        row += n


def norm_rotated(x, weight, eps, pos, freq, style, scale):
    x = x.astype(np.float64)
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight.astype(np.float64))
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float32).astype(np.float64)[None]
    c, s = np.cos(a)[:, None] * scale, np.sin(a)[:, None] * scale
    half = a.shape[1]
    i = np.arange(half)
    lo, hi = (i, i + half) if style == 0 else (2 * i, 2 * i + 1)
    z, size = y.copy(), np.abs(y)
    z[..., lo] = y[..., lo] * c - y[..., hi] * s
    z[..., hi] = y[..., hi] * c + y[..., lo] * s
    both = (np.abs(y[..., lo]) + np.abs(y[..., hi])) * scale
    size[..., lo] = size[..., hi] = both
    return z, size
