"""Plain 64-bit definitions of the chunk operators, for their tests: a cache's kept tokens read
back from its pages byte by byte, attention and scores of a chunk over them, rotary positions."""
import numpy as np
import torch

D, G32 = 128, 32


def unpack(b, bits):
    """Bytes [..., n] -> codes [..., n * 8 / bits], the lowest bits first."""
    per = 8 // bits
    return ((b[..., None] >> (np.arange(per) * bits)) & (2 ** bits - 1)).reshape(*b.shape[:-1], -1)


def kept_tokens(cache):
    """Per table: keys [n, D] and values [n, D] in 64 bits, positions, scores, and where they are
    (page, section, slot), the high section first."""
    L = cache.L
    table = cache.page_table.cpu().numpy()
    lens = cache.len.cpu().numpy()
    used = np.unique(table[(table >= 0) & (table < cache.num_pages)])
    pool = dict(zip(used.tolist(), cache.pool[torch.from_numpy(used).long().to(cache.pool.device)].cpu().numpy()))
    out = []
    for t in range(cache.num_tables):
        ks, vs, pos, score, where = [], [], [], [], []
        for sec in (0, 1):
            T, kb, vb = L.tokens_per_page[sec], L.k_bits[sec], L.v_bits[sec]
            for u0 in range(0, int(lens[t, sec]), T):
                n = min(T, int(lens[t, sec]) - u0)
                i = u0 // T
                page = int(table[t, i if sec == 0 else L.p_max - 1 - i])
                if page not in pool:  # an ID outside the pool counts no token
                    continue
                b = pool[page]

                def seg(off, size):
                    return b[off:off + size]

                kc = unpack(seg(L.off_kcode[sec], D * kb * T // 8).reshape(-1, T, 16), kb)  # [chunk, T, dims]
                kc = kc.transpose(1, 0, 2).reshape(T, D).astype(np.float64)
                km = seg(L.off_kmeta[sec], 16 * T).view(np.float16).reshape(T, 4, 2).astype(np.float64)
                vc = unpack(seg(L.off_vcode[sec], D * T * vb // 8).reshape(D, -1), vb).T.astype(np.float64)
                vm = seg(L.off_vmeta[sec], 16 * T).view(np.float16).reshape(4, T, 2).transpose(1, 0, 2).astype(np.float64)
                ks.append((kc * km[:, :, 0].repeat(G32, 1) + km[:, :, 1].repeat(G32, 1))[:n])
                vs.append((vc * vm[:, :, 0].repeat(G32, 1) + vm[:, :, 1].repeat(G32, 1))[:n])
                pos.append(seg(L.off_pos[sec], 4 * T).view(np.int32)[:n])
                score.append(seg(L.off_score[sec], 4 * T).view(np.float32)[:n].astype(np.float64))
                where += [(page, sec, s) for s in range(n)]
        cat = lambda x, shape: np.concatenate(x) if x else np.zeros(shape)
        out.append((cat(ks, (0, D)), cat(vs, (0, D)), cat(pos, (0,)).astype(np.int64), cat(score, (0,)), where))
    return out


def score_at(cache, where):
    """Scores now in the pages at `where`."""
    L = cache.L
    used = np.unique([p for p, _, _ in where]).astype(np.int64)
    pool = dict(zip(used.tolist(), cache.pool[torch.from_numpy(used).to(cache.pool.device)].cpu().numpy()))
    return np.array([pool[p][L.off_score[s] + 4 * i:L.off_score[s] + 4 * i + 4].view(np.float32)[0] for p, s, i in where],
                    np.float64)


def logits(cache, kept, new_len, q, k, sm_scale, cap=0.0, window=0, slopes=None):
    """Per (sequence, KV head): (b, h, row0, n, x [G, n, keys], bound on |x|'s products [G, n, keys])."""
    H = cache.num_kv_heads
    G = q.shape[1] // H
    seen = cache.seq_len.cpu().numpy()
    q, k = q.cpu().numpy().astype(np.float64), k.cpu().numpy().astype(np.float64)
    row = 0
    for b, n in enumerate(new_len):
        for h in range(H if n else 0):
            keys = np.concatenate([kept[b * H + h][0], k[row:row + n, h]])
            mine = seen[b] + np.arange(n)
            pos = np.concatenate([kept[b * H + h][2], mine])
            qq = q[row:row + n, h * G:(h + 1) * G].transpose(1, 0, 2)
            with np.errstate(invalid="ignore", over="ignore"):
                x = qq @ keys.T * sm_scale
                size = np.abs(qq) @ np.abs(keys.T) * sm_scale
            if cap:
                x = cap * np.tanh(x / cap)
            away = mine[:, None] - pos[None]
            if slopes is not None:
                x = x - np.asarray(slopes, np.float64)[h * G:(h + 1) * G, None, None] * away
            hide = away < 0
            if window:
                hide |= away >= window
            x[:, hide] = -np.inf
            size[:, hide] = 0.0
            yield b, h, row, n, x, size
        row += n


def softmax(x):
    top = x.max(-1, keepdims=True)
    p = np.exp(x - top)
    total = p.sum(-1, keepdims=True)
    return p / total, (top + np.log(total))[..., 0]


def rotated(x, pos, freq, style, scale):
    x = x.cpu().numpy().astype(np.float64)
    a = np.asarray(pos, np.float64)[:, None] * np.asarray(freq, np.float32).astype(np.float64)[None]
    c, s = np.cos(a)[:, None] * scale, np.sin(a)[:, None] * scale
    half = a.shape[1]
    i = np.arange(half)
    lo, hi = (i, i + half) if style == 0 else (2 * i, 2 * i + 1)
    y = x.copy()
    y[..., lo] = x[..., lo] * c - x[..., hi] * s
    y[..., hi] = x[..., hi] * c + x[..., lo] * s
    return y


def filled(dk, layout, B, Hkv, lens, seed, max_len=None, prune=0.3, high=0.4, device="cuda", kscale=1.0, before=0):
    """A cache that saw lens[b] tokens of each sequence, high / low / pruned by quota."""
    rng = np.random.default_rng(seed)
    lens = np.asarray(lens, np.int32)
    L = dk.layout(max_seq_len=max_len or int(lens.max(initial=1)) + 512, **layout)
    pages = int(sum(Hkv * (2 * (int(n) // 16 + 2)) for n in lens)) + 8
    # (`before` pages that nothing uses come first in the pool)
    ring = np.concatenate([before + rng.permutation(pages), np.arange(before)]).astype(np.int32)
    cache = dk.Cache(L, before + pages, B, Hkv, device=device, ring=torch.from_numpy(ring))
    rows = int(lens.sum())
    if rows:
        k = rng.standard_normal((rows, Hkv, D)) * kscale
        k[:, :, [3, 40, 77, 120]] *= 6.0
        v = rng.standard_normal((rows, Hkv, D))
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)
        quota = np.zeros((B, Hkv, 2), np.int32)
        for b in range(B):
            for h in range(Hkv):
                hi = int(rng.uniform(0.5, 1.5) * high * lens[b])
                quota[b, h] = hi, max(0, int(lens[b]) - hi - int(prune * lens[b]))
        dk.quantize_append(cache, to(lens), to(k.astype(np.float16)), to(v.astype(np.float16)),
                           to(rng.random((rows, Hkv), dtype=np.float32) * 0.1), quota=to(quota), total_new=rows,
                           max_new=int(lens.max()))
        torch.cuda.synchronize()
        assert int(cache.status.cpu()[0]) == 0
    return cache
