"""Chunks of new tokens over the compressed cache: rotation, attention, scores.

What a serving program does with the new tokens of its sequences before they are
appended: one token each (decoding), a few (checking drafted tokens), hundreds (a
prompt's next part), or a mixture.  Three operators:

  rotate   rotary positions of queries and keys, read from a fused projection
  attend   attention of every new token over the kept tokens of its sequence's cache
           and the new tokens up to itself, in 16 bits, with its normalizers
  score    the significance of the new tokens and the running means of the cached
           ones, updated in their pages

Keys and values of the cache are quantized N(0, 1) draws with four key channels per KV
head times 10, a random part of the positions kept; a case's `split` says how many are
kept high / low: "mixed" high U[0.1, 0.5], pruned U[0.2, 0.6]; "long" pruned
0.1 + 0.8 Beta(2, 2), the rest halved; "fixed" 30 / 40 / 30.
"""
import math
import random
import types

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
# (k_bits, v_bits, tokens per page) of the high and the low section
LAYOUTS = (
    ((8, 4, 16), (4, 2, 32)),
    ((8, 8, 16), (4, 2, 32)),
    ((8, 2, 16), (4, 1, 32)),
    ((8, 4, 16), (4, 2, 16)),
)
SHARES = {"mixed": (0.3, 0.3), "long": (0.25, 0.25), "fixed": (0.3, 0.4)}


def _case(kind, name=None, **c):
    c = dict(dict(kind=kind), **c)
    if name:
        c["name"] = name
    if kind != "rotate":
        for key, value in dict(layout=0, split="mixed", cap=0.0, window=0, slopes=False, long_chunks=-1).items():
            c.setdefault(key, value)
    return c


def listed():
    return [
        # A decode step of 64 requests: one token each, all of the head rotated.
        _case("rotate", "rotate_step", rows=64, Hq=32, Hkv=8, rot=128, style="half", base=500000.0, scale=1.0,
              start=4096),
        # Long prompts far into their context: neighbouring pairs, half of the head, stretched positions.
        _case("rotate", "rotate_prompts", rows=32767, Hq=40, Hkv=8, rot=64, style="interleaved", base=10000.0,
              scale=1.1386, start=100000),
        # One user alone, one token after a short prompt: nothing but latency.
        _case("attend", "attend_single", B=1, Hq=32, Hkv=8, L_min=600, L_max=600, n_min=1, n_max=1),
        # A decode step of a full batch of ragged requests.
        _case("attend", "attend_step_8b", B=64, Hq=32, Hkv=8, L_min=1024, L_max=4096, n_min=1, n_max=1),
        # A decode step of few long generations, scores capped and biased by distance.
        _case("attend", "attend_step_32k_biased", B=16, Hq=40, Hkv=8, L_min=32768, L_max=32768, n_min=1, n_max=1,
              split="long", cap=30.0, slopes=True),
        # Up to eight drafted tokens per request are checked, GQA 7, 8-bit values, windowed scores.
        _case("attend", "attend_drafts", B=24, Hq=28, Hkv=4, L_min=501, L_max=5999, n_min=1, n_max=8, layout=1,
              window=2048),
        # A serving step that carries a part of one prompt beside 31 decoding requests.
        _case("attend", "attend_mixed", B=32, Hq=32, Hkv=8, L_min=1024, L_max=4096, n_min=1, n_max=1,
              long_chunks=512),
        # The next parts of eight prompts, ragged, some of them the first part.
        _case("attend", "attend_parts_8b", B=8, Hq=32, Hkv=8, L_min=0, L_max=8192, n_min=257, n_max=512),
        # A large part of one long prompt, GQA 8.
        _case("attend", "attend_part_70b", B=1, Hq=64, Hkv=8, L_min=8192, L_max=8192, n_min=2048, n_max=2048,
              split="fixed"),
        # Scores after the decode step of the full batch.
        _case("score", "score_step_8b", B=64, Hq=32, Hkv=8, L_min=1024, L_max=4096, n_min=1, n_max=1),
        # Scores of drafted tokens, distance bias, the narrowest page formats.
        _case("score", "score_drafts", B=24, Hq=20, Hkv=4, L_min=501, L_max=5999, n_min=1, n_max=8, layout=2,
              slopes=True),
        # Scores of eight prompts' next parts.
        _case("score", "score_parts_8b", B=8, Hq=32, Hkv=8, L_min=0, L_max=8192, n_min=257, n_max=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rotate", "attend", "attend", "attend", "score", "score"))
    Hkv = rng.choice((1, 2, 4, 8))
    G = rng.randint(1, 8)
    if kind == "rotate":
        rows = _log_int(rng, 1, 32767 * 48 // (Hkv * (G + 1)) if Hkv * (G + 1) > 48 else 32767)
        return _case("rotate", rows=rows, Hq=Hkv * G, Hkv=Hkv, rot=rng.choice((16, 32, 64, 96, 128)),
                     style=rng.choice(("half", "interleaved")), base=rng.choice((10000.0, 500000.0)),
                     scale=rng.choice((1.0, 1.1386)), start=_log_int(rng, 1, 1000000))
    form = rng.choice(("step", "drafts", "parts", "parts"))
    n_max = {"step": 1, "drafts": rng.randint(2, 16), "parts": _log_int(rng, 17, 2048)}[form]
    n_min = rng.randint(0 if n_max > 1 else 1, n_max)
    L_max = _log_int(rng, 16, 32768 if form != "parts" else 8192)
    L_min = rng.choice((0, int(L_max * rng.uniform(0.1, 1.0)), L_max))
    pairs = {"step": 16 * 32768, "drafts": 24 * 8 * 6000, "parts": 2048 * 8192}[form]
    most = min(64, max(1, int(pairs / (n_max * (L_max + n_max)))), 16 * 32768 // (L_max + 1) or 1)
    return _case(kind, B=_log_int(rng, 1, most), Hq=G * Hkv, Hkv=Hkv, L_min=L_min, L_max=L_max, n_min=n_min,
                 n_max=n_max, split=rng.choice(tuple(SHARES)), layout=rng.choice((0, 0, 1, 2, 3)),
                 cap=rng.choice((0.0, 0.0, 30.0, 50.0)), window=rng.choice((0, 0, _log_int(rng, 1, 4096))),
                 slopes=rng.random() < 0.3)


# ---- inputs -------------------------------------------------------------------


def _gen(seed, part):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000 + part)
    return g


def _lens(case):
    """Tokens seen and new tokens per sequence: the case's (they set the outputs' sizes)."""
    r = random.Random("lengths %(B)d %(L_min)d %(L_max)d %(n_min)d %(n_max)d" % case)
    seen = [r.randint(case["L_min"], case["L_max"]) for _ in range(case["B"])]
    new = [r.randint(case["n_min"], case["n_max"]) for _ in range(case["B"])]
    if case["long_chunks"] > 0:
        new[case["B"] // 3] = case["long_chunks"]
    return seen, new if any(new) else new[:-1] + [1]


def _kept(case, seen):
    """[tables, 2] tokens kept high and low."""
    r = random.Random("kept %d %s" % (case["Hkv"], seen))
    rows = []
    for n in seen:
        for _ in range(case["Hkv"]):
            if case["split"] == "mixed":
                hi, pruned = r.uniform(0.1, 0.5), r.uniform(0.2, 0.6)
                pruned = min(pruned, 1.0 - hi)
            elif case["split"] == "long":
                pruned = 0.1 + 0.8 * r.betavariate(2.0, 2.0)
                hi = (1.0 - pruned) / 2
            else:
                hi, pruned = 0.3, 0.3
            rows.append((int(hi * n), n - int(hi * n) - int(pruned * n)))
    return torch.tensor(rows, dtype=torch.int64).reshape(-1, 2)


def _offsets(case):
    """Per section: where its codes, scales, scores and positions start in a page; page bytes."""
    out = []
    for kb, vb, T in LAYOUTS[case["layout"]]:
        at, o = 0, {}
        for name, size in (("kc", D * kb * T // 8), ("km", T * 16), ("vc", D * T * vb // 8), ("vm", T * 16),
                           ("score", 4 * T), ("pos", 4 * T)):
            o[name] = at
            at = (at + size + 63) // 64 * 64
        o["used"] = at
        out.append(o)
    return out, max(o["used"] for o in out)


def _quantized(x, bits):
    """x [n, D] fp32 -> codes [n, D] uint8 and scales / zeros [n, D / 32, 2] fp16."""
    g = x.reshape(-1, D // 32, 32)
    z = g.amin(2)
    s = ((g.amax(2) - z) / (2 ** bits - 1)).half()
    z = z.half()
    q = (g - z.float()[..., None]) / s.float().clamp(min=1e-8)[..., None]
    return q.round_().clamp_(0, 2 ** bits - 1).to(torch.uint8).reshape(-1, D), torch.stack([s, z], 2)


def _packed(codes, bits):
    """Codes along the last axis, 8 / bits to a byte, the first lowest."""
    if bits == 8:
        return codes
    per = 8 // bits
    c = codes.reshape(*codes.shape[:-1], -1, per).to(torch.int32)
    return (c << (torch.arange(per, device=c.device, dtype=torch.int32) * bits)).sum(-1).to(torch.uint8)


def _heads_scale(case, seed):
    scale = torch.ones((case["Hkv"], D), device="cuda")
    at = torch.rand((case["Hkv"], D), generator=_gen(seed, 5), device="cuda").argsort(dim=1)[:, :4]
    return scale.scatter_(1, at, 10.0)


def _filled(case, seed):
    """The cache's device buffers, and per section its tokens in table and position order:
    (table, position, page, slot, key codes and scales, value codes and scales, score)."""
    seen, _ = _lens(case)
    B, H, T = case["B"], case["Hkv"], case["B"] * case["Hkv"]
    kept = _kept(case, seen)
    offsets, page_bytes = _offsets(case)
    fmt = LAYOUTS[case["layout"]]
    held = torch.stack([-(-kept[:, i] // fmt[i][2]) for i in (0, 1)], 1)
    most = held.amax(0).tolist()
    p_max = -(-(case["L_max"] + case["n_max"] + 64) // fmt[0][2]) + 1
    n_high, total = int(held[:, 0].sum()), int(held.sum())
    # one page more than the cache has: nobody's
    pool = torch.zeros((total + 9, page_bytes), dtype=torch.uint8, device="cuda")
    scale = _heads_scale(case, seed)
    longest = max(max(seen), 1)
    order = torch.rand((T, longest), generator=_gen(seed, 1), device="cuda")
    lens = torch.tensor(seen, device="cuda").repeat_interleave(H)
    order.masked_fill_(torch.arange(longest, device="cuda")[None] >= lens[:, None], 2.0)
    rank = order.argsort(dim=1).argsort(dim=1)
    keep = kept.cuda()
    table = torch.full((T, p_max), -1, dtype=torch.int32, device="cuda")
    tokens = []
    for sec in (0, 1):
        kb, vb, per = fmt[sec]
        low, high = (torch.zeros_like(keep[:, 0]), keep[:, 0]) if sec == 0 else (keep[:, 0], keep.sum(1))
        member = (rank >= low[:, None]) & (rank < high[:, None])
        t, pos = member.nonzero(as_tuple=True)
        u = (member.cumsum(1) - 1)[member]
        n = t.numel()
        first = (held[:, sec].cumsum(0) - held[:, sec]).cuda()
        pages = int(held[:, sec].sum())
        ids = torch.randperm(pages, generator=_gen(seed, 6 + sec), device="cuda") + (n_high if sec else 0)
        at = torch.repeat_interleave(torch.arange(T, device="cuda"), held[:, sec].cuda())
        ordinal = torch.arange(pages, device="cuda") - first[at]
        table[at, ordinal if sec == 0 else p_max - 1 - ordinal] = ids.int()
        slot = (first[t] + u // per) * per + u % per  # in the section's pages laid end to end
        head = t % H
        score = torch.rand(n, generator=_gen(seed, 8 + sec), device="cuda") ** 4 * 0.05
        sides = []
        for side, bits in enumerate((kb, vb)):
            codes = torch.zeros((pages * per, D), dtype=torch.uint8, device="cuda")
            meta = torch.zeros((pages * per, D // 32, 2), dtype=torch.float16, device="cuda")
            g = _gen(seed, 10 + 2 * sec + side)
            for i in range(0, n, 1 << 19):
                part = slice(i, min(n, i + (1 << 19)))
                x = torch.randn((part.stop - i, D), generator=g, device="cuda")
                if side == 0:
                    x *= scale[head[part]]
                codes[slot[part]], meta[slot[part]] = _quantized(x, bits)
            sides += [codes, meta]
        kc, km, vc, vm = sides
        o = offsets[sec]

        def put(name, x):
            b = x.contiguous().view(torch.uint8).reshape(pages, -1)
            pool[ids, o[name]:o[name] + b.shape[1]] = b

        def laid(x, dtype):
            return torch.zeros(pages * per, dtype=dtype, device="cuda").index_copy_(0, slot, x.to(dtype))

        if pages:
            put("kc", _packed(kc, kb).reshape(pages, per, -1, 16).transpose(1, 2))
            put("km", km)
            put("vc", _packed(vc.reshape(pages, per, D).transpose(1, 2), vb))
            put("vm", vm.reshape(pages, per, D // 32, 2).transpose(1, 2))
            put("score", laid(score, torch.float32))
            put("pos", laid(pos, torch.int32))
        tokens.append((t, pos, ids[slot // per] if n else slot, slot % per, kc[slot], km[slot], vc[slot], vm[slot],
                       score))
    cache = types.SimpleNamespace(
        pool=pool, num_pages=total + 8, num_seqs=B, num_kv_heads=H, page_table=table, pages=held.int().cuda(),
        len=kept.int().cuda(), seq_len=torch.tensor(seen, dtype=torch.int32, device="cuda"),
        ring=torch.arange(total + 8, dtype=torch.int32, device="cuda"),
        ring_ptr=torch.tensor([total, total + 8], device="cuda"),
        status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    views = tuple(pool[lo:hi, offsets[i]["score"]:offsets[i]["score"] + 4 * fmt[i][2]].view(torch.float32)
                  for i, (lo, hi) in enumerate(((0, n_high), (n_high, total))))
    return cache, tokens, most, views


def _rows(case, seed):
    """The new tokens' queries, keys, values: slices of one projection's output."""
    rows, Hq, Hkv = sum(_lens(case)[1]), case["Hq"], case["Hkv"]
    x = torch.randn((rows, Hq + 2 * Hkv, D), generator=_gen(seed, 20), device="cuda")
    x[:, Hq:Hq + Hkv] *= _heads_scale(case, seed)
    x = x.half()
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def _slopes(case):
    h = torch.arange(1, case["Hq"] + 1, device="cuda", dtype=torch.float32)
    return torch.exp2(-8.0 * h / case["Hq"]) if case["slopes"] else None


def prepare(case, seed):
    if case["kind"] == "rotate":
        return _prepare_rotate(case, seed)
    cache, _, most, views = _filled(case, seed)
    seen, new = _lens(case)
    q, k, v = _rows(case, seed)
    s = {"case": case, "cache": cache, "most": most, "longest": max(new), "q": q, "k": k, "v": v,
         "new_len": torch.tensor(new, dtype=torch.int32, device="cuda"), "slopes": _slopes(case)}
    if case["kind"] == "score":
        s["views"] = views
        s["lse"] = _plain_attention(s)[1]  # as attention wrote them
        s["score"] = torch.empty((q.shape[0], case["Hkv"]), dtype=torch.float32, device="cuda")
    else:
        s["out"] = torch.empty((q.shape[0], case["Hq"], D), dtype=torch.float16, device="cuda")
        s["lse"] = torch.empty((q.shape[0], case["Hq"]), dtype=torch.float32, device="cuda")
    return s


def run(s):
    if own:
        return _RUN_OWN[s["case"]["kind"]](s)
    return _RUN_PLAIN[s["case"]["kind"]](s)


# ---- rotation -------------------------------------------------------------------


def _prepare_rotate(case, seed):
    rows, Hq, Hkv, half = case["rows"], case["Hq"], case["Hkv"], case["rot"] // 2
    x = torch.randn((rows, Hq + 2 * Hkv, D), generator=_gen(seed, 1), device="cuda").half()
    start = torch.randint(0, case["start"] + 1, (1,), generator=_gen(seed, 2), device="cuda")
    if rows <= 64:  # one token of every sequence
        pos = torch.randint(0, case["start"] + 1, (rows,), generator=_gen(seed, 2), device="cuda")
    else:
        pos = start + torch.arange(rows, device="cuda")
    freq = case["base"] ** (-torch.arange(half, dtype=torch.float64) / half)
    return {"case": case, "q": x[:, :Hq], "k": x[:, Hq:Hq + Hkv], "pos": pos.int(), "freq": freq.float().cuda(),
            "out": torch.empty((rows, Hq, D), dtype=torch.float16, device="cuda"),
            "k_out": torch.empty((rows, Hkv, D), dtype=torch.float16, device="cuda")}


def _own_rotate(s):
    from paper_2412_03131_amd import diffkv as dk
    if "L" not in s:
        s["L"] = dk.layout()
    c = s["case"]
    return dk.rotate(s["L"], s["pos"], s["freq"], s["q"], s["k"],
                     style=dk.ROPE_HALF if c["style"] == "half" else dk.ROPE_INTERLEAVED, scale=c["scale"],
                     q_out=s["out"], k_out=s["k_out"])


def _turned(x, cos, sin, style):
    half = cos.shape[1]
    y = x.float()
    r, rest = y[..., :2 * half], y[..., 2 * half:]
    a, b = (r[..., :half], r[..., half:]) if style == "half" else (r[..., 0::2], r[..., 1::2])
    a, b = a * cos[:, None] - b * sin[:, None], b * cos[:, None] + a * sin[:, None]
    r = torch.cat([a, b], -1) if style == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([r, rest], -1).half()


def _plain_rotate(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["freq"].double()[None]
    cos, sin = (angle.cos() * c["scale"]).float(), (angle.sin() * c["scale"]).float()
    return _turned(s["q"], cos, sin, c["style"]), _turned(s["k"], cos, sin, c["style"])


def _exact_rotate(case, seed):
    s = _prepare_rotate(case, seed)
    rot = case["rot"]
    turn = torch.polar(torch.full_like(s["freq"], case["scale"], dtype=torch.float64)[None].expand(case["rows"], -1),
                       torch.outer(s["pos"].double(), s["freq"].double()))
    got = []
    for x in (s["q"], s["k"]):
        y = x.double()
        pairs = y[..., :rot].reshape(*y.shape[:2], 2, -1).transpose(2, 3) if case["style"] == "half" else \
            y[..., :rot].reshape(*y.shape[:2], -1, 2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        z = z.transpose(2, 3) if case["style"] == "half" else z
        got.append(torch.cat([z.reshape(*y.shape[:2], rot), y[..., rot:]], 2))
    return tuple(got)


# ---- attention and scores: the framework's calls ---------------------------------------


def _handle(s):
    """The layout and workspace that a program keeps beside its cache."""
    from paper_2412_03131_amd import diffkv as dk
    if "ws" not in s:
        c, cache = s["case"], s["cache"]
        hi, lo = LAYOUTS[c["layout"]]
        cache.L = dk.layout(k_bits=(hi[0], lo[0]), v_bits=(hi[1], lo[1]), tokens_per_page=(hi[2], lo[2]),
                            max_seq_len=(cache.page_table.shape[1] - 1) * hi[2])
        need = dk.workspace_size(dk.OP_CHUNK_ATTENTION if c["kind"] == "attend" else dk.OP_CHUNK_SIGNIFICANCE, cache.L,
                                 c["B"], c["Hq"], c["Hkv"], s["q"].shape[0])
        s["ws"] = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    return dk


def _own_attend(s):
    dk = _handle(s)
    c = s["case"]
    return dk.chunk_attention(s["cache"], s["new_len"], s["q"], s["k"], s["v"], SCALE, cap=c["cap"],
                              window=c["window"], slopes=s["slopes"], out=s["out"], lse=s["lse"],
                              max_new=s["longest"], ws=s["ws"])


def _own_score(s):
    dk = _handle(s)
    c = s["case"]
    dk.chunk_significance(s["cache"], s["new_len"], s["q"], s["k"], SCALE, s["lse"], cap=c["cap"],
                          window=c["window"], slopes=s["slopes"], score=s["score"], max_new=s["longest"], ws=s["ws"])
    return {"score": s["score"], "cached": s["views"]}


# ---- attention and scores: plain ------------------------------------------------------------


def _section(s, sec):
    """A section's tokens of all tables, padded: keys and values [tables, tokens, D] fp32, their
    positions and page IDs, and which of them exist."""
    c, cache = s["case"], s["cache"]
    kb, vb, per = LAYOUTS[c["layout"]][sec]
    o, pages = _offsets(c)[0][sec], s["most"][sec]
    ids = cache.page_table[:, :pages] if sec == 0 else cache.page_table.flip(1)[:, :pages]
    ids = torch.where(ids < 0, cache.num_pages, ids).long()
    raw = cache.pool[ids]
    T = raw.shape[0]

    def part(name, size, dtype=None):
        x = raw[:, :, o[name]:o[name] + size]
        return x if dtype is None else x.contiguous().view(dtype)

    def unpacked(x, bits):
        per_byte = 8 // bits
        shift = torch.arange(per_byte, device=x.device, dtype=torch.uint8) * bits
        return ((x[..., None] >> shift) & (2 ** bits - 1)).flatten(-2).float()

    kc = unpacked(part("kc", D * kb * per // 8), kb).reshape(T, pages, D * kb // 128, per, 128 // kb).transpose(2, 3)
    km = part("km", 16 * per, torch.float16).reshape(T, pages * per, D // 32, 2).float()
    vc = unpacked(part("vc", D * per * vb // 8), vb).reshape(T, pages, D, per).transpose(2, 3)
    vm = part("vm", 16 * per, torch.float16).reshape(T, pages, D // 32, per, 2).transpose(2, 3).float()
    k = kc.reshape(T, pages * per, D // 32, 32) * km[..., :1] + km[..., 1:]
    v = vc.reshape(T, pages * per, D // 32, 32) * vm.reshape(T, pages * per, D // 32, 2)[..., :1] + \
        vm.reshape(T, pages * per, D // 32, 2)[..., 1:]
    there = torch.arange(pages * per, device=ids.device)[None] < cache.len[:, sec:sec + 1]
    return (k.reshape(T, pages * per, D), v.reshape(T, pages * per, D),
            part("pos", 4 * per, torch.int32).reshape(T, pages * per), ids, there,
            part("score", 4 * per, torch.float32).reshape(T, pages * per))


def _padded(s, x):
    """Rows of x [rows, heads, ...] as [sequences, longest, heads, ...], and where they are."""
    n = s["new_len"].long()
    at = (n.cumsum(0) - n)[:, None] + torch.arange(s["longest"], device=x.device)[None]
    return x[at.clamp(max=x.shape[0] - 1)]


def _unpadded(s, x, rows):
    """The inverse: [sequences, longest, ...] back to rows."""
    n = s["new_len"].long()
    end = n.cumsum(0)
    row = torch.arange(rows, device=x.device)
    b = torch.searchsorted(end, row, right=True)
    return x[b, row - (end - n)[b]]


def _plain_logits(s):
    """Scores [tables, longest, G, tokens] of every new token, -inf where a key is not seen; values;
    the two sections."""
    c, cache = s["case"], s["cache"]
    B, H, G, n = c["B"], c["Hkv"], c["Hq"] // c["Hkv"], s["longest"]
    T = B * H
    high, low = _section(s, 0), _section(s, 1)
    k_new, v_new = (_padded(s, s[x]).float().transpose(1, 2).reshape(T, n, D) for x in ("k", "v"))
    keys = torch.cat([high[0], low[0], k_new], 1)
    values = torch.cat([high[1], low[1], v_new], 1)
    step = torch.arange(n, device=keys.device)
    first = cache.seq_len.long().repeat_interleave(H)[:, None]
    pos = torch.cat([high[2].long(), low[2].long(), first + step], 1)
    there = torch.cat([high[4], low[4], step[None] < s["new_len"].repeat_interleave(H)[:, None]], 1)
    q = _padded(s, s["q"]).float().reshape(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(T, n * G, D)
    x = torch.bmm(q, keys.transpose(1, 2).contiguous()).reshape(T, n, G, -1).mul_(SCALE)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    far = (first + step)[:, :, None] - pos[:, None, :]  # [tables, longest, tokens]
    if s["slopes"] is not None:
        x -= s["slopes"].reshape(H, G).repeat(B, 1)[:, None, :, None] * far[:, :, None].float()
    seen = there[:, None] & (far >= 0)
    if c["window"]:
        seen &= far < c["window"]
    return x.masked_fill_(~seen[:, :, None], -math.inf), values, high, low


def _plain_attention(s):
    c = s["case"]
    B, H, n = c["B"], c["Hkv"], s["longest"]
    x, values, _, _ = _plain_logits(s)
    top = x.amax(3, keepdim=True).clamp_(min=-1e30)  # a padding row of a sequence without new tokens has no key
    p = x.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    out = torch.bmm(p.reshape(B * H, -1, p.shape[3]), values).reshape(B, H, n, -1, D) / total.reshape(B, H, n, -1, 1)
    lse = (top + total.log()).reshape(B, H, n, -1)
    rows = s["q"].shape[0]
    return (_unpadded(s, out.transpose(1, 2), rows).reshape(rows, -1, D).half(),
            _unpadded(s, lse.transpose(1, 2), rows).reshape(rows, -1))


def _plain_score(s):
    c, cache = s["case"], s["cache"]
    B, H, n = c["B"], c["Hkv"], s["longest"]
    x, _, high, low = _plain_logits(s)
    lse = _padded(s, s["lse"]).reshape(B, n, H, -1).transpose(1, 2).reshape(B * H, n, -1, 1)
    x = x.sub_(lse).exp_().amax(2)
    mine = torch.arange(n, device=x.device)[None] < s["new_len"].repeat_interleave(H)[:, None]
    x = torch.where(mine[:, :, None], x, 0.0).sum(1)
    new = s["new_len"].repeat_interleave(H)[:, None].float()
    total = (cache.seq_len + s["new_len"]).repeat_interleave(H)[:, None]
    n_high = high[0].shape[1]
    n_kept = n_high + low[0].shape[1]
    _put_scores(s, 0, high, x[:, :n_high], new, total)
    _put_scores(s, 1, low, x[:, n_high:n_kept], new, total)
    received = (new - torch.arange(n, device=x.device)[None]).clamp(min=1.0)
    score = (x[:, n_kept:] / received).reshape(B, H, n).transpose(1, 2)
    return {"score": _unpadded(s, score, s["q"].shape[0]), "cached": s["views"]}


def _put_scores(s, sec, section, x, new, total):
    _, _, pos, ids, there, old = section
    per, o = LAYOUTS[s["case"]["layout"]][sec][2], _offsets(s["case"])[0][sec]["score"]
    now = old + (x - new * old) / (total - pos).clamp(min=1).float()
    now = torch.where(there, now, old).reshape(-1, per).contiguous()
    s["cache"].pool[ids.reshape(-1), o:o + 4 * per] = now.view(torch.uint8)


_RUN_OWN = {"rotate": _own_rotate, "attend": _own_attend, "score": _own_score}
_RUN_PLAIN = {"rotate": _plain_rotate, "attend": _plain_attention, "score": _plain_score}


# ---- what a pass cannot do without ------------------------------------------------------------


def work(case):
    if case["kind"] == "rotate":
        values = case["rows"] * (case["Hq"] + case["Hkv"]) * D
        return {"bytes": 4.0 * values + 4 * case["rows"], "flops": 3.0 * values * case["rot"] / D}
    seen, new = _lens(case)
    kept = _kept(case, seen).reshape(case["B"], case["Hkv"], 2).sum(1).tolist()
    fmt, G, H = LAYOUTS[case["layout"]], case["Hq"] // case["Hkv"], case["Hkv"]
    attend = case["kind"] == "attend"
    total, pairs, positions = 0.0, 0.0, bool(case["window"] or case["slopes"]) or not attend
    for n, L, (hi, lo) in zip(new, seen, kept):
        if not n:
            continue
        W = case["window"] or L + n
        # kept tokens that some new token sees, and pairs of a new token and one that it sees
        part = min(1.0, (W - 1) / L) if L else 0.0
        hi, lo = hi * part, lo * part
        for count, (kb, vb, T) in ((hi, fmt[0]), (lo, fmt[1])):
            total += count * (D * kb // 8 + 16 + (D * vb // 8 + 16 if attend else 8) + 4 / T + (4 if positions else 0))
        pairs += n * (hi + lo) + H * sum(min(j + 1, W) for j in range(n))
        rows = n * H * D * 2
        total += rows * (2 * G + 2 if attend else G + 1) + 4 * n * G * H + (0 if attend else 4 * n * H)
    return {"bytes": total, "flops": (4.0 if attend else 2.0) * D * G * pairs}


# ---- the same in 64 bits, a table at a time ---------------------------------------------------------


def _exact_tables(case, seed):
    """Per table: its sequence, rows, KV head, and for its query heads [G, rows, tokens] the scores in
    64 bits over the kept tokens (high, then low) and the new ones; values; where the kept ones are."""
    _, tokens, _, _ = _filled(case, seed)
    seen, new = _lens(case)
    q, k, v = _rows(case, seed)
    G, H = case["Hq"] // case["Hkv"], case["Hkv"]
    slopes = _slopes(case)
    bounds = [torch.searchsorted(t[0].contiguous(), torch.arange(case["B"] * H + 1, device="cuda")).tolist()
              for t in tokens]

    def real(codes, meta):
        m = meta.double().repeat_interleave(32, 1)
        return codes.double() * m[:, :, 0] + m[:, :, 1]

    row = 0
    for b, n in enumerate(new):
        for h in range(H if n else 0):
            at = [slice(e[b * H + h], e[b * H + h + 1]) for e in bounds]
            keys = torch.cat([real(t[4][i], t[5][i]) for t, i in zip(tokens, at)] + [k[row:row + n, h].double()])
            vals = torch.cat([real(t[6][i], t[7][i]) for t, i in zip(tokens, at)] + [v[row:row + n, h].double()])
            mine = seen[b] + torch.arange(n, device="cuda")
            pos = torch.cat([t[1][i] for t, i in zip(tokens, at)] + [mine])
            x = torch.matmul(q[row:row + n, h * G:(h + 1) * G].double().transpose(0, 1), keys.t()) * SCALE
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            away = mine[:, None] - pos[None]
            if slopes is not None:
                x = x - slopes[h * G:(h + 1) * G].double()[:, None, None] * away
            hidden = (away < 0) | (away >= case["window"]) if case["window"] else away < 0
            yield b, row, n, h, x.masked_fill(hidden, -math.inf), vals, at
        row += n


def _exact_attend(case, seed):
    rows, G = sum(_lens(case)[1]), case["Hq"] // case["Hkv"]
    out = torch.empty((rows, case["Hq"], D), dtype=torch.float64, device="cuda")
    lse = torch.empty((rows, case["Hq"]), dtype=torch.float64, device="cuda")
    for _, row, n, h, x, vals, _ in _exact_tables(case, seed):
        norm = torch.logsumexp(x, 2)
        out[row:row + n, h * G:(h + 1) * G] = torch.matmul(torch.exp(x - norm[..., None]), vals).transpose(0, 1)
        lse[row:row + n, h * G:(h + 1) * G] = norm.t()
    return out, lse


def _exact_score(case, seed):
    s = prepare(case, seed)
    _, tokens, _, _ = _filled(case, seed)
    seen, new = _lens(case)
    G = case["Hq"] // case["Hkv"]
    cached = [x.double() for x in s["views"]]
    first = (0, cached[0].shape[0])
    score = torch.empty((sum(new), case["Hkv"]), dtype=torch.float64, device="cuda")
    for b, row, n, h, x, _, at in _exact_tables(case, seed):
        norm = s["lse"][row:row + n, h * G:(h + 1) * G].double().t()
        got = torch.exp(x - norm[..., None]).amax(0).sum(0)
        done = 0
        for sec in (0, 1):
            t, i = tokens[sec], at[sec]
            count = i.stop - i.start
            old = t[8][i].double()
            cached[sec][t[2][i] - first[sec], t[3][i]] = \
                old + (got[done:done + count] - n * old) / (seen[b] + n - t[1][i])
            done += count
        score[row:row + n, h] = got[done:] / torch.arange(n, 0, -1, device="cuda")
    return {"score": score, "cached": tuple(cached)}


def exact(case, seed):
    return {"rotate": _exact_rotate, "attend": _exact_attend, "score": _exact_score}[case["kind"]](case, seed)
