"""What surrounds the serving operators in a decoding step and in a prompt of images: what
it costs and how its results are checked.

* ``norm``: the residual's addition and the norm (root mean square) of whole rows, with an
  output in 16 bits (``rms_norm``) or in E4M3 with scales (``rms_norm_fp8``);
* ``axes``: head norms with a rotation by positions of several axes (time, height, width),
  ``qk_norm_rope`` and ``qk_norm_rope_append`` with ``positions``;
* ``shared``: attention of one new token per sequence over a paged cache whose first tokens
  all sequences share (``decode_shared``).

``listed()`` names the cases, ``draw(rng)`` gives one more of the same ranges.  With
``own`` false, ``run`` computes the operators in elementary torch operations in 32
bits; with ``own`` true, it calls the package.  ``exact`` gives the results in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6
E4M3_MAX = 448.0
LEAST_SCALE = 2.0 ** -126   # of a row or group, zeros among them


# ------------------------------------------------------------------ the cases

def _norm(name, dtype, rows, width, residual, out, group=0, padding=0):
    """out: "same" (the inputs' type), or E4M3 with one scale a row ("row"), one a group of
    columns ("group"), or one given for all ("fixed").  padding: columns between x's rows."""
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "width": width,
            "residual": residual, "out": out, "group": group, "padding": padding}


def _axes(name, dtype, cache, B, N, H, Hkv, d, rotary, axes, alternating, shortest, start, layout,
          page=16, cache_layout="bhnd", interleaved=False):
    """cache: "" (q and k alone), or the type of the cache that keys and values go to.
    alternating: the axes take the pairs in turn, else a run of pairs each."""
    return {"name": name, "op": "axes", "dtype": dtype, "cache": cache, "B": B, "N": N, "H": H,
            "Hkv": Hkv, "d": d, "rotary": rotary, "axes": axes, "alternating": alternating,
            "shortest": shortest, "longest": N, "start": start, "layout": layout, "page": page,
            "cache_layout": cache_layout, "interleaved": interleaved}


def _shared(name, dtype, cache, B, H, Hkv, d, prefix, shortest, longest, free, page, cache_layout):
    """shortest to longest tokens of a sequence's own after the prefix; free: one slot of
    the batch holds no sequence."""
    return {"name": name, "op": "shared", "dtype": dtype, "cache": cache, "B": B, "H": H,
            "Hkv": Hkv, "d": d, "prefix": prefix, "shortest": shortest, "longest": longest,
            "free": free, "page": page, "cache_layout": cache_layout}


def listed():
    return [
        # one token between two layers: latency
        _norm("norm_token_bf16", "bf16", 1, 4096, True, "same"),
        # one token of each of 64 sequences before an FP8 product with a scale a row
        _norm("norm_tokens_fp8", "bf16", 64, 8192, True, "row"),
        # a long prompt between two layers, 16 bits in and out
        _norm("norm_prompt_bf16", "bf16", 8192, 8192, True, "same"),
        # a part of a wider projection, an odd count of rows, a scale for 128 columns each
        _norm("norm_groups_f16", "f16", 4097, 5120, False, "group", 128, 640),
        # one new token of each of 64 conversations with pictures in them
        _axes("axes_tokens_bf16", "bf16", "bf16", 64, 1, 64, 8, 128, 128, 3, False, 1, 500, "bnhd", 64),
        # a prompt that is mostly one large picture
        _axes("axes_picture_bf16", "bf16", "", 1, 8192, 64, 8, 128, 128, 3, False, 8192, 0, "bnhd"),
        # a padded batch of film prompts into FP8 pages, axes in turn over the pairs
        _axes("axes_films_fp8", "f16", "e4m3", 4, 1999, 32, 8, 128, 128, 3, True, 777, 0, "bhnd", 16),
        # the next tokens of four answers to one question: latency
        _shared("shared_answers_bf16", "bf16", "bf16", 4, 32, 8, 128, 2048, 1, 100, False, 16, "bhnd"),
        # 64 conversations, a free slot among them, behind the same instructions
        _shared("shared_batch_bf16", "bf16", "bf16", 64, 64, 8, 128, 8192, 1, 1000, True, 64, "bhnd"),
        # 16 questions about one long document in an FP8 cache, its length no multiple of a page
        _shared("shared_document_fp8", "bf16", "e4m3", 16, 64, 8, 128, 65500, 1, 500, False, 128, "bhnd"),
        # one shared key/value head of narrow rows
        _shared("shared_one_head_f16", "f16", "f16", 32, 16, 1, 64, 16384, 0, 300, False, 32, "bnhd"),
        # many long conversations behind one long prefix
        _shared("shared_long_bf16", "bf16", "bf16", 128, 32, 8, 128, 16384, 1, 4096, False, 64, "bnhd"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """A case of the same ranges: one row to 8192 of 64 to 16384 columns, one token to 8192
    of one to four axes, prefixes of one token to 65536, every type, width, page and layout."""
    op = rng.choice(("norm", "axes", "shared"))
    dtype = rng.choice(("f16", "bf16", "bf16"))
    if op == "norm":
        out = rng.choice(("same", "row", "group", "fixed"))
        group = rng.choice((32, 64, 128, 256)) if out == "group" else 0
        width = 8 * _log(rng, 8, 2048)
        if group:
            width = max(group, width - width % group)
        case = _norm("", dtype, 1 if rng.random() < 0.2 else _log(rng, 2, 65536), width,
                     rng.random() < 0.6, out, group, 8 * rng.choice((0, 0, 1, 80)))
        size = "rows"
    else:
        d = rng.choice((64, 128, 128))
        H = rng.choice((8, 16, 32, 40, 64))
        Hkv = max(1, H // rng.choice((1, 4, 8, 16)))
        H -= H % Hkv
        cache_layout = rng.choice(("bhnd", "bnhd"))
        cache = rng.choice((dtype, dtype, "e4m3"))
        page = rng.choice((16, 32, 48, 64, 128, 256))
        B = _log(rng, 1, 128 if op == "shared" else 64)
    if op == "axes":
        N = 1 if rng.random() < 0.3 else _log(rng, 2, 8192)
        B = max(1, min(B, 8192 // N))
        case = _axes("", dtype, rng.choice(("", cache)), B, N, H, Hkv, d, d if rng.random() < 0.7 else d // 2,
                     rng.choice((1, 2, 3, 3, 4)), rng.random() < 0.4,
                     rng.randint(1, N) if rng.random() < 0.5 else N, rng.choice((0, rng.randint(1, 4000))),
                     rng.choice(("bhnd", "bnhd")), page, cache_layout, rng.random() < 0.3)
        size = "N"
    elif op == "shared":
        longest = rng.choice((0, _log(rng, 1, 4096), _log(rng, 1, 4096)))
        case = _shared("", dtype, cache, B, H, Hkv, d, _log(rng, 1, 65536), rng.randint(0, longest), longest,
                       B > 1 and rng.random() < 0.3, page, cache_layout)
        size = "prefix"
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while _cost(case) > most or _held(case) > 3e9:
        if op == "shared" and case["longest"] * B > case["prefix"]:
            case["longest"] -= case["longest"] // 8 + 1
            case["shortest"] = min(case["shortest"], case["longest"])
            continue
        case[size] -= case[size] // 8 + 1
        if op == "axes":
            case["longest"] = case["N"]
            case["shortest"] = min(case["shortest"], case["N"])
    del case["name"]
    return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 100)


def _held(case):
    """Bytes of a shared case's cache, own pages among them."""
    if case["op"] != "shared":
        return 0
    return (2 * (case["prefix"] + case["B"] * (case["longest"] + case["page"])) * case["Hkv"] * case["d"]
            * _bytes(case["cache"]))


def _bytes(dtype):
    return 1 if dtype == "e4m3" else 2


def _between(case):
    """One number per sequence, from shortest to longest in mixed order."""
    B, low, high = case["B"], case["shortest"], case["longest"]
    return [high - (high - low) * ((i * 5) % B) // max(1, B - 1) for i in range(B)]


def _lengths(case):
    """Cached tokens of each sequence of a shared case, prefix and own."""
    lengths = [case["prefix"] + n for n in _between(case)]
    if case["free"]:
        lengths[case["B"] // 2] = 0
    return lengths


def work(case):
    """Each input read once (rows that hold a token, angles once a token, cached tokens that
    are seen, the prefix once for all), each output written once."""
    op = case["op"]
    if op == "norm":
        rows, width = case["rows"], case["width"]
        moved = rows * width * (2 + (4 if case["residual"] else 0) + (2 if case["out"] == "same" else 1))
        moved += 2 * width + 4 * rows * _scales_of(case)
        return {"bytes": moved, "flops": rows * width * (5 if case["out"] == "same" else 8)}
    d, H, Hkv, B = case["d"], case["H"], case["Hkv"], case["B"]
    if op == "axes":
        tokens, rows = sum(_between(case)), B * case["N"]
        moved = 4 * (case["rotary"] + case["axes"]) * tokens
        if case["cache"]:
            moved += 2 * d * (H * (tokens + rows) + 2 * Hkv * tokens) + 2 * Hkv * d * tokens * _bytes(case["cache"])
        else:
            moved += 2 * d * (H + Hkv) * (tokens + rows)
        return {"bytes": moved, "flops": tokens * (H + Hkv) * (4 * d + 3 * case["rotary"])}
    lengths = _lengths(case)
    new = sum(max(0, n - case["prefix"]) for n in lengths)
    moved = (2 * (case["prefix"] + new) * Hkv * d * _bytes(case["cache"]) + B * H * (4 * d + 4)
             + 4 * ((case["prefix"] + new) // case["page"] + 2 * B))
    return {"bytes": moved, "flops": 4 * sum(lengths) * H * d}


def _scales_of(case):
    """Scales of a row that a norm writes."""
    return {"same": 0, "fixed": 0, "row": 1}.get(case["out"]) if case["out"] != "group" else case["width"] // case["group"]


# ---------------------------------------------------------------- the inputs

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(case):
    """Tokens that each sequence has before this call, up to start."""
    return [case["start"] * (i + 1) // case["B"] for i in range(case["B"])]


def _axis_of_pair(case):
    """The axis that turns each pair: in turn, or a run each (the first axis the shortest)."""
    half, axes = case["rotary"] // 2, case["axes"]
    if case["alternating"]:
        return [j % axes for j in range(half)]
    first = half // 4 if axes > 1 else half
    return [0 if j < first else 1 + (j - first) * (axes - 1) // (half - first) for j in range(half)]


def _positions(case):
    """[axes, B, N] positions: text, whose axes go together, then frames of a square
    picture, row by row, each frame one step on in time; -1 where no token is."""
    at = torch.full((case["axes"], case["B"], case["N"]), -1, dtype=torch.int32, device="cuda")
    for b, (start, n) in enumerate(zip(_starts(case), _between(case))):
        t = torch.arange(n, device="cuda", dtype=torch.int32)
        text = n // 8
        side = max(1, min(64, math.isqrt(max(1, n - text))))
        spot = t - text
        place = (spot // (side * side), spot // side % side, spot % side, spot // (4 * side * side))
        for a in range(case["axes"]):
            at[a, b, :n] = start + torch.where(t < text, t, text + place[a])
    return at


def _angles(case):
    """cos and sin [positions, rotary / 2] of base 10000, formed in 64 bits."""
    half = case["rotary"] // 2
    rate = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    at = torch.arange(case["start"] + case["N"] + 64, dtype=torch.float64, device="cuda")
    phase = at[:, None] * rate
    return phase.cos().float(), phase.sin().float()


def _pages(case, first, tokens, gen, spare):
    """Page table of sequences that hold tokens first .. tokens[b] - 1, its pages in random
    order among spare others; entries that are not in use are -1.  And the pages in all."""
    page, low = case["page"], first // case["page"]
    high = [(n + page - 1) // page if n > first else low for n in tokens]
    width = max(1, max(high))
    pages = sum(h - low for h in high) + spare
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device="cuda")
    at = spare
    for b, h in enumerate(high):
        table[b, low:h] = order[at:at + h - low]
        at += h - low
    return table, order[:spare], pages


def _cache_shape(case, pages):
    if case["cache_layout"] == "bnhd":
        return (pages, case["page"], case["Hkv"], case["d"])
    return (pages, case["Hkv"], case["page"], case["d"])


def _shape(case, heads):
    if case["layout"] == "bnhd":
        return (case["B"], case["N"], heads, case["d"])
    return (case["B"], heads, case["N"], case["d"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(*shape, dtype=dtype):
        if dtype == torch.float8_e4m3fn:   # codes of values spread over the type's middle
            return (torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)
                    .mul_(32).to(dtype))
        return torch.randn(*shape, generator=gen, device="cuda", dtype=dtype)

    s = {"case": case}
    op = case["op"]
    if op == "norm":
        rows, width = case["rows"], case["width"]
        s["x"] = normal(rows, width + case["padding"])[:, :width]
        # the stream between layers has grown larger than what a layer adds
        s["residual"] = normal(rows, width).mul_(4) if case["residual"] else None
        s["weight"] = (1 + 0.2 * normal(width)).to(dtype)
        s["scale"] = 1 / 64
        return s
    H, Hkv, B, d = case["H"], case["Hkv"], case["B"], case["d"]
    if op == "shared":
        lengths, prefix = _lengths(case), case["prefix"]
        s["q"] = normal(B, H, d)
        shared = (prefix + case["page"] - 1) // case["page"]
        s["table"], s["prefix_table"], pages = _pages(case, prefix, lengths, gen, shared)
        s["lengths"] = _ints(lengths)
        s["k_cache"], s["v_cache"] = (normal(*_cache_shape(case, pages), dtype=TYPES[case["cache"]])
                                      for _ in range(2))
        s["scales"] = (1 / 32, 1 / 40) if case["cache"] == "e4m3" else (1.0, 1.0)
        return s
    counts, starts = _between(case), _starts(case)
    # activations of uneven sizes, as a projection gives them
    s["q"], s["k"], s["v"] = (normal(*_shape(case, heads)).mul_(3) for heads in (H, Hkv, Hkv))
    s["q_weight"], s["k_weight"] = ((1 + 0.2 * normal(d)).to(dtype) for _ in range(2))
    s["cos"], s["sin"] = _angles(case)
    s["axis"], s["positions"] = tuple(_axis_of_pair(case)), _positions(case)
    s["starts"], s["counts"] = _ints(starts), _ints(counts)
    if case["cache"]:
        s["table"], _, pages = _pages(case, 0, [a + n for a, n in zip(starts, counts)], gen, 0)
        s["scales"] = (1 / 32, 1 / 24) if case["cache"] == "e4m3" else (1.0, 1.0)
        # a page more at the end, that no table names
        s["whole"] = [normal(*_cache_shape(case, pages + 1), dtype=TYPES[case["cache"]])
                      for _ in range(2)]
        s["k_cache"], s["v_cache"] = (w[:-1] for w in s["whole"])
    return s


# ------------------------------------------------------ the operators, plainly

def _plain_norm(s):
    case = s["case"]
    x = s["x"].float()
    if case["residual"]:
        x = x + s["residual"].float()
    y = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * s["weight"].float()
    total = x.to(s["x"].dtype) if case["residual"] else None
    if case["out"] == "same":
        return y.to(s["x"].dtype), total
    if case["out"] == "fixed":
        return (y / s["scale"]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), None, total
    groups = y.view(case["rows"], _scales_of(case), -1)
    scales = (groups.abs().amax(dim=-1) / E4M3_MAX).clamp(min=LEAST_SCALE)
    codes = (groups / scales[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return codes.view(y.shape), scales, total


def _by_token(t, layout):
    """[B, N, heads, width], whatever the layout."""
    return t if layout == "bnhd" else t.transpose(1, 2)


def _norm_rope(s, x, weight, held):
    """x [B, N, heads, d] normalised and rotated, in 32 bits; zero where no token is."""
    case = s["case"]
    R, half = case["rotary"], case["rotary"] // 2
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    rows = s["positions"].clamp(min=0).long()[list(s["axis"])].movedim(0, -1)   # [B, N, half]
    pair = torch.arange(half, device="cuda")
    cos, sin = (t[rows, pair][:, :, None] for t in (s["cos"], s["sin"]))
    turned, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((turned, rest), dim=-1) * held[:, :, None, None]


def _plain_axes(s):
    case = s["case"]
    t = torch.arange(case["N"], device="cuda")
    held = t[None] < s["counts"][:, None]
    q = _norm_rope(s, _by_token(s["q"], case["layout"]), s["q_weight"], held)
    k = _norm_rope(s, _by_token(s["k"], case["layout"]), s["k_weight"], held)
    q = _by_token(q, case["layout"]).to(s["q"].dtype).contiguous()
    if not case["cache"]:
        return q, _by_token(k, case["layout"]).to(s["k"].dtype).contiguous()
    page = case["page"]
    at = torch.where(held, s["starts"][:, None] + t, 0).long()
    pages = torch.gather(s["table"].long(), 1, at // page)
    spare = s["whole"][0].shape[0] - 1   # rows without a token are written there
    pages, inside = torch.where(held, pages, spare), torch.where(held, at % page, 0)
    _put(case, s["whole"][0], pages, inside, k / s["scales"][0])
    _put(case, s["whole"][1], pages, inside, _by_token(s["v"], case["layout"]).float() / s["scales"][1])
    return q, s["k_cache"], s["v_cache"]


def _put(case, cache, pages, inside, rows):
    rows = (rows.clamp(-E4M3_MAX, E4M3_MAX) if case["cache"] == "e4m3" else rows).to(cache.dtype)
    if case["cache"] == "e4m3":
        cache, rows = cache.view(torch.uint8), rows.view(torch.uint8)
    if case["cache_layout"] == "bnhd":
        cache[pages, inside] = rows
    else:
        cache.transpose(1, 2)[pages, inside] = rows


def _gathered(case, cache, table, scale):
    """[..., Hkv, tokens, d] in 32 bits of the pages that a table [..., columns] names."""
    rows = cache.view(torch.uint8)[table] if case["cache"] == "e4m3" else cache[table]
    rows = rows.view(cache.dtype).float() * scale
    if case["cache_layout"] == "bnhd":
        return rows.flatten(-4, -3).transpose(-3, -2)
    return rows.transpose(-4, -3).flatten(-3, -2)


def _plain_shared(s):
    """Scores against the prefix for all queries of a head at once, and against each
    sequence's own tokens; one softmax over both."""
    case = s["case"]
    B, H, Hkv, d, prefix = case["B"], case["H"], case["Hkv"], case["d"], case["prefix"]
    G, low = H // Hkv, prefix // case["page"]
    caches = tuple(zip((s["k_cache"], s["v_cache"]), s["scales"]))
    pk, pv = (_gathered(case, c, s["prefix_table"].long(), f)[:, :prefix] for c, f in caches)
    table = s["table"][:, low:].long().clamp(min=0)
    ok, ov = (_gathered(case, c, table, f) for c, f in caches)
    at, n = low * case["page"] + torch.arange(ok.shape[2], device="cuda")[None], s["lengths"][:, None]
    seen = (at >= prefix) & (at < n)
    q = s["q"].float().view(B, Hkv, G, d) * (1.0 / d ** 0.5)
    by_head = q.transpose(0, 1).reshape(Hkv, B * G, d)
    first = torch.matmul(by_head, pk.transpose(1, 2)).view(Hkv, B, G, prefix).transpose(0, 1)
    rest = torch.where(seen[:, None, None], torch.matmul(q, ok.transpose(2, 3)), -math.inf)
    top = first.amax(dim=-1, keepdim=True)
    if rest.shape[3]:
        top = torch.maximum(top, rest.amax(dim=-1, keepdim=True))
    p, r = torch.exp(first - top), torch.exp(rest - top)
    total = p.sum(dim=-1, keepdim=True) + r.sum(dim=-1, keepdim=True)
    o = torch.matmul(p.transpose(0, 1).reshape(Hkv, B * G, prefix), pv).view(Hkv, B, G, d).transpose(0, 1)
    o = (o + torch.matmul(r, torch.where(seen[:, None, :, None], ov, 0.0))) / total
    lse = top + torch.log(total)
    none = (n == 0)[:, None, :, None]
    o, lse = torch.where(none, 0.0, o), torch.where(none, -math.inf, lse)
    return o.reshape(B, H, d).to(s["q"].dtype), lse.reshape(B, H)


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return (_plain_norm if op == "norm" else _plain_axes if op == "axes" else _plain_shared)(s)
    import paper_2506_12355_amd as qa
    if op == "norm":
        if case["out"] == "same":
            return qa.rms_norm(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        return qa.rms_norm_fp8(s["x"], s["weight"], residual=s["residual"], eps=EPS,
                               scale=s["scale"] if case["out"] == "fixed" else None,
                               group=case["group"] or None)
    if op == "axes":
        how = dict(cos=s["cos"], sin=s["sin"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                   counts=s["counts"], positions=s["positions"], axes=s["axis"],
                   interleaved=case["interleaved"], layout=case["layout"])
        if not case["cache"]:
            return qa.qk_norm_rope(s["q"], s["k"], **how)
        q = qa.qk_norm_rope_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"],
                                   s["starts"], k_scale=s["scales"][0], v_scale=s["scales"][1],
                                   cache_layout=case["cache_layout"], **how)
        return q, s["k_cache"], s["v_cache"]
    return qa.decode_shared(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"],
                            s["prefix_table"], case["prefix"], k_scale=s["scales"][0],
                            v_scale=s["scales"][1], cache_layout=case["cache_layout"])


# ------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "axes": _exact_axes, "shared": _exact_shared}[case["op"]](s)


def _exact_norm(s):
    case = s["case"]
    rows, width = case["rows"], case["width"]
    sums, outs, scales = [], [], []
    for lo in range(0, rows, 1024):
        x = s["x"][lo:lo + 1024].double()
        if case["residual"]:
            x += s["residual"][lo:lo + 1024].double()
            sums.append(x)
        y = x / torch.sqrt(x.square().sum(dim=1, keepdim=True) / width + EPS) * s["weight"].double()
        if case["out"] == "fixed":
            y = (y / s["scale"]).clamp(-E4M3_MAX, E4M3_MAX)
        elif case["out"] != "same":
            parts = y.reshape(-1, case["group"] or width)
            f = torch.clamp(parts.abs().max(dim=1).values / E4M3_MAX, min=LEAST_SCALE)
            y = (parts / f[:, None]).reshape(y.shape)
            scales.append(f.view(x.shape[0], -1))
        outs.append(y)
    total = torch.cat(sums) if sums else None
    if case["out"] == "same":
        return torch.cat(outs), total
    return torch.cat(outs), torch.cat(scales) if scales else None, total


def _exact_axes(s):
    """The rotation as a product of complex numbers, pair by pair of its axis' position."""
    case = s["case"]
    R, layout = case["rotary"], case["layout"]
    starts, counts = _starts(case), _between(case)

    def turned(x, weight):
        out = torch.zeros_like(x, dtype=torch.float64)
        for b, n in enumerate(counts):
            y = x[b, :n].double()
            y = y / torch.sqrt(y.square().sum(dim=-1, keepdim=True) / case["d"] + EPS) * weight.double()
            for j, a in enumerate(s["axis"]):
                at = s["positions"][a, b, :n].long()
                unit = torch.complex(s["cos"][at, j].double(), s["sin"][at, j].double())[:, None]
                c0, c1 = (2 * j, 2 * j + 1) if case["interleaved"] else (j, j + R // 2)
                z = torch.complex(y[..., c0], y[..., c1]) * unit
                y[..., c0], y[..., c1] = z.real, z.imag
            out[b, :n] = y
        return out

    q = turned(_by_token(s["q"], layout), s["q_weight"])
    k = turned(_by_token(s["k"], layout), s["k_weight"])
    if not case["cache"]:
        return _by_token(q, layout).contiguous(), _by_token(k, layout).contiguous()
    caches = []
    for cache, rows, f in ((s["k_cache"], k, s["scales"][0]),
                           (s["v_cache"], _by_token(s["v"], layout).double(), s["scales"][1])):
        values = cache.float().double()
        by_slot = values if case["cache_layout"] == "bnhd" else values.transpose(1, 2)
        for b in range(case["B"]):
            at = torch.arange(starts[b], starts[b] + counts[b], device="cuda")
            new = rows[b, :counts[b]] / f
            by_slot[s["table"][b, at // case["page"]].long(), at % case["page"]] = (
                new.clamp(-E4M3_MAX, E4M3_MAX) if case["cache"] == "e4m3" else new)
        caches.append(values)
    return _by_token(q, layout).contiguous(), caches[0], caches[1]


def _exact_shared(s):
    """Sequence by sequence, over its tokens in order, with 64-bit scores and weights."""
    case = s["case"]
    B, H, Hkv, d, page, prefix = (case[x] for x in ("B", "H", "Hkv", "d", "page", "prefix"))
    G = H // Hkv
    o = torch.zeros((B, H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")

    def tokens(cache, pages, f):
        t = cache.view(torch.uint8)[pages].view(cache.dtype) if case["cache"] == "e4m3" else cache[pages]
        t = t.float() if case["cache_layout"] == "bnhd" else t.float().permute(0, 2, 1, 3)
        return t.reshape(-1, Hkv, d).permute(1, 0, 2).double() * f   # [Hkv, tokens, d]

    both = tuple(zip((s["k_cache"], s["v_cache"]), s["scales"]))
    pk, pv = (tokens(c, s["prefix_table"].long(), f)[:, :prefix].contiguous() for c, f in both)
    low = prefix // page
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        pages = s["table"][b, low:(n + page - 1) // page if n > prefix else low].long()
        k, v = (tokens(c, pages, f)[:, prefix - low * page:n - low * page].contiguous() if n > prefix
                else p[:, :0] for (c, f), p in zip(both, (pk, pv)))
        q = s["q"][b].double().view(Hkv, G, d)
        x = torch.cat((torch.matmul(q, pk.transpose(1, 2)), torch.matmul(q, k.transpose(1, 2))), dim=2) * d ** -0.5
        total = torch.logsumexp(x, dim=2)
        w = torch.exp(x - total[:, :, None])
        o[b] = (torch.matmul(w[:, :, :prefix], pv) + torch.matmul(w[:, :, prefix:], v)).view(H, d)
        lse[b] = total.view(H)
    return o, lse
