"""The operators around the attention forward that serve a model: what they cost and
how their results are checked.

* ``rope``: each head of q and k normalised (root mean square) and rotated by its
  token's position (``qk_norm_rope``);
* ``append``: the same, with the keys and values written into the pages of a cache
  (``qk_norm_rope_append``);
* ``decode``: attention of one new token per sequence over such a cache (``decode``);
* ``window``: attention of a whole prompt with a sliding window and a few first tokens
  that stay visible (``fwd_window``).

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


# ------------------------------------------------------------------ the cases

def _rope(name, dtype, B, N, H, Hkv, d, rotary, shortest, start, layout, interleaved=False):
    return {"name": name, "op": "rope", "dtype": dtype, "B": B, "N": N, "H": H, "Hkv": Hkv,
            "d": d, "rotary": rotary, "shortest": shortest, "longest": N, "start": start,
            "layout": layout, "interleaved": interleaved}


def _append(name, dtype, cache, B, N, H, Hkv, d, rotary, shortest, start, page, cache_layout):
    return dict(_rope(name, dtype, B, N, H, Hkv, d, rotary, shortest, start, "bnhd"), op="append",
                cache=cache, page=page, cache_layout=cache_layout)


def _decode(name, dtype, cache, B, H, Hkv, d, shortest, longest, page, cache_layout, window=0,
            sinks=0):
    return {"name": name, "op": "decode", "dtype": dtype, "cache": cache, "B": B, "H": H,
            "Hkv": Hkv, "d": d, "shortest": shortest, "longest": longest, "page": page,
            "cache_layout": cache_layout, "window": window, "sinks": sinks}


def _window(name, dtype, B, H, Hkv, N, d, window, sinks, layout):
    return {"name": name, "op": "window", "dtype": dtype, "B": B, "H": H, "Hkv": Hkv, "N": N,
            "d": d, "dv": min(d, 128), "window": window, "sinks": sinks, "layout": layout}


def listed():
    return [
        # one new token of one sequence: latency alone
        _rope("rope_token_bf16", "bf16", 1, 1, 32, 8, 128, 128, 1, 4095, "bnhd"),
        # a prompt as the projections write it (64 query, 8 key/value heads)
        _rope("rope_prompt_bf16", "bf16", 1, 8192, 64, 8, 128, 128, 8192, 0, "bnhd"),
        # a padded batch of continued prompts, narrow heads, half of each rotated
        _rope("rope_padded_f16", "f16", 8, 777, 16, 16, 64, 32, 100, 300, "bhnd", True),
        # one new token of each of 64 sequences into a cache of the model's own type
        _append("append_tokens_bf16", "bf16", "bf16", 64, 1, 64, 8, 128, 128, 1, 500, 64, "bhnd"),
        # four prompts of odd lengths into FP8 pages, token by token
        _append("append_prompts_fp8", "bf16", "e4m3", 4, 2000, 32, 8, 128, 128, 777, 0, 16, "bnhd"),
        # the next token of one short conversation: latency
        _decode("decode_one_bf16", "bf16", "bf16", 1, 32, 8, 128, 1000, 1000, 16, "bhnd"),
        # the next tokens of 64 conversations of all lengths, a free slot among them
        _decode("decode_batch_bf16", "bf16", "bf16", 64, 64, 8, 128, 0, 8192, 64, "bhnd"),
        # the next token over one long document in an FP8 cache
        _decode("decode_document_fp8", "bf16", "e4m3", 1, 64, 8, 128, 131072, 131072, 128, "bhnd"),
        # one shared key/value head, of which a window and the first four tokens are seen
        _decode("decode_window_f16", "f16", "f16", 32, 16, 1, 64, 1000, 32768, 32, "bnhd", 4096, 4),
        # one prompt of an odd length, narrow heads, a short window
        _window("window_prompt_f16", "f16", 1, 16, 4, 1000, 64, 256, 4, "bhnd"),
        # a batch as the projections write it, window without first tokens
        _window("window_batch_bf16", "bf16", 8, 16, 16, 2048, 128, 512, 0, "bnhd"),
        # one long document
        _window("window_document_bf16", "bf16", 1, 32, 8, 16384, 128, 4096, 4, "bhnd"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """A case of the same ranges: one token to 16k (a cache: 131k), odd counts, 1 to 64
    sequences, every type, width, page size, mask and layout."""
    op = rng.choice(("rope", "append", "decode", "window"))
    dtype = rng.choice(("f16", "bf16", "bf16"))
    d = rng.choice((64, 128, 128))
    H = rng.choice((8, 16, 32, 64))
    Hkv = max(1, H // rng.choice((1, 4, 8, 16)))
    layout, cache_layout = rng.choice(("bhnd", "bnhd")), rng.choice(("bhnd", "bnhd"))
    cache = rng.choice((dtype, dtype, "e4m3"))
    page = rng.choice((16, 32, 48, 64, 128, 256))
    B = _log(rng, 1, 64)
    if op in ("rope", "append"):
        N = 1 if rng.random() < 0.3 else _log(rng, 2, 8192)
        B = max(1, min(B, 8192 // N))
        shortest = rng.randint(1, N) if rng.random() < 0.5 else N
        start = rng.choice((0, rng.randint(1, 4000)))
        rotary = d if rng.random() < 0.7 else d // 2
        if op == "rope":
            case = _rope("", dtype, B, N, H, Hkv, d, rotary, shortest, start, layout,
                         rng.random() < 0.4)
        else:
            case = _append("", dtype, cache, B, N, H, Hkv, d, rotary, shortest, start, page,
                           cache_layout)
            case["layout"] = layout
        size = "N"
    elif op == "decode":
        longest = _log(rng, 1, 131072)
        shortest = rng.randint(0, longest)
        window = _log(rng, 1, 8192) if rng.random() < 0.3 else 0
        sinks = rng.choice((0, 1, 4, 64)) if window else 0
        case = _decode("", dtype, cache, B, H, Hkv, d, shortest, longest, page, cache_layout,
                       window, sinks)
        size = "longest"
    else:
        if rng.random() < 0.15:
            d, Hkv, layout = 192, H, "bhnd"
        N = _log(rng, 16, 16384)
        case = _window("", dtype, max(1, min(B, 16384 // N)), H, Hkv, N, d, _log(rng, 8, 4096),
                       rng.choice((0, 1, 4, 64)), layout)
        size = "N"
    most = max(_cost(c) for c in listed() if c["op"] == op)
    # the paged cache as a whole (windowed or not) stays as small as the listed ones too
    while _cost(case) > most or (op == "decode" and _held(case) > 3e9):
        case[size] -= case[size] // 8 + 1
        if "shortest" in case:
            case["shortest"] = min(case["shortest"], case[size])
        if op in ("rope", "append"):
            case["longest"] = case["N"]
    del case["name"]
    return case


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def _held(case):
    return 2 * case["B"] * case["longest"] * case["Hkv"] * case["d"] * _bytes(case["cache"])


def _bytes(dtype):
    return 1 if dtype == "e4m3" else 2


def _lengths(case):
    """One length per sequence, from shortest to longest in mixed order."""
    B, low, high = case["B"], case["shortest"], case["longest"]
    return [high - (high - low) * ((i * 5) % B) // max(1, B - 1) for i in range(B)]


def _seen(case, n):
    """Cached tokens that a new token after n sees."""
    if not case["window"]:
        return n
    return min(n, case["window"] + min(case["sinks"], max(0, n - case["window"])))


def work(case):
    """Each input read once (rows of the batch that hold a token, keys that are seen,
    table rows that a token needs), each output written once."""
    op, d, H, Hkv = case["op"], case["d"], case["H"], case["Hkv"]
    if op in ("rope", "append"):
        tokens = sum(_lengths(case))
        rows = case["B"] * case["N"]
        angles = 4 * case["rotary"] * case["N"]
        if op == "rope":
            moved = 2 * d * (H + Hkv) * (tokens + rows) + angles
        else:
            moved = (2 * d * (H * (tokens + rows) + 2 * Hkv * tokens) + angles
                     + 2 * Hkv * d * tokens * _bytes(case["cache"]))
        return {"bytes": moved, "flops": tokens * (H + Hkv) * (4 * d + 3 * case["rotary"])}
    if op == "decode":
        seen = sum(_seen(case, n) for n in _lengths(case))
        moved = (2 * seen * Hkv * d * _bytes(case["cache"]) + case["B"] * H * (4 * d + 4)
                 + 4 * (seen // case["page"] + 2 * case["B"]))
        return {"bytes": moved, "flops": 4 * seen * H * d}
    N, w = case["N"], case["window"]
    pairs = sum(min(i + 1, w + min(case["sinks"], max(0, i + 1 - w))) for i in range(N))
    moved = case["B"] * N * (2 * H * (d + case["dv"]) + 2 * Hkv * (d + case["dv"]) + 4 * H)
    return {"bytes": moved, "flops": 2 * case["B"] * H * pairs * (d + case["dv"])}


# ---------------------------------------------------------------- the inputs

def _angles(case):
    """cos and sin [positions, rotary / 2] of base 10000, formed in 64 bits."""
    half = case["rotary"] // 2
    rate = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    at = torch.arange(case["start"] + case["N"] + 64, dtype=torch.float64, device="cuda")
    phase = at[:, None] * rate
    return phase.cos().float(), phase.sin().float()


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _starts(case):
    """Tokens that each sequence has before this call, up to start."""
    return [case["start"] * (i + 1) // case["B"] for i in range(case["B"])]


def _pages(case, tokens, gen):
    """Page table of a cache with room for `tokens` per sequence: pages in random order,
    a spare page at the end that no table names; unused entries are -1."""
    per = [(n + case["page"] - 1) // case["page"] for n in tokens]
    width = max(1, max(per))
    order = torch.randperm(case["B"] * width, generator=gen, device="cuda").to(torch.int32)
    table = order.view(case["B"], width)
    used = torch.arange(width, device="cuda")[None] < _ints(per)[:, None]
    return torch.where(used, table, -1), case["B"] * width


def _cache_shape(case, pages):
    if case["cache_layout"] == "bnhd":
        return (pages, case["page"], case["Hkv"], case["d"])
    return (pages, case["Hkv"], case["page"], case["d"])


def _shape(case, heads, width):
    if case["layout"] == "bnhd":
        return (case["B"], case["N"], heads, width)
    return (case["B"], heads, case["N"], width)


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
    op, d, H, Hkv, B = case["op"], case["d"], case["H"], case["Hkv"], case["B"]
    if op == "window":
        s["q"], s["k"], s["v"] = (normal(*_shape(case, heads, width)) for heads, width in
                                  ((H, d), (Hkv, d), (Hkv, case["dv"])))
        return s
    if op == "decode":
        lengths = _lengths(case)
        s["q"] = normal(B, H, d)
        s["table"], pages = _pages(case, lengths, gen)
        s["lengths"] = _ints(lengths)
        s["k_cache"], s["v_cache"] = (normal(*_cache_shape(case, pages), dtype=TYPES[case["cache"]])
                                      for _ in range(2))
        s["scales"] = (1 / 32, 1 / 40) if case["cache"] == "e4m3" else (1.0, 1.0)
        return s
    counts, starts = _lengths(case), _starts(case)
    # activations of uneven sizes, as a projection gives them
    s["q"], s["k"], s["v"] = (normal(*_shape(case, heads, d)).mul_(3) for heads in (H, Hkv, Hkv))
    s["q_weight"], s["k_weight"] = ((1 + 0.2 * normal(d)).to(dtype) for _ in range(2))
    s["cos"], s["sin"] = _angles(case)
    s["starts"], s["counts"] = _ints(starts), _ints(counts)
    if op == "append":
        s["table"], pages = _pages(case, [a + n for a, n in zip(starts, counts)], gen)
        s["scales"] = (1 / 32, 1 / 24) if case["cache"] == "e4m3" else (1.0, 1.0)
        s["whole"] = [normal(*_cache_shape(case, pages + 1), dtype=TYPES[case["cache"]])
                      for _ in range(2)]
        s["k_cache"], s["v_cache"] = (w[:-1] for w in s["whole"])
    return s


# ------------------------------------------------------ the operators, plainly

def _by_token(t, layout):
    """[B, N, heads, width], whatever the layout."""
    return t if layout == "bnhd" else t.transpose(1, 2)


def _norm_rope(s, x, weight, positions):
    """x [B, N, heads, d] normalised and rotated, in 32 bits; zero where no token is."""
    case = s["case"]
    R, half = case["rotary"], case["rotary"] // 2
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight.float()
    cos, sin = (t[positions][:, :, None] for t in (s["cos"], s["sin"]))
    turned, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = turned[..., :half], turned[..., half:]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    held = torch.arange(case["N"], device="cuda")[None] < s["counts"][:, None]
    return torch.cat((turned, rest), dim=-1) * held[:, :, None, None], held


def _plain_rope(s):
    case = s["case"]
    t = torch.arange(case["N"], device="cuda")
    positions = (s["starts"][:, None] + t).long()
    q, held = _norm_rope(s, _by_token(s["q"], case["layout"]), s["q_weight"], positions)
    k, held = _norm_rope(s, _by_token(s["k"], case["layout"]), s["k_weight"], positions)
    q = _by_token(q, case["layout"]).to(s["q"].dtype).contiguous()
    if case["op"] == "rope":
        return q, _by_token(k, case["layout"]).to(s["k"].dtype).contiguous()
    page = case["page"]
    where = torch.where(held, positions, 0)
    pages = torch.gather(s["table"].long(), 1, where // page)
    spare = s["whole"][0].shape[0] - 1   # rows without a token are written there
    pages, inside = torch.where(held, pages, spare), torch.where(held, where % page, 0)
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
    """[B, Hkv, tokens, d] in 32 bits."""
    rows = cache.view(torch.uint8)[table] if case["cache"] == "e4m3" else cache[table]
    rows = rows.view(cache.dtype).float() * scale
    if case["cache_layout"] == "bnhd":
        return rows.flatten(1, 2).transpose(1, 2)
    return rows.transpose(1, 2).flatten(2, 3)


def _plain_decode(s):
    case = s["case"]
    B, H, Hkv, d = case["B"], case["H"], case["Hkv"], case["d"]
    table = s["table"].long().clamp(min=0)
    k, v = (_gathered(case, c, table, f) for c, f in zip((s["k_cache"], s["v_cache"]), s["scales"]))
    at, n = torch.arange(k.shape[2], device="cuda")[None], s["lengths"][:, None]
    seen = at < n
    if case["window"]:
        seen = seen & ((at >= n - case["window"]) | (at < case["sinks"]))
    q = s["q"].float().view(B, Hkv, H // Hkv, d)
    scores = torch.matmul(q, k.transpose(2, 3)) * (1.0 / d ** 0.5)
    scores = torch.where(seen[:, None, None], scores, -math.inf)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    top = scores.amax(dim=-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(scores - top)
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, v) / total.clamp(min=1e-30)
    return o.view(B, H, d).to(s["q"].dtype), (top + torch.log(total)).view(B, H)


def _plain_window(s):
    """Blocks of queries against the keys of their window and the first tokens."""
    case = s["case"]
    B, H, Hkv, N, d = case["B"], case["H"], case["Hkv"], case["N"], case["d"]
    w, first = min(case["window"], N), min(case["sinks"], N)
    rows = min(N, max(64, w // 4))
    blocks = (N + rows - 1) // rows
    q, k, v = (_by_token(t, case["layout"]).transpose(1, 2).float() for t in (s["q"], s["k"], s["v"]))
    q = torch.nn.functional.pad(q, (0, 0, 0, blocks * rows - N)).view(B, Hkv, H // Hkv, blocks, rows, d)
    at = torch.arange(blocks * rows, device="cuda").view(blocks, rows, 1)
    band = (torch.arange(blocks, device="cuda")[:, None] * rows
            + torch.arange(-w + 1, rows, device="cuda"))          # keys of a block's windows
    sinks = torch.arange(first, device="cuda").expand(blocks, first)
    key = torch.cat((sinks, band), dim=1)[:, None]                   # [blocks, 1, keys]
    in_window = (key <= at) & (at - key < w) & (key >= 0) & (key < N)
    is_sink = torch.arange(key.shape[2], device="cuda") < first
    seen = torch.where(is_sink, (key <= at) & (at - key >= w), in_window)
    index = key[:, 0].clamp(0, N - 1)
    kb, vb = k[:, :, index], v[:, :, index]                         # [B, Hkv, blocks, keys, width]
    scores = torch.matmul(q, kb.transpose(3, 4)[:, :, None]) * (1.0 / d ** 0.5)
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(dim=-1, keepdim=True).clamp(min=-1e30)
    p = scores.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = (torch.matmul(p, vb[:, :, None]) / total.clamp(min=1e-30)).view(B, H, blocks * rows, -1)[:, :, :N]
    lse = (top + torch.log(total)).view(B, H, blocks * rows)[:, :, :N].contiguous()
    return _by_token(o.transpose(1, 2), case["layout"]).to(s["q"].dtype).contiguous(), lse


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return (_plain_window if op == "window" else _plain_decode if op == "decode" else _plain_rope)(s)
    import paper_2506_12355_amd as qa
    if op == "rope":
        return qa.qk_norm_rope(s["q"], s["k"], cos=s["cos"], sin=s["sin"], q_weight=s["q_weight"],
                               k_weight=s["k_weight"], eps=EPS, starts=s["starts"], counts=s["counts"],
                               interleaved=case["interleaved"], layout=case["layout"])
    if op == "append":
        q = qa.qk_norm_rope_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"],
                                   s["starts"], counts=s["counts"], cos=s["cos"], sin=s["sin"],
                                   q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                   k_scale=s["scales"][0], v_scale=s["scales"][1],
                                   layout=case["layout"], cache_layout=case["cache_layout"])
        return q, s["k_cache"], s["v_cache"]
    if op == "decode":
        return qa.decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"],
                         window=case["window"] or None, sinks=case["sinks"], k_scale=s["scales"][0],
                         v_scale=s["scales"][1], cache_layout=case["cache_layout"])
    return qa.fwd_window(s["q"], s["k"], s["v"], case["window"], sinks=case["sinks"],
                         layout=case["layout"])


# ------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "window":
        return _exact_window(s)
    if case["op"] == "decode":
        return _exact_decode(s)
    return _exact_rope(s)


def _attend(q, k, v, scale, hidden):
    """One head in 64 bits: rows q against k and v, `hidden` true where a key is not seen."""
    x = (q @ k.t().contiguous()) * scale
    x.masked_fill_(hidden, -math.inf)
    lse = torch.logsumexp(x, dim=1)
    weights = torch.exp(x - lse.clamp(min=-1e300)[:, None])
    return weights @ v, lse


def _exact_window(s):
    case = s["case"]
    B, H, N, d = case["B"], case["H"], case["N"], case["d"]
    bnhd = case["layout"] == "bnhd"
    o = torch.empty(_shape(case, H, case["dv"]), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, H, N), dtype=torch.float64, device="cuda")

    def head(t, b, h):
        return (t[b, :, h] if bnhd else t[b, h]).double()

    for b in range(B):
        for h in range(H):
            g = h // (H // case["Hkv"])
            q, k, v = head(s["q"], b, h), head(s["k"], b, g), head(s["v"], b, g)
            out = o[b, :, h] if bnhd else o[b, h]
            for lo in range(0, N, 2048):
                hi = min(N, lo + 2048)
                i = torch.arange(lo, hi, device="cuda")[:, None]
                # the first tokens, then what any of these rows sees of its window
                from_ = max(0, lo - case["window"] + 1)
                keys = torch.cat((torch.arange(min(case["sinks"], from_), device="cuda"),
                                  torch.arange(from_, hi, device="cuda")))
                hidden = (keys > i) | ((i - keys >= case["window"]) & (keys >= case["sinks"]))
                out[lo:hi], lse[b, h, lo:hi] = _attend(q[lo:hi], k[keys], v[keys], d ** -0.5, hidden)
    return o, lse


def _exact_decode(s):
    case = s["case"]
    B, H, Hkv, d, page = case["B"], case["H"], case["Hkv"], case["d"], case["page"]
    o = torch.zeros((B, H, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        if n == 0:
            continue
        pages = s["table"][b, :(n + page - 1) // page].long()

        def tokens(cache, f):
            t = (cache.view(torch.uint8)[pages].view(cache.dtype) if case["cache"] == "e4m3"
                 else cache[pages]).float()
            t = t if case["cache_layout"] == "bnhd" else t.permute(0, 2, 1, 3)
            return t.reshape(-1, Hkv, d)[:n].double() * f

        k, v = tokens(s["k_cache"], s["scales"][0]), tokens(s["v_cache"], s["scales"][1])
        back = n - 1 - torch.arange(n, device="cuda")   # how far a key lies back
        hidden = torch.zeros(n, dtype=torch.bool, device="cuda")
        if case["window"]:
            hidden = (back >= case["window"]) & (n - 1 - back >= case["sinks"])
        for g in range(Hkv):
            heads = slice(g * (H // Hkv), (g + 1) * (H // Hkv))
            o[b, heads], lse[b, heads] = _attend(s["q"][b, heads].double(), k[:, g].contiguous(),
                                                 v[:, g].contiguous(), d ** -0.5, hidden)
    return o, lse


def _exact_rope(s):
    """The rotation as a product of complex numbers."""
    case = s["case"]
    N, R, layout = case["N"], case["rotary"], case["layout"]
    starts, counts = _starts(case), _lengths(case)

    def turned(x, weight):
        out = torch.zeros_like(x, dtype=torch.float64)
        for b in range(case["B"]):
            n = counts[b]
            y = x[b, :n].double()
            y = y / torch.sqrt(y.square().sum(dim=-1, keepdim=True) / case["d"] + EPS) * weight.double()
            unit = torch.complex(s["cos"][starts[b]:starts[b] + n].double(),
                                 s["sin"][starts[b]:starts[b] + n].double())[:, None]
            r = y[..., :R].clone()
            pairs = r.unflatten(-1, (-1, 2)) if case["interleaved"] else r.unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
            y[..., :R] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            out[b, :n] = y
        return out

    q = turned(_by_token(s["q"], layout), s["q_weight"])
    k = turned(_by_token(s["k"], layout), s["k_weight"])
    if case["op"] == "rope":
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
