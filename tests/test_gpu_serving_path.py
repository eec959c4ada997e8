"""The serving operators together, as a program runs them: a padded batch of prompts
through norm, rotation and cache, attention over the prompts, then token after token over
the cache; on other streams, and captured into a graph."""
from __future__ import annotations

import math

import pytest

from tests import serving_oracle as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    return qa


def _bits(t):
    import torch
    return t.contiguous().view(torch.uint8 if t.element_size() == 1 else torch.int16 if t.element_size() == 2 else torch.int32)


class Model:
    """What a program keeps for one layer: weights, angles, cache and page table."""

    def __init__(self, B, H, Hkv, d, longest, page, cache, seed, dtype=None):
        import torch
        self.dtype = dtype or torch.bfloat16
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.B, self.H, self.Hkv, self.d = B, H, Hkv, d
        self.cos, self.sin = so.rotation_table(longest, d)
        self.qw, self.kw = ((1 + 0.2 * self.normal(d)).to(self.dtype) for _ in range(2))
        columns = (longest + page - 1) // page
        self.table = torch.randperm(B * columns, generator=self.gen, device="cuda").to(torch.int32).view(B, columns)
        kind = torch.float8_e4m3fn if cache == "e4m3" else self.dtype
        self.scales = (1 / 60, 1 / 80) if cache == "e4m3" else (1.0, 1.0)
        self.cache = [torch.full((B * columns, Hkv, page, d), math.nan, device="cuda").to(kind) for _ in range(2)]

    def normal(self, *shape):
        import torch
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def projections(self, N):
        """q, k and v as parts of one [B, N, heads, d] output."""
        x = self.normal(self.B, N, self.H + 2 * self.Hkv, self.d).to(self.dtype)
        return x.split((self.H, self.Hkv, self.Hkv), dim=2)

    def append(self, qa, q, k, v, starts, counts=None, k_out=None, **kw):
        return qa.qk_norm_rope_append(
            q, k, v, *self.cache, self.table, starts, cos=self.cos, sin=self.sin, q_weight=self.qw,
            k_weight=self.kw, counts=counts, k_scale=self.scales[0], v_scale=self.scales[1],
            k_out=k_out, layout="bnhd", **kw)

    def decode(self, qa, q, lengths, **kw):
        return qa.decode(q, *self.cache, self.table, lengths, k_scale=self.scales[0],
                         v_scale=self.scales[1], **kw)


@pytest.mark.parametrize("window,sinks", [(None, 0), (60, 4)])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_then_tokens(qa, window, sinks, cache, d):
    """Against attention in 64 bits on the normalised and rotated rows of all tokens.  The
    rows that enter are rounded to bf16 (the cache: to its type): the definition is taken on
    the rows as rounded, which the cache holds and qk_norm_rope returns."""
    import torch
    B, H, Hkv, N, page, steps = 4, 8, 2, 150, 16, 5
    counts = [150, 1, 77, 16]
    m = Model(B, H, Hkv, d, N + steps, page, cache, 20)
    lengths = torch.tensor(counts, dtype=torch.int32, device="cuda")
    q, k, v = m.projections(N)
    k_out = torch.empty(B, N, Hkv, d, device="cuda", dtype=m.dtype)
    starts = torch.zeros(B, dtype=torch.int32, device="cuda")
    q_out = m.append(qa, q, k, v, starts, counts=lengths, k_out=k_out)
    held = (torch.arange(N, device="cuda") < lengths[:, None])[:, :, None, None]
    vc = torch.where(held, v, 0).contiguous()
    if window:
        o, lse = qa.fwd_window(q_out, k_out, vc, window, sinks, layout="bnhd")
    else:
        o, lse = qa.fwd(q_out, k_out, vc, causal=True, layout="bnhd")
    for b, n in enumerate(counts):
        seen = so.window_mask(n, window or N, sinks)
        for h in range(H):
            want = so.attention_row_bounds(q_out[b, :n, h], k_out[b, :n, h // 4], vc[b, :n, h // 4],
                                           1 / d ** 0.5, seen, m.dtype)
            so.check_attention(o[b, :n, h], lse[b, h, :n], want, f"prompt b={b} h={h}")
    for step in range(steps):
        q, k, v = m.projections(1)
        q_out = m.append(qa, q, k, v, lengths)
        lengths += 1
        o, lse = m.decode(qa, q_out[:, 0], lengths, window=window, sinks=sinks)
        now = [n + step + 1 for n in counts]
        for b, heads, want in so.decode(q_out[:, 0], *m.cache, m.table, now, 1 / d ** 0.5,
                                        window or 0, sinks, *m.scales, "bhnd"):
            so.check_attention(o[b, heads], lse[b, heads], want, f"step {step} b={b}")


def test_the_last_row_of_a_prompt_is_what_decode_gives(qa):
    """The same tokens as a prompt and as cache and new token: within both bounds."""
    import torch
    B, H, Hkv, d, N = 2, 4, 2, 128, 333
    m = Model(B, H, Hkv, d, N, 32, "same", 21)
    q, k, v = m.projections(N)
    k_out = torch.empty(B, N, Hkv, d, device="cuda", dtype=m.dtype)
    q_out = m.append(qa, q, k, v, None, k_out=k_out)
    lengths = torch.full((B,), N, dtype=torch.int32, device="cuda")
    o1, lse1 = qa.fwd_window(q_out, k_out, v.contiguous(), 100, 7, layout="bnhd")
    o2, lse2 = m.decode(qa, q_out[:, -1].contiguous(), lengths, window=100, sinks=7)
    for b, heads, want in so.decode(q_out[:, -1], *m.cache, m.table, [N, N], 1 / d ** 0.5, 100, 7, 1.0, 1.0, "bhnd"):
        so.check_attention(o1[b, -1, heads], lse1[b, heads, -1], want)
        so.check_attention(o2[b, heads], lse2[b, heads], want)


def test_other_streams(qa):
    """Calls on several streams at once (each decode with a workspace of its own) give what
    the same calls give one after another."""
    import torch
    work = []
    for i, (cache, window) in enumerate((("same", None), ("e4m3", None), ("same", 700))):
        m = Model(3, 8, 2, 128, 4000, 64, cache, 30 + i)
        q, k, v = m.projections(3900)
        m.append(qa, q, k, v, None)
        work.append((m, m.projections(1), torch.tensor([3900, 5, 2000], dtype=torch.int32, device="cuda"), window))

    def steps(item, stream=None):
        m, (q, k, v), starts, window = item
        out = []
        for s in range(4):
            q_out = m.append(qa, q, k, v, starts + s, stream=stream)
            out.append(m.decode(qa, q_out[:, 0], starts + s + 1, window=window, stream=stream))
        return out
    ref = [[(o.clone(), lse.clone()) for o, lse in steps(item)] for item in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(3):
        got = []
        for item, s in zip(work, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(steps(item))
        torch.cuda.synchronize()
        for a, b in zip(ref, got):
            for (o, lse), (o2, lse2) in zip(a, b):
                assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    # the stream argument, with the tensors made on the current stream
    s = streams[0]
    m, (q, k, v), starts, window = work[0]
    lens = starts + 1
    s.wait_stream(torch.cuda.current_stream())
    q_out = m.append(qa, q, k, v, starts, stream=s)
    o, lse = m.decode(qa, q_out[:, 0], lens, window=window, stream=s)
    s.synchronize()
    assert torch.equal(_bits(o), _bits(ref[0][0][0])) and torch.equal(_bits(lse), _bits(ref[0][0][1]))


@pytest.mark.parametrize("longest", [400, 6000])
def test_captured_steps_replay(qa, longest):
    """One step (append, decode) captured once and replayed with other tokens, starts and
    lengths in the same buffers, an eager step of another model between the replays; and a
    second graph of the same calls, replayed in turn with the first."""
    import torch
    B, H, Hkv, d = 3, 8, 2, 64
    m, eager = (Model(B, H, Hkv, d, longest, 16, "same", 40 + i) for i in range(2))
    prompt = m.projections(longest - 20)
    m.append(qa, *prompt, None)
    eager.append(qa, *eager.projections(longest - 20), None)
    q, k, v = (t.clone() for t in m.projections(1))
    starts, lengths = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    assert (qa.decode_workspace(q[:, 0], m.cache[0], m.table) > 0) == (longest > 1000)
    m.decode(qa, m.append(qa, q, k, v, starts)[:, 0], lengths)
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            q_out = m.append(qa, q, k, v, starts)
            out = m.decode(qa, q_out[:, 0], lengths)
        graphs.append((g, out))
    for rep in range(6):
        g, (o, lse) = graphs[rep % 2]
        new = m.projections(1)
        for t, x in zip((q, k, v), new):
            t.copy_(x)
        starts.copy_(torch.tensor([longest - 20 + rep, rep, 37 * rep], dtype=torch.int32))
        lengths.copy_(starts + 1)
        o.fill_(math.nan)
        lse.fill_(math.nan)
        g.replay()
        e = eager.decode(qa, eager.append(qa, *eager.projections(1), starts)[:, 0], lengths)
        assert torch.isfinite(e[0]).all()
        torch.cuda.synchronize()
        got = o.clone(), lse.clone()
        ref = m.decode(qa, m.append(qa, *new, starts)[:, 0], lengths)
        torch.cuda.synchronize()
        assert torch.equal(_bits(got[0]), _bits(ref[0])) and torch.equal(_bits(got[1]), _bits(ref[1])), rep


def test_window_prompts_captured(qa):
    import torch
    x = [torch.randn(1, 4, 900, 64, device="cuda").bfloat16() for _ in range(3)]
    qa.fwd_window(*x, 200, 4)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, lse = qa.fwd_window(*x, 200, 4)
    for rep in range(4):
        for t in x:
            t.copy_(torch.randn_like(t))
        ref = qa.fwd_window(*x, 200, 4)
        o.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(_bits(o), _bits(ref[0])) and torch.equal(_bits(lse), _bits(ref[1])), rep


def test_results_repeat(qa):
    """The same bytes every time, however the work is divided."""
    import torch
    m = Model(5, 16, 2, 128, 3000, 16, "e4m3", 50)
    m.append(qa, *m.projections(2900), None)
    lengths = torch.tensor([2900, 1, 1500, 0, 33], dtype=torch.int32, device="cuda")
    q = m.normal(5, 16, 128).to(m.dtype)
    for kw in (dict(), dict(max_length=2900), dict(window=100, sinks=3)):
        ref = [t.clone() for t in m.decode(qa, q, lengths, **kw)]
        for _ in range(5):
            got = m.decode(qa, q, lengths, **kw)
            assert all(torch.equal(_bits(a), _bits(b)) for a, b in zip(ref, got))


def test_new_outputs_are_plain_tensors(qa):
    import torch

    class Tagged(torch.Tensor):
        pass

    m = Model(2, 4, 2, 64, 64, 16, "same", 51)
    q, k, v = (t.contiguous().as_subclass(Tagged) for t in m.projections(3))
    lengths = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    res = [*qa.qk_norm_rope(q, k, layout="bnhd"), m.append(qa, q, k, v, None),
           *m.decode(qa, q[:, 0].contiguous(), lengths), *qa.fwd_window(q, k, v, 2, layout="bnhd")]
    assert all(type(t) is torch.Tensor for t in res)
