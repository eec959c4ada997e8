"""A decoding step as a program runs it: the residual's addition and norm, a projection, the
rotation by several axes with the cache's writes, attention behind a shared prefix; eagerly
and captured, against 64 bits on the rounded values that each call was given.  And the
README's example of such a step, as it stands there."""
from __future__ import annotations

import os
import re

import pytest

from tests import serving_oracle as so
from tests.test_gpu_rope_axes import _axes_of, _define
from tests.test_gpu_rms_norm import FP32, _define as _define_norm

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    return qa


class Layer:
    """One layer's weights, its cache with a shared prefix in it, and what a step changes."""

    def __init__(self, B, H, Hkv, d, width, prefix, page, cache, seed):
        import torch
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.B, self.H, self.Hkv, self.d, self.prefix, self.page = B, H, Hkv, d, prefix, page
        self.norm_weight = (1 + 0.2 * self.normal(width)).bfloat16()
        self.w_qkv = (self.normal(width, (H + 2 * Hkv) * d) / width ** 0.5).bfloat16()
        self.qw, self.kw = ((1 + 0.2 * self.normal(d)).bfloat16() for _ in range(2))
        self.cos, self.sin = so.rotation_table(prefix + 64, d)
        self.axes = tuple(_axes_of("runs", d // 2, 3))
        low, shared = prefix // page, (prefix + page - 1) // page
        per = (prefix + 64) // page + 1 - low
        order = torch.randperm(shared + B * per, generator=self.gen, device="cuda").to(torch.int32)
        self.prefix_table = order[:shared].contiguous()
        self.page_table = torch.full((B, low + per), -1, dtype=torch.int32, device="cuda")
        self.page_table[:, low:] = order[shared:].view(B, per)
        kind = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
        self.scales = (1 / 60, 1 / 80) if cache == "e4m3" else (1.0, 1.0)
        self.cache = [(self.normal(shared + B * per, Hkv, page, d) / f).to(kind) for f in self.scales]
        self.lengths = torch.full((B,), prefix, dtype=torch.int32, device="cuda")
        self.h = self.normal(B, 1, width, mult=4).bfloat16()
        self.x = self.normal(B, 1, width).bfloat16()
        self.positions = torch.full((3, B, 1), prefix, dtype=torch.int32, device="cuda")

    def normal(self, *shape, mult=1.0):
        import torch
        return torch.randn(*shape, generator=self.gen, device="cuda") * mult

    def step(self, qa, fp8):
        """The tensors that the step goes through."""
        import torch
        if fp8:
            codes, scales, h = qa.rms_norm_fp8(self.x, self.norm_weight, residual=self.h, sum_out=self.h)
            y = (codes.float() * scales).bfloat16()
        else:
            codes = scales = None
            y, h = qa.rms_norm(self.x, self.norm_weight, residual=self.h, sum_out=self.h)
        qkv = (y @ self.w_qkv).view(self.B, 1, self.H + 2 * self.Hkv, self.d)
        q, k, v = qkv.split((self.H, self.Hkv, self.Hkv), dim=2)
        q_rot = qa.qk_norm_rope_append(q, k, v, *self.cache, self.page_table, self.lengths, cos=self.cos, sin=self.sin,
                                       q_weight=self.qw, k_weight=self.kw, positions=self.positions, axes=self.axes,
                                       k_scale=self.scales[0], v_scale=self.scales[1], layout="bnhd")
        self.lengths += 1
        o, lse = qa.decode_shared(q_rot[:, 0], *self.cache, self.page_table, self.lengths, self.prefix_table, self.prefix,
                                  k_scale=self.scales[0], v_scale=self.scales[1])
        return dict(y=y, h=h, codes=codes, scales=scales, q=q, q_rot=q_rot, o=o, lse=lse)

    def check(self, before_x, before_h, got, n):
        import torch
        y, s = _define_norm(before_x, self.norm_weight, before_h, 1e-6)
        so.check_rounded(got["h"], s, 2.0 ** -24 * s.abs(), "sum")
        if got["codes"] is None:
            so.check_rounded(got["y"], y, FP32 * y.abs(), "norm")
        else:
            scaled = y / got["scales"].double()
            so.check_rounded(got["codes"], scaled, 2 * FP32 * scaled.abs(), "codes")
        want, slack = _define(got["q"], self.qw, self.cos, self.sin, self.positions, self.axes, 1e-6, False)
        so.check_rounded(got["q_rot"], want, slack, "q")
        low = self.prefix // self.page
        for b in range(self.B):
            k, v = (torch.cat((so.tokens_of(c, self.prefix_table, self.prefix, "bhnd"),
                               so.tokens_of(c, self.page_table[b, low:], n - low * self.page, "bhnd")[self.prefix - low * self.page:])) * f
                    for c, f in zip(self.cache, self.scales))
            G = self.H // self.Hkv
            for g in range(self.Hkv):
                heads = slice(g * G, (g + 1) * G)
                w = so.attention_row_bounds(got["q_rot"][b, 0, heads], k[:, g].contiguous(), v[:, g].contiguous(),
                                            self.d ** -0.5, torch.ones(G, n, dtype=torch.bool, device="cuda"), torch.bfloat16)
                so.check_attention(got["o"][b, heads], got["lse"][b, heads], w, f"b={b} heads={heads}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("B", [3, 24])
def test_decoding_steps(qa, B, cache, fp8):
    import torch
    m = Layer(B, 8, 2, 128, 1024, 203, 16, cache, 50)
    for n in range(4):
        x, h = m.x.clone(), m.h.clone()
        m.positions[1] += 1
        m.positions[2] += 2
        m.check(x, h, m.step(qa, fp8), m.prefix + n + 1)
        m.x = m.normal(B, 1, 1024).bfloat16()


def test_captured_steps(qa):
    """A captured step, replayed with the lengths and positions of the next tokens, gives the
    bytes of eager steps from the same state."""
    import torch
    a, b = (Layer(6, 8, 2, 64, 512, 150, 16, "e4m3", 51) for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    warm = Layer(6, 8, 2, 64, 512, 150, 16, "e4m3", 51)
    with torch.cuda.stream(s):
        warm.step(qa, True)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = a.step(qa, True)
    for step in range(5):
        x = a.normal(6, 1, 512).bfloat16()
        for m in (a, b):
            m.x.copy_(x)
            m.positions[1] = m.prefix + step // 2
        graph.replay()
        eager = b.step(qa, True)
        torch.cuda.synchronize()
        for name in ("h", "codes", "scales", "q_rot", "o", "lse"):
            assert torch.equal(captured[name].view(torch.uint8), eager[name].contiguous().view(torch.uint8)), (step, name)
        for c, d in zip(a.cache, b.cache):
            assert torch.equal(c.view(torch.uint8), d.view(torch.uint8))
        assert torch.equal(a.lengths, b.lengths)


def test_the_readme_example(qa):
    import torch
    with open(README) as f:
        block, = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "decode_shared(" in b]
    m = Layer(5, 8, 2, 128, 1024, 100, 16, "same", 52)
    x, h = m.x.clone(), m.h.clone()
    env = dict(torch=torch, qa=qa, x=m.x, h=m.h, norm_weight=m.norm_weight, w_qkv=m.w_qkv, B=5, H=8, Hkv=2, d=128,
               k_cache=m.cache[0], v_cache=m.cache[1], page_table=m.page_table, lengths=m.lengths, cos=m.cos, sin=m.sin,
               qw=m.qw, kw=m.kw, positions=m.positions, axes=m.axes, prefix_table=m.prefix_table, prefix_length=m.prefix)
    exec(block, env)
    m.check(x, h, dict(y=env["y"], h=env["h"], codes=None, q=env["q"], q_rot=env["q_rot"], o=env["o"], lse=env["lse"]), 101)
