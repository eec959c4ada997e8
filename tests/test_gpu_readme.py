"""The README's serving example as it stands there: a padded batch of prompts, whose rows
past the counts hold NaN, then a token of each, against 64 bits."""
from __future__ import annotations

import math
import os
import re

import pytest

from tests import serving_oracle as so

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def _example():
    """Its two halves: the prompts, and the steps of one token."""
    with open(README) as f:
        block, = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "# prompts:" in b]
    prompts, tokens = block.split("# then token by token")
    return prompts, "#" + tokens


def test_the_serving_example():
    import torch
    import paper_2506_12355_amd as qa
    prompts, tokens = _example()
    B, N, H, Hkv, d, page, window = 3, 100, 8, 2, 128, 16, 40
    counts = [100, 37, 1]
    g = torch.Generator(device="cuda")
    g.manual_seed(60)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda").bfloat16()

    qkv = normal(B, N, H + 2 * Hkv, d)
    for b, n in enumerate(counts):
        qkv[b, n:] = math.nan
    cos, sin = so.rotation_table(N + 1, d)
    columns = (N + page) // page
    env = dict(
        torch=torch, qa=qa, qkv=qkv, B=B, N=N, H=H, Hkv=Hkv, d=d, window=window, cos=cos, sin=sin,
        qw=normal(d), kw=normal(d), counts=torch.tensor(counts, dtype=torch.int32, device="cuda"),
        starts=torch.zeros(B, dtype=torch.int32, device="cuda"),
        page_table=torch.arange(B * columns, dtype=torch.int32, device="cuda").view(B, columns))
    env["k_cache"], env["v_cache"] = (normal(B * columns, Hkv, page, d) for _ in range(2))
    env["lengths"] = env["counts"].clone()
    exec(prompts, env)
    o, lse, q_rot, k_rot, v = (env[name] for name in ("o", "lse", "q_rot", "k_rot", "v"))
    for b, n in enumerate(counts):
        seen = so.window_mask(n, window, 0)
        for h in range(H):
            want = so.attention_row_bounds(q_rot[b, :n, h], k_rot[b, :n, h // 4], v[b, :n, h // 4],
                                           d ** -0.5, seen, torch.bfloat16)
            so.check_attention(o[b, :n, h], lse[b, h, :n], want, f"prompt b={b} h={h}")
    env["q"], env["k"], env["v"] = (normal(B, 1, heads, d) for heads in (H, Hkv, Hkv))
    exec(tokens, env)
    assert env["lengths"].tolist() == [n + 1 for n in counts]
    for b, heads, want in so.decode(env["q_rot"][:, 0], env["k_cache"], env["v_cache"], env["page_table"],
                                    [n + 1 for n in counts], d ** -0.5, window, 0, 1.0, 1.0, "bhnd"):
        so.check_attention(env["o"][b, heads], env["lse"][b, heads], want, f"token b={b}")
