"""fwd_window where workgroups run several query blocks one after another: the next one's
blocks are set up, and its first loads go out, while the last one is written.  Every row of
the heads looked at against the definition in 64 bits, in each kind of instance, with more
query blocks than the device's 256 CUs hold at once (three workgroups of 128 rows a CU at
d = 64, two at d = 128, one of 192-wide keys, one of 256 rows)."""
from __future__ import annotations

import pytest

from tests import serving_oracle as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    yield qa
    qa.set_tile_rows(0)


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


# B, H, Hkv, N, d, window, sinks, dtype, and the query blocks of 128 rows (256 where `rows`
# says so) that a device of 256 CUs holds at once
CASES = [
    (2, 64, 8, 1500, 64, 200, 70, "bfloat16", 128, 768),
    (1, 48, 48, 3000, 64, 64, 0, "float16", 128, 768),
    (2, 40, 8, 1300, 128, 300, 70, "bfloat16", 128, 512),
    (1, 32, 32, 4100, 128, 1000, 4, "float16", 128, 512),
    (1, 16, 4, 8000, 128, 2600, 65, "bfloat16", 256, 256),
    (2, 30, 30, 1537, 128, 500, 1, "float16", 256, 256),
    (1, 24, 24, 3000, 192, 500, 4, "bfloat16", 256, 256),
    (2, 20, 20, 1025, 192, 100, 100, "float16", 128, 256),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_every_row_of_later_runs(qa, case):
    import torch
    B, H, Hkv, N, d, window, sinks, dtype, rows, resident = case
    dtype, dv = getattr(torch, dtype), min(d, 128)
    assert B * H * ((N + rows - 1) // rows) > resident
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    q, k, v = (torch.randn(B, h, N, w, generator=g, device="cuda").to(dtype) for h, w in ((H, d), (Hkv, d), (Hkv, dv)))
    results = []
    try:
        for tile in (0, 128, 256):   # 0: the call's own choice
            qa.set_tile_rows(tile)
            results.append(qa.fwd_window(q, k, v, window, sinks))
    finally:
        qa.set_tile_rows(0)
    o, lse = results[0]
    for o2, lse2 in results[1:]:
        assert torch.equal(_bits(o2), _bits(o)) and torch.equal(_bits(lse2), _bits(lse))
    if d != 192:
        t = (x.transpose(1, 2).contiguous() for x in (q, k, v))
        o2, lse2 = qa.fwd_window(*t, window, sinks, layout="bnhd")
        assert torch.equal(_bits(o2.transpose(1, 2)), _bits(o)) and torch.equal(_bits(lse2), _bits(lse))
    seen = so.window_mask(N, window, sinks)
    # heads of the first, the middle and the last runs
    for bh in sorted({0, 1, B * H // 3, B * H // 2, B * H - 2, B * H - 1}):
        b, h = divmod(bh, H)
        want = so.attention_row_bounds(q[b, h], k[b, h // (H // Hkv)], v[b, h // (H // Hkv)], d ** -0.5, seen, dtype)
        so.check_attention(o[b, h], lse[b, h], want, f"b={b} h={h}")
