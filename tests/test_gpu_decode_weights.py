"""decode loses next to nothing of the probabilities between the softmax and the product
with the values: against 64 bits, o is off by the rounding of the result and by fp32
arithmetic.

Bound, per element, before the last rounding:

    (lost + 2 D + 2^-18 + sums) sum_j p_j |v_j|  +  floor max_j p_j sum_j |v_j|

with `lost` what two values of the 16-bit type leave of a weight: half a step of half a
step, 2^-16 (bf16) or 2^-22 (f16); `floor` 2^-40 for f16, whose smallest step, 2^-24, is
halved and divided by the 2^15 that the weights are multiplied by (bf16 has the exponents
of fp32); D the error of the scores (serving_oracle); 2^-18 the exponential, the quotient
and the weights' sum, as there; and `sums` 2^-24 for each of a wavefront's additions to O,
at most four a block of 32 tokens, and 128 for the joins.  Then half a step of the type at
the value itself.  (A weight rounded once would be off by up to 2^-8 or 2^-11.)"""
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


def _half_step(x, dtype):
    """Half the spacing of the type at |x| (x in 64 bits)."""
    import torch
    bits, lowest = (7, -126) if dtype == torch.bfloat16 else (10, -14)
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** lowest)))
    return torch.exp2(e - bits - 1)


def _check(q, k, v, scale, got, dtype, what):
    """One key/value head: q [G, d], k and v [n, d] in 64 bits, got [G, d]."""
    import torch
    q = q.double()
    s = (q @ k.T.contiguous()) * scale
    p = torch.softmax(s, dim=1)
    o, size = p @ v, p @ v.abs()
    D = ((q.abs() @ k.abs().T.contiguous()) * abs(scale) * q.shape[1] * 2.0 ** -24).amax(1, keepdim=True)
    lost, floor = (2.0 ** -16, 0.0) if dtype == torch.bfloat16 else (2.0 ** -22, 2.0 ** -40)
    sums = (4 * math.ceil(k.shape[0] / 32) + 128) * 2.0 ** -24
    bound = (lost + 2 * D + 2.0 ** -18 + sums) * size + floor * p.amax(1, keepdim=True) * v.abs().sum(0)
    bound = bound + _half_step(o.abs() + bound, dtype)
    off = (got.double() - o).abs()
    assert bool((off <= bound).all()), (
        f"{what}: {int((off > bound).sum())} of {off.numel()} over, by up to {float((off / bound).max()):.2f} times the bound")


@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_weights_keep_their_bits(qa, dtype, d, cache, shares):
    import torch
    dtype = getattr(torch, dtype)
    lengths, page, H, Hkv = [2, 3, 5, 9, 40, 300, 1500], 16, 16, 2
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    columns = 600 if shares else 96
    per = [(n + page - 1) // page for n in lengths]
    table = torch.full((len(lengths), columns), -1, dtype=torch.int32, device="cuda")
    for b in range(len(lengths)):
        first = sum(per[:b])
        table[b, :per[b]] = torch.arange(first, first + per[b])
    q = torch.randn(len(lengths), H, d, generator=g, device="cuda").to(dtype)
    kind = torch.float8_e4m3fn if cache == "e4m3" else dtype
    kc, vc = ((torch.randn(sum(per), Hkv, page, d, generator=g, device="cuda") * (30 if cache == "e4m3" else 1)).to(kind)
              for _ in range(2))
    ks, vs = (1 / 32, 1 / 16) if cache == "e4m3" else (1.0, 1.0)
    most = None if shares else 512
    lens = lengths if shares else [min(n, 512) for n in lengths]
    assert (qa.decode_workspace(q, kc, table, max_length=most) > 0) == shares
    o, _ = qa.decode(q, kc, vc, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), scale=0.125,
                     k_scale=ks, v_scale=vs, max_length=most)
    for b, n in enumerate(lens):
        k, v = (so.tokens_of(c, table[b], n, "bhnd") * f for c, f in ((kc, ks), (vc, vs)))
        for h in range(Hkv):
            heads = slice(h * 8, h * 8 + 8)
            _check(q[b, heads], k[:, h].contiguous(), v[:, h].contiguous(), 0.125, o[b, heads], dtype, f"n={n} head {h}")


def test_many_weights_far_below_the_largest(qa):
    """f16: one key outweighs each of 65535 others 2^25.5 times, whose values alone are not
    zero.  Rounded to f16 as they are, the weights of the 16384 that share its wavefront
    would be zero.  (64 sequences of the same pages, so that a workgroup has a whole row.)"""
    import torch
    B, Hkv, n, d, page = 64, 8, 65536, 64, 64
    kc, vc = (torch.zeros(n // page, Hkv, page, d, device="cuda", dtype=torch.float16) for _ in range(2))
    table = torch.arange(n // page, device="cuda", dtype=torch.int32).expand(B, n // page).contiguous()
    q = torch.zeros(B, Hkv, d, device="cuda", dtype=torch.float16)
    q[..., 0] = 1.0
    at = 37777
    kc[at // page, :, at % page, 0] = 25.5 * math.log(2.0)   # (rounded to f16; the check takes it so)
    vc[:] = torch.linspace(1, 8, d, device="cuda").half()
    vc[at // page, :, at % page] = 0.0
    o, _ = qa.decode(q, kc, vc, table, torch.full((B,), n, dtype=torch.int32, device="cuda"), scale=1.0)
    k, v = (so.tokens_of(c, table[0], n, "bhnd") for c in (kc, vc))
    for b, h in ((0, 0), (17, 3), (63, 7)):
        _check(q[b, h:h + 1], k[:, h].contiguous(), v[:, h].contiguous(), 1.0, o[b, h:h + 1], torch.float16, f"b={b} head {h}")
    assert float(o.min()) > 1e-3   # about 0.14% of the values


def test_scores_too_large_for_steps_of_one(qa):
    """f16: scores past 2^24, whose fp32 steps exceed the weights' factor: the largest weight
    stays finite."""
    import torch
    for size in (300.0, 2000.0, 20000.0):
        q = torch.full((1, 1, 128), size, device="cuda", dtype=torch.float16)
        kc = torch.full((1, 1, 16, 128), size, device="cuda", dtype=torch.float16)
        vc = torch.arange(16, device="cuda").half()[:, None].expand(16, 128).contiguous()[None, None]
        table = torch.zeros(1, 1, device="cuda", dtype=torch.int32)
        for n in (1, 7, 16):
            o, lse = qa.decode(q, kc, vc, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
            assert torch.isfinite(lse).all()
            assert bool((o == (n - 1) / 2).all()), (size, n)
