"""New outputs belong to the stream that the call runs on (see test_output_pools.py, which
shows it on the host for every tensor that a call makes)."""
from __future__ import annotations

import pytest

import seeded_inputs as si
from tests.gpu_util import to_device

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
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def test_new_outputs_are_of_the_calls_stream(qa):
    """The allocator's segments of a call's outputs are those of the stream it ran on, and
    their bytes those of the same call on the current stream."""
    import torch
    q, k, v = (to_device(x, "bf16") for x in si.make_qkv(1, 4, 200, 64, "bf16", seed=130))
    cache = [torch.zeros(16, 4, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    table = torch.arange(16, device="cuda", dtype=torch.int32)[None]
    lengths = torch.full((1,), 200, device="cuda", dtype=torch.int32)
    token = q[:, :, -1].contiguous()
    codes = [x.repeat(1, 1, 1, 2).to(torch.float8_e4m3fn) for x in (q, k, v)]
    calls = [lambda **kw: qa.fwd(q, k, v, **kw), lambda **kw: qa.fwd_window(q, k, v, 50, **kw),
             lambda **kw: qa.fwd_fp8(*codes, (1.0, 1.0, 1.0), **kw), lambda **kw: qa.qk_norm_rope(q, k, **kw),
             lambda **kw: (qa.qk_norm_rope_append(q, k, v, *cache, table, **kw),),
             lambda **kw: qa.decode(token, *cache, table, lengths, **kw)]
    ref = [call() for call in calls]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = [call(stream=s) for call in calls]
    s.synchronize()
    segments = torch.cuda.memory_snapshot()
    for a, b in zip(ref, got):
        for x, y in zip(a, b):
            assert torch.equal(_bits(x), _bits(y))
            own, = [g["stream"] for g in segments if g["address"] <= y.data_ptr() < g["address"] + g["total_size"]]
            assert own == s.cuda_stream
