"""New outputs and workspaces of the row norms, of the rotation by several axes and of decoding
behind a shared prefix come from the pool of the call's stream (how it is shown:
test_output_pools.py)."""
from __future__ import annotations

import pytest
import torch

import paper_2506_12355_amd as qa
from tests.test_output_pools import Stream, made  # noqa: F401


def _calls():
    """Each entry point with every output new, and how many tensors it makes."""
    def x(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)
    q, k, v = x(1, 4, 32, 64), x(1, 2, 32, 64), x(1, 2, 32, 64)
    token, cache = x(1, 4, 64), [x(4, 2, 16, 64) for _ in range(2)]
    table, lengths, first = x(1, 4, dtype=torch.int32), x(1, dtype=torch.int32), x(2, dtype=torch.int32)
    rows = x(5, 64)
    turn = dict(cos=x(9, 32, dtype=torch.float32), sin=x(9, 32, dtype=torch.float32),
                positions=x(2, 1, 32, dtype=torch.int32), axes=[0, 1] * 16)
    return {
        "rms_norm": (lambda **kw: qa.rms_norm(rows, **kw), 1),
        "rms_norm of a sum": (lambda **kw: qa.rms_norm(rows, residual=rows, **kw), 2),
        "rms_norm_fp8": (lambda **kw: qa.rms_norm_fp8(rows, residual=rows, **kw), 3),
        "rms_norm_fp8 with one scale": (lambda **kw: qa.rms_norm_fp8(rows, scale=2.0, **kw), 1),
        "qk_norm_rope": (lambda **kw: qa.qk_norm_rope(q, k, **turn, **kw), 2),
        "qk_norm_rope_append": (lambda **kw: qa.qk_norm_rope_append(q, k, v, *cache, table, **turn, **kw), 1),
        "decode_shared": (lambda **kw: qa.decode_shared(token, *cache, table, lengths, first, 20, **kw), 3),   # o, lse, workspace
    }


@pytest.mark.parametrize("name", list(_calls()))
def test_new_tensors_are_made_under_the_calls_stream(made, name):  # noqa: F811
    call, n = _calls()[name]
    s = Stream()
    call(stream=s)
    assert made == [s] * n


@pytest.mark.parametrize("name", list(_calls()))
def test_without_a_stream_argument_the_current_stream_stays(made, name):  # noqa: F811
    call, n = _calls()[name]
    call()
    assert made == [None] * n


def test_outputs_of_the_callers_change_no_stream(made, monkeypatch):  # noqa: F811
    rows, sums = (torch.zeros(5, 64, dtype=torch.bfloat16) for _ in range(2))
    out, codes = torch.zeros_like(rows), torch.zeros(5, 64, dtype=torch.uint8)
    made.clear()

    def stream(s):
        raise AssertionError("the current stream was changed")
    monkeypatch.setattr(torch.cuda, "stream", stream)
    y, s = qa.rms_norm(rows, residual=sums, out=out, sum_out=sums, stream=Stream())
    assert y is out and s is sums
    y, f, s = qa.rms_norm_fp8(rows, residual=sums, out=codes, scales=torch.zeros(5, 2), group=32, sum_out=sums, stream=Stream())
    assert y is codes and s is sums and f.shape == (5, 2)
    y, f, s = qa.rms_norm_fp8(rows, out=codes, scale=1.0, stream=Stream())
    assert f is None and s is None and made == []
