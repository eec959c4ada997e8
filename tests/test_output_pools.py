"""New outputs and workspaces come from the pool of the stream that the call runs on:
memory of another stream's pool may still be in use by that stream's work, and is given
out again in that stream's order.  Without a GPU: host tensors that say they are on
cuda:0, a library that enqueues nothing, and torch's allocating calls recorded."""
from __future__ import annotations

import contextlib

import pytest
import torch

import paper_2506_12355_amd as qa
from paper_2506_12355_amd import binding, serving

GPU = torch.device("cuda", 0)


class Stream:
    device = GPU
    cuda_stream = 7


class Library:
    def __getattr__(self, name):
        return lambda *args: qa.QM_OK


@pytest.fixture
def made(monkeypatch):
    """The streams that were current (None: the caller's own) as each tensor was made."""
    current, made = [None], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    def recorded(make):
        def call(*args, device=None, **kw):
            made.append(current[-1])
            return make(*args, **kw)
        return call

    monkeypatch.setattr(torch, "empty", recorded(torch.empty))
    monkeypatch.setattr(torch, "empty_like", recorded(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.Tensor, "device", GPU, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0, raising=False)
    for module in (binding, serving):
        monkeypatch.setattr(module, "load_library", Library)
    monkeypatch.setattr(serving, "_workspace_bytes", lambda *sizes: 64)
    return made


def _calls():
    """Each entry point with every output new, and how many tensors it makes."""
    def x(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)
    q, k, v = x(1, 4, 32, 64), x(1, 2, 32, 64), x(1, 2, 32, 64)
    codes = [x(1, 2, 32, 128, dtype=torch.uint8) for _ in range(3)]
    wide = x(1, 2, 32, 192), x(1, 2, 32, 192), x(1, 2, 32, 128)
    token, cache = x(1, 4, 64), [x(4, 2, 16, 64) for _ in range(2)]
    table, lengths = x(1, 4, dtype=torch.int32), x(1, dtype=torch.int32)
    return {
        "fwd": (lambda **kw: qa.fwd(q, k, v, **kw), 2),
        "fwd mla": (lambda **kw: qa.fwd(*wide, **kw), 2),
        "fwd_fp8": (lambda **kw: qa.fwd_fp8(*codes, (1.0, 1.0, 1.0), **kw), 2),
        "fwd_window": (lambda **kw: qa.fwd_window(q, k, v, 8, **kw), 2),
        "qk_norm_rope": (lambda **kw: qa.qk_norm_rope(q, k, **kw), 2),
        "qk_norm_rope of a view": (lambda **kw: qa.qk_norm_rope(q.transpose(1, 2), k.transpose(1, 2), layout="bnhd", **kw), 2),
        "qk_norm_rope_append": (lambda **kw: qa.qk_norm_rope_append(q, k, v, *cache, table, **kw), 1),
        "decode": (lambda **kw: qa.decode(token, *cache, table, lengths, **kw), 3),   # o, lse, workspace
    }


@pytest.mark.parametrize("name", list(_calls()))
def test_new_tensors_are_made_under_the_calls_stream(made, name):
    call, n = _calls()[name]
    s = Stream()
    call(stream=s)
    assert made == [s] * n


@pytest.mark.parametrize("name", list(_calls()))
def test_without_a_stream_argument_the_current_stream_stays(made, name):
    call, n = _calls()[name]
    call()
    assert made == [None] * n


@pytest.mark.parametrize("name", ["fwd", "fwd_fp8", "fwd_window", "qk_norm_rope", "qk_norm_rope_append"])
def test_outputs_of_the_callers_change_no_stream(made, name, monkeypatch):
    call, _ = _calls()[name]
    given = call()
    names = ("q_out", "k_out") if "rope" in name else ("out", "lse")
    given = dict(zip(names, given if isinstance(given, tuple) else (given,)))
    made.clear()

    def stream(s):
        raise AssertionError("the current stream was changed")
    monkeypatch.setattr(torch.cuda, "stream", stream)
    call(stream=Stream(), **given)
    assert made == []
