import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line(
        "markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


def pytest_collection_modifyitems(config, items):
    # GPU tests run only where a GPU is present; without one they are skipped
    # (on a machine with an MI355X they run, selected with -m gpu).
    try:
        import torch
        have_gpu = torch.cuda.is_available()
    except Exception:  # pragma: no cover - torch missing
        have_gpu = False
    if have_gpu:
        return
    skip = pytest.mark.skip(reason="no GPU in this environment")
    for item in items:
        if "gpu" in item.keywords:
            item.add_marker(skip)


@pytest.fixture(autouse=True)
def lengths_live_as_long_as_their_calls(request, monkeypatch):
    """test_gpu_decode_shared.py's State makes the lengths of each of its calls anew, and a call
    on another stream reads them after it has returned.  As binding.fwd says of inputs, they
    have to live until that stream is done: here, to the test's end.  Dropped before,
    their memory is the next call's lengths while the last call still reads it."""
    shared = sys.modules.get("tests.test_gpu_decode_shared")
    if shared is None or getattr(request.module, "State", None) is not shared.State:
        yield
        return
    held, make = [], shared._ints

    def ints(values):
        held.append(make(values))
        return held[-1]
    monkeypatch.setattr(shared, "_ints", ints)
    yield
