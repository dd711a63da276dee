"""perf/operators.py without a GPU: which handle a pass uses."""
import importlib.util
import os
import types

import pytest

from conftest import ROOT


@pytest.fixture
def operators():
    spec = importlib.util.spec_from_file_location("perf_operators", os.path.join(ROOT, "perf", "operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_a_pass_uses_the_handle_of_the_current_stream(operators, monkeypatch):
    """A state that is run on one stream and then, or captured, on another: its calls go where the current stream is."""
    import paper_2311_09445_b200 as package
    streams, device = {0: 16, 1: 16}, [0]                            # (two devices' streams may have one number)
    cuda = operators.torch.cuda
    monkeypatch.setattr(cuda, "current_device", lambda: device[0])
    monkeypatch.setattr(cuda, "current_stream", lambda d=None: (device[0] if d is None else d, streams[device[0] if d is None else d]))
    monkeypatch.setattr(operators.torch._C, "_cuda_getCurrentRawStream", lambda d: streams[d], raising=False)
    monkeypatch.setattr(package, "RowRouter", lambda device=None, stream=None: types.SimpleNamespace(stream=stream))
    state, handles = {"case": {}}, []
    for raw in (16, 16, 32, 16):
        streams[0] = raw
        handles.append(operators._router(state))
        assert handles[-1].stream == (0, raw)
    assert handles[0] is handles[1] is handles[3]
    assert operators._router({"case": {}}) is handles[3]            # another program's state shares the stream's handle
    device[0] = 1
    assert operators._router({"case": {}}).stream == (1, 16)
