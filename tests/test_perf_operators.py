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
    current = []
    monkeypatch.setattr(operators.torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(package, "RowRouter", lambda device=None, stream=None: types.SimpleNamespace(stream=stream))
    a, b, other_device = (types.SimpleNamespace(device_index=d, cuda_stream=p) for d, p in ((0, 16), (0, 32), (1, 16)))
    state, handles = {"case": {}}, []
    for s in (a, a, b, a, other_device):
        current.append(s)
        handles.append(operators._router(state))
        assert handles[-1].stream is s
    assert handles[0] is handles[1] is handles[3]
    assert operators._router({"case": {}}) is handles[4]            # another program's state shares the stream's handle
