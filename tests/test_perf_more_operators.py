"""perf/more_operators.py without a GPU: its cases, its generator against the known answers, and which handle a pass uses."""
import importlib.util
import os
import random
import types

import numpy as np
import pytest
import torch

from conftest import ROOT, golden_lines


@pytest.fixture(scope="module")
def operators():
    spec = importlib.util.spec_from_file_location("perf_more_operators", os.path.join(ROOT, "perf", "more_operators.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_cases_are_within_what_the_calls_take(operators):
    from paper_2311_09445_b200 import layers, routing
    cases, rng = operators.listed(), random.Random(3)
    cases += [operators.draw(rng) for _ in range(300)]
    for c in cases:
        assert operators.work(c)["bytes"] > 0
        if c["op"] == "experts":
            assert 1 <= c["rows"] <= layers.MAX_FEW and 1 <= c["k"] <= min(c["experts"], routing.MAX_CHOICES)
            assert max(c["width"], c["hidden"]) <= layers.MAX_INNER and c["experts"] <= routing.MAX_EXPERTS
        elif c["op"] != "dropout":
            assert 1 <= c["width"] <= layers.MAX_WIDTH and c["ld"] in (0,) or c["ld"] >= c["width"]


def test_generator_has_the_known_answers(operators):
    for line in golden_lines("philox4x32_10_kat.txt"):
        words = [int(v, 16) for v in line]
        c = tuple(torch.tensor([w]) for w in words[:4])
        for i in range(10):
            c = operators._philox_round(c, (words[4] + i * 0x9E3779B9) & 0xFFFFFFFF, (words[5] + i * 0xBB67AE85) & 0xFFFFFFFF)
        assert [int(w) for w in c] == words[6:]


def test_both_forms_of_the_mask_agree(operators):
    c = operators.dropout("", "fp32", 9, 21, 0.3)
    s = {"case": c, "x": torch.zeros(9, 21), "seed": (5 << 32) + 7, "call": (3 << 32) + 9}
    assert np.array_equal(operators._kept(s).numpy(), operators._exact_kept(c, s["seed"], s["call"]).numpy())


def test_a_pass_uses_the_handle_of_the_current_stream(operators, monkeypatch):
    import paper_2311_09445_b200 as package
    streams, device = {0: 16, 1: 16}, [0]                            # (two devices' streams may have one number)
    cuda = operators.torch.cuda
    monkeypatch.setattr(cuda, "current_device", lambda: device[0])
    monkeypatch.setattr(cuda, "current_stream", lambda d=None: (device[0] if d is None else d, streams[device[0] if d is None else d]))
    monkeypatch.setattr(operators.torch._C, "_cuda_getCurrentRawStream", lambda d: streams[d], raising=False)
    monkeypatch.setattr(package, "RowLayers", lambda device=None, stream=None: types.SimpleNamespace(stream=stream))
    state, handles = {"case": {}}, []
    for raw in (16, 16, 32, 16):
        streams[0] = raw
        handles.append(operators._handle(state))
        assert handles[-1].stream == (0, raw)
    assert handles[0] is handles[1] is handles[3]
    device[0] = 1
    assert operators._handle({"case": {}}).stream == (1, 16)
