"""The tests of a layer's operators on special values and of their less common forms against the bounds-checked build, as test_checked_layers.py does;
and that the sources have that build's comparisons where rows are read and written (no GPU needed for that)."""
import os
import re
import subprocess
import sys

import pytest

from conftest import ROOT
from test_rows_sources import code

CSRC = os.path.join(ROOT, "paper_2311_09445_b200", "csrc")


@pytest.mark.gpu
def test_special_values_and_forms_against_the_checked_library():
    from paper_2311_09445_b200 import build
    env = dict(os.environ, PEARL_PRB_LIB=build.build(checked=True))
    files = [os.path.join("tests", name) for name in ("test_gpu_layers_values.py", "test_gpu_layers_forms.py")]
    r = subprocess.run([sys.executable, "-m", "pytest", *files, "-x", "-q", "-m", "gpu"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    assert " passed" in r.stdout and "failed" not in r.stdout, tail


# what reads or writes a row's words: how many such calls a source has, each under a comparison of its own
ACCESSES = {"layer_norm.cu": (r"(?:load|store)_word<E, kBroken>\(", 3), "layer_dropout.cu": (r"layer_(?:load|store)_part<E, N>\(|\bload\(", 5)}


@pytest.mark.parametrize("name", ACCESSES)
def test_row_accesses_are_compared_in_the_checked_build(name):
    call, count = ACCESSES[name]
    text = code(os.path.join(CSRC, name))
    text = re.sub(r"template <[^>]*> __device__ __forceinline__ [^;{]*\{", "", text)
    lines = text.split("\n")
    found = [i for i, line in enumerate(lines) if re.search(call, line)]
    assert len(found) == count
    for i in found:
        assert re.search(r"layer_in_rows<", "\n".join(lines[max(0, i - 2):i + 1])) or "load(" in lines[i], lines[i]
    assert all(re.search(r"layer_in_rows<", body[:400]) for body in text.split("const auto load = ")[1:])
