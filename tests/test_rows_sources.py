"""Rules that the sources of the row operators' kernels follow (no GPU needed)."""
import glob
import os
import re

import pytest

from conftest import ROOT

KERNELS = sorted(glob.glob(os.path.join(ROOT, "paper_2311_09445_b200", "csrc", "rows_*")))


def code(path):
    """The file without its comments."""
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)


@pytest.mark.parametrize("path", KERNELS, ids=os.path.basename)
def test_no_load_may_move_ahead_of_the_wait_for_the_kernel_before(path):
    """Every row kernel is launched while the one before it on the stream may still run, and waits for it before it reads.  A pointer that
    promises unchanging bytes, or a load by the read-only path, would let the compiler or the hardware read earlier."""
    text = code(path)
    for promise in (r"__restrict__", r"__ldg\b", r"__ldc[agsv]\b", r"ld\.global(?:\.\w+)*\.nc\b"):
        assert not re.search(promise, text), promise


@pytest.mark.parametrize("path", [p for p in KERNELS if p.endswith(".cu") and "__global__" in code(p)], ids=os.path.basename)
def test_every_kernel_waits_for_the_one_before(path):
    bodies = re.split(r"__global__", code(path))[1:]
    assert bodies and all("rows_begin();" in body for body in bodies)
