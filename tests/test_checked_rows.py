"""The row operators' tests against the bounds-checked build of the library: an index that a kernel computed and that is out of its
extent raises PEARL_ST_INTERNAL there, and those tests ask for a clean status word."""
import os
import subprocess
import sys

import pytest

from conftest import ROOT

pytestmark = pytest.mark.gpu


def test_row_operators_against_the_checked_library():
    from paper_2311_09445_b200 import build
    env = dict(os.environ, PEARL_PRB_LIB=build.build(checked=True))
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join("tests", "test_gpu_rows.py"), "-x", "-q", "-m", "gpu"], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=900)
    tail = r.stdout[-3000:] + r.stderr[-2000:]
    assert r.returncode == 0, tail
    assert " passed" in r.stdout and "failed" not in r.stdout, tail
