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


def test_no_cta_leaves_its_cluster_before_all_have_sent():
    """Beam selection's CTAs send lists into one another's shared memory.  A CTA that gives up waiting for them, or has them all, waits at
    the cluster's barrier, at which the others arrive when they have sent theirs, before it leaves."""
    text = code(os.path.join(ROOT, "paper_2311_09445_b200", "csrc", "rows_beam.cu"))
    kernel = text[text.index("select_kernel(const SelectArgs a)"):text.index("struct ReorderArgs")]
    behind = kernel[kernel.index("cluster_arrive_relaxed();"):]
    assert "send(" not in behind
    assert re.search(r"if \(late\) \{\s*cluster_wait\(\);\s*if \(!arrived\(", behind)
    assert re.search(r"if \(!late\) cluster_wait\(\);\s*\}\s*$", behind)


@pytest.mark.parametrize("name,checked", [
    ("rows_route.cu", ["held_id", "mine", "experts", "pitch"]), ("rows_sort.cu", ["slots", "kHeld"]), ("rows_copy.cu", []),
    ("rows_beam.cu", ["kThreads", "a.src_end", "a.dst_end", "units", "a.V"]), ("rows_internal.cuh", ["lo, hi"])])
def test_the_checked_build_has_something_to_check(name, checked):
    """tests/test_checked_rows.py runs the row operators' tests on a build that compares computed indices with their extents: it says
    something about a kernel only where that is written."""
    text = code(os.path.join(ROOT, "paper_2311_09445_b200", "csrc", name))
    checks = re.findall(r"ROWS_IN_(?:BOUNDS|ARRAY)\((.*)", text)
    for what in checked:
        assert any(what in c for c in checks), what
    if "RowsAny<" in text:                                   # rows at odd places: read and stored through the checked helpers, with their extents
        assert re.search(r"\.fetch\((?:a\.)?status, ", text)
        if name != "rows_internal.cuh":
            assert all(c.count(",") >= 6 for c in re.findall(r"rows_store_part<S>\((.*?)\);", text, flags=re.S))


def test_the_sample_kernel_reads_the_tree_behind_the_wait():
    """prb_sample_kernel is launched in the same way, beside the kernel that may be writing the tree."""
    text = code(os.path.join(ROOT, "paper_2311_09445_b200", "csrc", "prb_sample.cu"))
    kernel = text[text.index("prb_sample_kernel(const __grid_constant__"):text.index("prb_leaf_min_kernel(")]
    walk = text[:text.index("prb_sample_kernel(const __grid_constant__")]
    assert "prb_dep_wait();" in kernel and "__ldg" not in kernel and "__ldg" not in walk
