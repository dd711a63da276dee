"""include/pearl_layers.h: its symbols, what its calls and the binding refuse before they touch a device, and the rules that its kernels'
sources follow (no GPU needed)."""
import ctypes as C
import glob
import os
import re

import numpy as np
import pytest
import torch

import layer_reference as ref
from conftest import ROOT, golden_lines
from paper_2311_09445_b200 import RowLayers, layers
from test_rows_binding import Library, ints, meta
from test_rows_sources import code

NULL, BAD_BATCH, ALIGN, OOM, BAD_ARG = -1, -3, -5, -6, -7
F32, F16, BF16 = 0, 1, 2
HEADER = os.path.join(ROOT, "include", "pearl_layers.h")
SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2311_09445_b200", "csrc", "layer_*")))
P = 4096            # an address that nobody follows


@pytest.fixture(scope="module")
def lib():
    from paper_2311_09445_b200 import build
    build.build()
    return layers.load_library()


@pytest.fixture(scope="module")
def handle():
    """Stands for a handle: a call that is refused does not look into it."""
    return C.cast(C.create_string_buffer(256), C.c_void_p)


def test_header_symbols_are_exported_and_bound(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(pearl_layer_[a-z_]+)\s*\(", text)))
    assert names == sorted(layers.SIGNATURES)
    for name in names:
        assert hasattr(lib, name), name


def test_limits_are_those_of_the_header():
    text = open(HEADER).read()
    for name in ("WIDTH", "FEW", "INNER"):
        assert int(re.search(r"#define PEARL_LAYER_MAX_%s (\d+)u" % name, text).group(1)) == getattr(layers, "MAX_" + name)


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_load_may_move_ahead_of_the_wait_for_the_kernel_before(path):
    for promise in (r"__restrict__", r"__ldg\b", r"__ldc[agsv]\b", r"ld\.global(?:\.\w+)*\.nc\b"):
        assert not re.search(promise, code(path)), promise


@pytest.mark.parametrize("path", [p for p in SOURCES if p.endswith(".cu") and "__global__" in code(p)], ids=os.path.basename)
def test_every_kernel_waits_for_the_one_before(path):
    bodies = re.split(r"__global__", code(path))[1:]
    assert bodies and all("rows_begin();" in body for body in bodies)


def test_norm_refuses(lib, handle):
    def norm(T=4, D=8, dtype=BF16, x=P, ld=8, ptype=F32, gamma=P, beta=P, eps=1e-5, y=P, ld_y=8, mean=P, rstd=P, h=handle):
        return lib.pearl_layer_norm(h, T, D, dtype, x, ld, ptype, gamma, beta, eps, y, ld_y, mean, rstd)

    assert norm(h=None) == NULL and norm(T=0) == 0
    for bad in (dict(D=0), dict(D=65537, ld=65537, ld_y=65537), dict(dtype=3), dict(ptype=F16), dict(ptype=5), dict(ld=7), dict(ld_y=7), dict(eps=-1e-9),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(ld=(1 << 40) + 1)):
        assert norm(**bad) == BAD_ARG, bad
    assert norm(T=1 << 31) == BAD_BATCH
    for bad in (dict(x=None), dict(y=None)):
        assert norm(**bad) == NULL, bad
    for bad in (dict(x=P + 1), dict(y=P + 1), dict(gamma=P + 2), dict(beta=P + 2), dict(mean=P + 2), dict(rstd=P + 1), dict(ptype=BF16, gamma=P + 1)):
        assert norm(**bad) == ALIGN, bad


def test_norm_grad_refuses(lib, handle):
    def grad(T=4, D=8, dtype=F16, dy=P, ld_dy=8, x=P, ld_x=8, mean=P, rstd=P, ptype=F16, gamma=P, dx=P, ld_dx=8, dg=P, db=P, work=P,
             size=4 * 2 * 8 * 4, h=handle):
        return lib.pearl_layer_norm_grad(h, T, D, dtype, dy, ld_dy, x, ld_x, mean, rstd, ptype, gamma, dx, ld_dx, dg, db, work, size)

    assert lib.pearl_layer_norm_grad_work_bytes(4, 8) == 4 * 2 * 8 * 4 and lib.pearl_layer_norm_grad_work_bytes(0, 8) > 0
    assert lib.pearl_layer_norm_grad_work_bytes(4, 0) == 0 and lib.pearl_layer_norm_grad_work_bytes(4, 65537) == 0
    assert grad(h=None) == NULL and grad(T=0, dg=None, db=None) == 0
    for bad in (dict(D=0), dict(D=65537, ld_dy=1 << 17, ld_x=1 << 17, ld_dx=1 << 17), dict(dtype=3), dict(ptype=BF16), dict(ld_dy=7), dict(ld_x=7), dict(ld_dx=7)):
        assert grad(**bad) == BAD_ARG, bad
    assert grad(T=1 << 31) == BAD_BATCH
    for bad in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(work=None), dict(dx=None, dg=None, db=None)):
        assert grad(**bad) == NULL, bad
    for bad in (dict(dy=P + 1), dict(x=P + 1), dict(dx=P + 1), dict(gamma=P + 1), dict(mean=P + 2), dict(rstd=P + 2), dict(dg=P + 2), dict(db=P + 2), dict(work=P + 128)):
        assert grad(**bad) == ALIGN, bad
    assert grad(size=4 * 2 * 8 * 4 - 1) == OOM


def test_dropout_refuses(lib, handle):
    def drop(T=4, D=8, dtype=F32, x=P, ld=8, r=P, ld_r=8, p=0.1, calls=P, y=2 * P, ld_y=8, h=handle):
        return lib.pearl_layer_dropout(h, T, D, dtype, x, ld, r, ld_r, p, 1, 2, calls, y, ld_y)

    assert drop(h=None) == NULL and drop(T=0) == 0
    for bad in (dict(D=0), dict(D=(1 << 21) + 1, ld=1 << 22, ld_r=1 << 22, ld_y=1 << 22), dict(dtype=3), dict(ld=7), dict(ld_r=7), dict(ld_y=7), dict(p=-0.01),
                dict(p=1.01), dict(p=float("nan")), dict(y=P, ld_y=9), dict(x=3 * P, y=P, ld_y=9)):
        assert drop(**bad) == BAD_ARG, bad
    assert drop(T=1 << 31) == BAD_BATCH
    for bad in (dict(x=None), dict(y=None)):
        assert drop(**bad) == NULL, bad
    for bad in (dict(x=P + 2), dict(y=P + 2), dict(r=P + 1), dict(calls=P + 4)):
        assert drop(**bad) == ALIGN, bad


def test_expert_layer_refuses(lib, handle):
    def layer(T=4, D=8, H=16, E=4, k=2, dtype=BF16, act=0, x=P, ld=8, router=P, up=P, down=P, w=P, ids=P, y=P, ld_y=8, work=P, size=1 << 40, h=handle):
        return lib.pearl_layer_experts(h, T, D, H, E, k, dtype, act, x, ld, router, 1, up, down, w, ids, y, ld_y, work, size)

    need = lib.pearl_layer_experts_work_bytes
    assert layer(h=None) == NULL and layer(T=0) == 0
    for bad in (dict(D=0), dict(D=65537, ld=1 << 17, ld_y=1 << 17), dict(H=0), dict(H=65537), dict(E=0), dict(E=1025), dict(k=0), dict(k=5), dict(E=64, k=33),
                dict(dtype=3), dict(act=2), dict(ld=7), dict(ld_y=7)):
        assert layer(**bad) == BAD_ARG, bad
    assert layer(T=65) == BAD_BATCH
    for bad in (dict(x=None), dict(up=None), dict(down=None), dict(w=None), dict(ids=None), dict(y=None), dict(work=None)):
        assert layer(**bad) == NULL, bad
    for bad in (dict(x=P + 1), dict(router=P + 1), dict(up=P + 1), dict(down=P + 1), dict(y=P + 1), dict(w=P + 2), dict(ids=P + 2), dict(work=P + 64)):
        assert layer(**bad) == ALIGN, bad
    assert layer(size=need(4, 8, 16, 4, 2) - 1) == OOM
    for bad in ((65, 8, 16, 4, 2), (4, 0, 16, 4, 2), (4, 8, 0, 4, 2), (4, 8, 16, 0, 1), (4, 8, 16, 4, 5), (4, 8, 65537, 4, 2)):
        assert need(*bad) == 0, bad
    sizes = [4, 8, 16, 4, 2]
    for i in range(5):
        more = [n * 2 if j == i else n for j, n in enumerate(sizes)]
        assert need(*more) >= need(*sizes)


# ---- the binding -----------------------------------------------------------------------------------------------------

class Work(Library):
    def __getattr__(self, name):
        if name.endswith("_work_bytes"):
            return lambda *sizes: 1
        return super().__getattr__(name)


@pytest.fixture
def rows():
    r = object.__new__(RowLayers)
    r._h, r._lib, r._ordinal, r.device = None, Work(), -1, torch.device("meta")
    return r


def scratch(n=64):
    return meta(n, dtype=torch.uint8)


CALLS = {
    "norm rows": lambda r, n: r.layer_norm(meta(n, 4), meta(n, 4)),
    "norm width": lambda r, n: r.layer_norm(meta(1, n), meta(1, n)),
    "norm_grad rows": lambda r, n: r.layer_norm_grad(meta(n, 4), meta(n, 4), meta(n), meta(n), None, meta(n, 4)),
    "norm_grad width": lambda r, n: r.layer_norm_grad(meta(1, n), meta(1, n), meta(1), meta(1), None, meta(1, n)),
    "dropout rows": lambda r, n: r.dropout(meta(n, 4), meta(n, 4), 0.1, 1),
    "dropout width": lambda r, n: r.dropout(meta(1, n), meta(1, n), 0.1, 1),
    "layer rows": lambda r, n: r.expert_layer(meta(n, 4), meta(2, 4), meta(2, 6, 4), meta(2, 4, 3), meta(n, 4), meta(n, 1), ints(n, 1), scratch()),
    "layer width": lambda r, n: r.expert_layer(meta(1, n), meta(2, n), meta(2, 6, n), meta(2, n, 3), meta(1, n), meta(1, 1), ints(1, 1), scratch()),
    "layer hidden": lambda r, n: r.expert_layer(meta(1, 4), meta(2, 4), meta(2, 2 * n, 4), meta(2, 4, n), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "layer experts": lambda r, n: r.expert_layer(meta(1, 4), meta(n, 4), meta(n, 6, 4), meta(n, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "layer choices": lambda r, n: r.expert_layer(meta(1, 4), meta(2, 4), meta(2, 6, 4), meta(2, 4, 3), meta(1, 4), meta(1, n), ints(1, n), scratch()),
}


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
def test_counts_that_the_library_has_no_room_for_are_refused(rows, call):
    with pytest.raises(ValueError):
        call(rows, (1 << 32) + 5)
    assert rows._lib.calls == []
    call(rows, 12)
    assert len(rows._lib.calls) == 1


def test_workspaces_of_sizes_without_room_are_refused(rows):
    big = (1 << 32) + 5
    for sizes in ((big, 4), (4, big)):
        with pytest.raises(ValueError):
            rows._work_bytes("pearl_layer_norm_grad_work_bytes", *sizes)
    for i in range(5):
        with pytest.raises(ValueError):
            rows._work_bytes("pearl_layer_experts_work_bytes", *[big if j == i else 4 for j in range(5)])


REFUSED = {
    "another type": lambda r: r.layer_norm(meta(3, 4), meta(3, 4, dtype=torch.float16)),
    "another shape": lambda r: r.layer_norm(meta(3, 4), meta(3, 5)),
    "whole numbers": lambda r: r.layer_norm(ints(3, 4), ints(3, 4)),
    "a transposed matrix": lambda r: r.layer_norm(meta(4, 3).t(), meta(3, 4)),
    "rows that overlap": lambda r: r.layer_norm(meta(3, 1).expand(3, 4), meta(3, 4)),
    "rows at one place": lambda r: r.dropout(meta(3, 4), meta(1, 4).expand(3, 4), 0.1, 1),
    "parameters of two types": lambda r: r.layer_norm(meta(3, 4, dtype=torch.float16), meta(3, 4, dtype=torch.float16), meta(4), meta(4, dtype=torch.float16)),
    "parameters of a third type": lambda r: r.layer_norm(meta(3, 4, dtype=torch.float16), meta(3, 4, dtype=torch.float16), meta(4, dtype=torch.bfloat16)),
    "a short weight": lambda r: r.layer_norm(meta(3, 4), meta(3, 4), meta(3)),
    "a short mean": lambda r: r.layer_norm(meta(3, 4), meta(3, 4), mean=meta(2)),
    "sums without scratch": lambda r: r.layer_norm_grad(meta(3, 4), meta(3, 4), meta(3), meta(3), dgamma=meta(4)),
    "sums of a narrow type": lambda r: r.layer_norm_grad(meta(3, 4), meta(3, 4), meta(3), meta(3), dgamma=meta(4, dtype=torch.float16), work=scratch()),
    "a seed of 65 bits": lambda r: r.dropout(meta(3, 4), meta(3, 4), 0.1, 1 << 64),
    "a negative call": lambda r: r.dropout(meta(3, 4), meta(3, 4), 0.1, 1, -1),
    "calls of 32 bits": lambda r: r.dropout(meta(3, 4), meta(3, 4), 0.1, 1, calls=ints(1)),
    "an ungated weight for a gated layer": lambda r: r.expert_layer(meta(1, 4), None, meta(2, 3, 4), meta(2, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "a router of other experts": lambda r: r.expert_layer(meta(1, 4), meta(3, 4), meta(2, 6, 4), meta(2, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "a weight in columns": lambda r: r.expert_layer(meta(1, 4), None, meta(2, 4, 6).transpose(1, 2), meta(2, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "a weight of another type": lambda r: r.expert_layer(meta(1, 4), None, meta(2, 6, 4, dtype=torch.float16), meta(2, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), scratch()),
    "scratch of floats": lambda r: r.expert_layer(meta(1, 4), None, meta(2, 6, 4), meta(2, 4, 3), meta(1, 4), meta(1, 1), ints(1, 1), meta(64)),
}


@pytest.mark.parametrize("call", REFUSED.values(), ids=REFUSED)
def test_refused(rows, call):
    with pytest.raises(ValueError):
        call(rows)
    assert rows._lib.calls == []


# ---- the definitions that the GPU tests compare with -----------------------------------------------------------------

def test_reference_generator_has_the_known_answers():
    for line in golden_lines("philox4x32_10_kat.txt"):
        words = [int(v, 16) for v in line]
        assert len(words) in (7, 10)
        if len(words) == 10:
            assert ref.philox([[w] for w in words[:4]], words[4:6])[:, 0].tolist() == words[6:]


def test_reference_norm_gradient_against_differences():
    rng = np.random.default_rng(1)
    x, gamma, beta, dy = rng.standard_normal((3, 9)), rng.standard_normal(9), rng.standard_normal(9), rng.standard_normal((3, 9))
    (_, mean, rstd), _ = ref.norm(x, gamma, beta, 1e-3)
    (dx, dg, db), _ = ref.norm_grad(dy, x, mean, rstd, gamma, 4)
    h = 1e-6
    for at, grad in ((0, dx), (1, dg), (2, db)):
        for i in np.ndindex(grad.shape):
            ends = []
            for sign in (1, -1):
                args = [x.copy(), gamma.copy(), beta.copy()]
                args[at][i] += sign * h
                ends.append((ref.norm(*args, 1e-3)[0][0] * dy).sum())
            assert abs((ends[0] - ends[1]) / (2 * h) - grad[i]) < 1e-7


def test_reference_mask_keeps_the_share_and_stays_under_another_width():
    mask, scale = ref.kept(64, 1000, 0.3, 5, 6)
    assert abs(mask.mean() - 0.7) < 0.01 and abs(scale * 0.7 - 1) < 1e-4
    assert (ref.kept(64, 77, 0.3, 5, 6)[0] == mask[:, :77]).all() and (ref.kept(9, 1000, 0.3, 5, 6)[0] == mask[:9]).all()
    assert (ref.kept(64, 1000, 0.3, 5, 7)[0] != mask).any() and (ref.kept(64, 1000, 0.3, 6, 6)[0] != mask).any()
