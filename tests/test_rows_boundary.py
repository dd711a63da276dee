"""include/pearl_rows.h: its symbols, and what its calls refuse before they touch a device (no GPU needed)."""
import ctypes as C
import os
import re

import pytest

from conftest import ROOT

NULL, BAD_BATCH, ALIGN, OOM, BAD_ARG = -1, -3, -5, -6, -7
F32, F16, BF16 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2311_09445_b200 import build
    build.build()
    from paper_2311_09445_b200 import routing
    return routing.load_library()


@pytest.fixture(scope="module")
def handle():
    """Stands for a handle: a call that is refused does not look into it."""
    return C.cast(C.create_string_buffer(256), C.c_void_p)


def declared_symbols():
    text = open(os.path.join(ROOT, "include", "pearl_rows.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(pearl_rows_[a-z_]+)\s*\(", text)))


def test_header_symbols_are_exported_and_bound(lib):
    from paper_2311_09445_b200 import routing
    assert declared_symbols() == sorted(routing.SIGNATURES)
    for name in declared_symbols():
        assert hasattr(lib, name), name


def test_limits_are_those_of_the_header():
    from paper_2311_09445_b200 import routing
    text = open(os.path.join(ROOT, "include", "pearl_rows.h")).read()
    for name in ("EXPERTS", "ROW_BYTES", "CHOICES", "BEAMS", "BEST", "VOCAB"):
        value = re.search(r"#define PEARL_ROWS_MAX_%s (.*?)(?:/\*|$)" % name, text, re.M).group(1)
        assert eval(value.replace("u", "")) == getattr(routing, "MAX_" + name)


P = 4096            # an address that nobody follows


def test_create_refuses(lib):
    h = C.c_void_p()
    assert lib.pearl_rows_create(None, 0, None, None, 0) == NULL
    assert lib.pearl_rows_create(C.byref(h), 0, None, P, lib.pearl_rows_slab_bytes() - 1) == OOM
    assert lib.pearl_rows_create(C.byref(h), 0, None, P + 16, lib.pearl_rows_slab_bytes()) == ALIGN
    assert lib.pearl_rows_destroy(None) == NULL and lib.pearl_rows_sync(None, None) == NULL
    assert lib.pearl_rows_kernel_launches(None) == 0


def test_route_refuses(lib, handle):
    def route(T=4, E=8, k=2, dtype=F32, logits=P, ld=8, w=P, ids=P, h=handle):
        return lib.pearl_rows_route(h, T, E, k, dtype, logits, ld, 0, w, ids)

    assert route(h=None) == NULL
    assert route(T=0) == 0                                    # nothing to do
    for bad in (dict(E=0), dict(E=1025), dict(k=0), dict(k=9), dict(E=64, k=33, ld=64), dict(dtype=3), dict(ld=7)):
        assert route(**bad) == BAD_ARG, bad
    assert route(T=1 << 30, k=2) == BAD_BATCH
    for bad in (dict(logits=None), dict(w=None), dict(ids=None)):
        assert route(**bad) == NULL, bad
    for bad in (dict(logits=P + 2), dict(dtype=F16, logits=P + 1), dict(w=P + 2), dict(ids=P + 1)):
        assert route(**bad) == ALIGN, bad


def test_route_grad_refuses(lib, handle):
    def grad(T=4, E=8, k=2, dtype=BF16, logits=P, ld=8, chosen=0, w=P, ids=P, dw=P, d=P, ld_d=8, h=handle):
        return lib.pearl_rows_route_grad(h, T, E, k, dtype, logits, ld, chosen, w, ids, dw, d, ld_d)

    assert grad(h=None) == NULL and grad(T=0) == 0
    for bad in (dict(E=0), dict(k=9), dict(dtype=7), dict(ld=7), dict(ld_d=3), dict(E=1025, ld=1025, ld_d=1025)):
        assert grad(**bad) == BAD_ARG, bad
    assert grad(T=1 << 30) == BAD_BATCH
    for bad in (dict(logits=None), dict(w=None), dict(ids=None), dict(dw=None), dict(d=None), dict(d=None, chosen=1)):
        assert grad(**bad) == NULL, bad
    for bad in (dict(logits=P + 1), dict(d=P + 1), dict(dw=P + 2), dict(w=P + 3), dict(ids=P + 2)):
        assert grad(**bad) == ALIGN, bad


def test_sort_refuses(lib, handle):
    def sort(n=4, E=8, ids=P, offsets=P, order=P, place=P, h=handle):
        return lib.pearl_rows_sort(h, n, E, ids, offsets, order, place)

    assert sort(h=None) == NULL
    for bad in (dict(E=0), dict(E=1025)):
        assert sort(**bad) == BAD_ARG
    assert sort(n=1 << 31) == BAD_BATCH
    for bad in (dict(ids=None), dict(offsets=None), dict(place=None)):
        assert sort(**bad) == NULL
    for bad in (dict(ids=P + 1), dict(offsets=P + 2), dict(order=P + 2), dict(place=P + 3)):
        assert sort(**bad) == ALIGN


def test_dispatch_refuses(lib, handle):
    def dispatch(T=4, k=2, row=12, x=P, ld=12, place=P, rows=8, xs=P, h=handle):
        return lib.pearl_rows_dispatch(h, T, k, row, x, ld, place, rows, xs)

    assert dispatch(h=None) == NULL and dispatch(T=0) == 0
    for bad in (dict(row=0), dict(row=(1 << 23) + 1, ld=1 << 24), dict(ld=11)):
        assert dispatch(**bad) == BAD_ARG
    for bad in (dict(k=0), dict(T=1 << 30)):
        assert dispatch(**bad) == BAD_BATCH
    for bad in (dict(x=None), dict(place=None), dict(xs=None)):
        assert dispatch(**bad) == NULL
    assert dispatch(place=P + 2) == ALIGN


def test_combine_refuses(lib, handle):
    def combine(T=4, k=2, D=12, dtype=F32, z=P, rows=8, place=P, w=P, y=P, ld=12, h=handle):
        return lib.pearl_rows_combine(h, T, k, D, dtype, z, rows, place, w, y, ld)

    def grad(T=4, k=2, D=12, dtype=F16, dy=P, ld=12, z=P, rows=8, place=P, w=P, dz=P, dw=P, h=handle):
        return lib.pearl_rows_combine_grad(h, T, k, D, dtype, dy, ld, z, rows, place, w, dz, dw)

    for call in (combine, grad):
        assert call(h=None) == NULL and call(T=0) == 0
        for bad in (dict(D=0), dict(ld=11), dict(dtype=3)):
            assert call(**bad) == BAD_ARG
        for bad in (dict(k=0), dict(T=1 << 30)):
            assert call(**bad) == BAD_BATCH
        for bad in (dict(z=None), dict(place=None)):
            assert call(**bad) == NULL
        for bad in (dict(place=P + 1), dict(w=P + 2), dict(z=P + 1)):
            assert call(**bad) == ALIGN
    assert combine(D=(1 << 21) + 1, ld=1 << 22) == BAD_ARG and grad(D=(1 << 22) + 1, ld=1 << 23) == BAD_ARG
    assert combine(y=None) == NULL and combine(y=P + 2) == ALIGN
    assert grad(dy=None) == NULL and grad(dz=None, dw=None) == NULL
    assert grad(dy=P + 1) == ALIGN and grad(dz=P + 1) == ALIGN and grad(dw=P + 2) == ALIGN


def test_beam_select_refuses(lib, handle):
    def select(G=2, W=4, V=100, best=8, dtype=F32, logits=P, ld=100, scores=P, done=P + 1, s=P, b=P, t=P, h=handle):
        return lib.pearl_rows_beam_select(h, G, W, V, best, dtype, logits, ld, scores, done, 2, s, b, t)

    assert select(h=None) == NULL and select(G=0) == 0
    for bad in (dict(W=0), dict(W=33), dict(V=0), dict(V=(1 << 24) + 1, ld=1 << 25), dict(best=0), dict(best=65), dict(dtype=9), dict(ld=99)):
        assert select(**bad) == BAD_ARG, bad
    assert select(G=(1 << 24) + 1) == BAD_BATCH
    for bad in (dict(logits=None), dict(scores=None), dict(s=None), dict(b=None), dict(t=None)):
        assert select(**bad) == NULL
    for bad in (dict(logits=P + 2), dict(scores=P + 2), dict(s=P + 1), dict(b=P + 2), dict(t=P + 3)):
        assert select(**bad) == ALIGN


def test_beam_reorder_refuses(lib, handle):
    from paper_2311_09445_b200.routing import _States

    def reorder(blocks=2, G=2, W=4, pieces=3, piece=32, parent=P, src=P, sp=(800, 100, 32), dst=1 << 20, dp=(800, 100, 32), h=handle):
        return lib.pearl_rows_beam_reorder(h, blocks, G, W, pieces, piece, parent, src, None if sp is None else C.byref(_States(*sp)),
                                           dst, None if dp is None else C.byref(_States(*dp)))

    assert reorder(h=None) == NULL
    for nothing in (dict(blocks=0), dict(G=0), dict(pieces=0), dict(piece=0)):
        assert reorder(**nothing) == 0
    for bad in (dict(W=0), dict(W=33)):
        assert reorder(**bad) == BAD_ARG
    for bad in (dict(parent=None), dict(src=None), dict(dst=None), dict(sp=None), dict(dp=None)):
        assert reorder(**bad) == NULL
    assert reorder(parent=P + 2) == ALIGN
    for overlap in (dict(dp=(800, 95, 32)),                       # a state runs into the next one
                    dict(dp=(700, 100, 32)),                      # a block into the next one
                    dict(dp=(800, 100, 31)),                      # a piece into the next one
                    dict(dst=P + 1595),                           # the last byte of src is the first of dst
                    dict(src=1 << 20, dst=(1 << 20) - 1595)):
        assert reorder(**overlap) == BAD_ARG, overlap
    assert reorder(dst=P, dp=(1600, 200, 32)) == BAD_ARG          # in place with other pitches
    assert reorder(sp=(1 << 62, 100, 32)) == BAD_ARG


def test_no_cpu_fallback():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    from paper_2311_09445_b200 import RowRouter
    with pytest.raises(RuntimeError):
        RowRouter()
