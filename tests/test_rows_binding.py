"""RowRouter's checks of sizes, on tensors without memory (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2311_09445_b200 import RowRouter, routing

BIG = 1 << 32


class Library:
    """Takes every call and says yes."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture
def router(monkeypatch):
    r = object.__new__(RowRouter)
    r._h, r._lib, r._ordinal, r.device = None, Library(), -1, torch.device("meta")
    return r


def meta(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="meta")


def ints(*shape):
    return meta(*shape, dtype=torch.int32)


def best(G, C):
    return meta(G, C), ints(G, C), ints(G, C)


CALLS = {
    "route rows": lambda r, n: r.route(meta(n, 4), meta(n, 2), ints(n, 2)),
    "route experts": lambda r, n: r.route(meta(1, n), meta(1, 2), ints(1, 2)),
    "route choices": lambda r, n: r.route(meta(1, 4), meta(1, n), ints(1, n)),
    "route_grad rows": lambda r, n: r.route_grad(None, meta(n, 2), ints(n, 2), meta(n, 2), meta(n, 4), over_chosen=True),
    "route_grad choices": lambda r, n: r.route_grad(None, meta(1, n), ints(1, n), meta(1, n), meta(1, 4), over_chosen=True),
    "sort slots": lambda r, n: r.sort(ints(n), 8, ints(9), None, ints(n)),
    "sort experts": lambda r, n: r.sort(ints(4), n, ints(n + 1), None, ints(4)),
    "dispatch rows": lambda r, n: r.dispatch(meta(n, 4), ints(n, 1), meta(8, 4)),
    "dispatch row bytes": lambda r, n: r.dispatch(meta(2, n // 4 + 1), ints(2, 1), meta(8, n // 4 + 1)),
    "dispatch choices": lambda r, n: r.dispatch(meta(1, 4), ints(1, n), meta(8, 4)),
    "dispatch sorted rows": lambda r, n: r.dispatch(meta(2, 4), ints(2, 1), meta(n, 4)),
    "combine rows": lambda r, n: r.combine(meta(8, 4), ints(n, 1), None, meta(n, 4)),
    "combine elements": lambda r, n: r.combine(meta(8, n), ints(2, 1), None, meta(2, n)),
    "combine choices": lambda r, n: r.combine(meta(8, 4), ints(1, n), None, meta(1, 4)),
    "combine sorted rows": lambda r, n: r.combine(meta(n, 4), ints(2, 1), None, meta(2, 4)),
    "combine_grad choices": lambda r, n: r.combine_grad(meta(1, 4), meta(8, 4), ints(1, n), None, meta(8, 4)),
    "combine_grad sorted rows": lambda r, n: r.combine_grad(meta(2, 4), None, ints(2, 1), None, meta(n, 4)),
    "beam_select groups": lambda r, n: r.beam_select(meta(n, 1, 4), meta(n, 1), *best(n, 1)),
    "beam_select beams": lambda r, n: r.beam_select(meta(1, n, 4), meta(1, n), *best(1, 1)),
    "beam_select tokens": lambda r, n: r.beam_select(meta(1, 1, n), meta(1, 1), *best(1, 1)),
    "beam_select best": lambda r, n: r.beam_select(meta(1, 1, 4), meta(1, 1), *best(1, n)),
    "beam_reorder blocks": lambda r, n: r.beam_reorder(meta(n, 1, 2, 4), ints(1, 2)),
    "beam_reorder groups": lambda r, n: r.beam_reorder(meta(1, n, 2, 4), ints(n, 2)),
    "beam_reorder beams": lambda r, n: r.beam_reorder(meta(1, 1, n, 4), ints(1, n)),
    "beam_reorder pieces": lambda r, n: r.beam_reorder(meta(1, 1, 2, n, 4)[..., :3], ints(1, 2)),
}


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
def test_counts_that_the_library_has_no_room_for_are_refused(router, call):
    """A count of 2^32 + 5 must not reach the library as 5."""
    with pytest.raises(ValueError):
        call(router, BIG + 5)
    assert router._lib.calls == []


@pytest.mark.parametrize("call", CALLS.values(), ids=CALLS)
def test_ordinary_counts_are_handed_on(router, call):
    call(router, 12)
    assert len(router._lib.calls) == 1


def test_end_token_must_be_a_token(router):
    for end in (1 << 31, -(1 << 31) - 1, BIG + 2):
        with pytest.raises(ValueError):
            router.beam_select(meta(1, 1, 4), meta(1, 1), *best(1, 1), end_token=end)
    assert router._lib.calls == []


def test_unsigned_arguments_are_the_ones_checked():
    """Every 32-bit argument of a call with arrays: their number, so that a new one is not forgotten above."""
    names = [n for n in routing.SIGNATURES if n not in ("pearl_rows_create", "pearl_rows_sync")]
    assert {n: routing.SIGNATURES[n][1].count(routing._u32) for n in names if routing._u32 in routing.SIGNATURES[n][1]} == {
        "pearl_rows_route": 4, "pearl_rows_route_grad": 4, "pearl_rows_sort": 2, "pearl_rows_dispatch": 4, "pearl_rows_combine": 5,
        "pearl_rows_combine_grad": 5, "pearl_rows_beam_select": 5, "pearl_rows_beam_reorder": 4}


def test_states_of_more_groups_than_a_grid_has_blocks_are_refused():
    """pearl_rows_beam_reorder refuses them by its own check, before it looks into the handle, and not by a failed launch."""
    from paper_2311_09445_b200 import build
    build.build()
    lib, handle = routing.load_library(), C.cast(C.create_string_buffer(256), C.c_void_p)
    for blocks, G in ((1 << 16, 1 << 15), (1, 1 << 31), (3, (1 << 30) + 1)):
        states = routing._States(8 * G, 8, 8)
        assert lib.pearl_rows_beam_reorder(handle, blocks, G, 1, 1, 8, 4096, 4096, C.byref(states), 4096, C.byref(states)) == -3
