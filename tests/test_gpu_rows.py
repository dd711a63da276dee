"""The row operators on the GPU against their definitions in 64 bits.

Tolerances count roundings: one of the result to its type (half a step, relative to the value), those of 32-bit sums (one
per addition, relative to the sum of the magnitudes), and the documented error of the exponential.
"""
import itertools
import math

import numpy as np
import pytest
import torch

import rows_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24
BAD_INDEX, BAD_SCORE = 1, 64


@pytest.fixture(scope="module")
def rows():
    from paper_2311_09445_b200 import RowRouter
    r = RowRouter()
    yield r
    r.close()


def gen(*seed):
    g = torch.Generator()
    g.manual_seed(hash(seed) & 0x7FFFFFFF)
    return g


def f64(t):
    return t.double().cpu().numpy()


def strided(x, extra, shift=0):
    """x on the GPU as a view whose rows lie `extra` elements further apart, `shift` elements into the storage."""
    T, D = x.shape
    store = torch.full((T * (D + extra) + shift,), 7, dtype=x.dtype, device="cuda")
    view = store[shift:].view(T, D + extra)[:, :D]
    view.copy_(x)
    return view


# ---- the router ------------------------------------------------------------------------------------------------------

def run_route(rows, logits, k, chosen):
    T = logits.shape[0]
    w = torch.full((T, k), 5.0, device="cuda")
    ids = torch.full((T, k), 99, dtype=torch.int32, device="cuda")
    rows.route(logits, w, ids, over_chosen=chosen)
    return w, ids


def route_tolerance(spread, E):
    # exp(x) with x = l - max in [-spread, 0]: within 2 + 1.2 |x| units of the last place (2^-23 at most, relative), the rounding
    # of x itself another |x| half steps; the sum's additions, and the division
    one = (2 + 1.2 * spread) * 2 * U + spread * U
    return 2 * one + (E + 3) * U


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (7, 3, 3), (64, 8, 2), (33, 16, 4), (100, 17, 5), (65, 60, 6), (41, 64, 8),
                                   (50, 128, 8), (3, 129, 1), (29, 255, 9), (17, 256, 32), (9, 500, 8), (5, 1000, 17), (2, 1024, 32)])
def test_route(rows, kind, T, E, k):
    l = (torch.randn(T, E, generator=gen(1, T, E, k)) * 1.5).clamp(-5, 5).to(TYPES[kind])
    for chosen in (False, True):
        w, ids = run_route(rows, l.cuda(), k, chosen)
        want_w, want_ids = ref.route(f64(l), k, chosen)
        assert (ids.cpu().numpy() == want_ids).all()
        np.testing.assert_allclose(f64(w), want_w, rtol=route_tolerance(10, E), atol=0)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind,E,extra,shift", [("fp32", 60, 3, 1), ("bf16", 128, 1, 1), ("fp16", 200, 8, 2), ("bf16", 64, 4, 4), ("fp32", 1024, 4, 4)])
def test_route_rows_apart(rows, kind, E, extra, shift):
    l = torch.randn(37, E, generator=gen(2, E)).to(TYPES[kind])
    view = strided(l, extra, shift)
    w, ids = run_route(rows, view, 4, False)
    dense_w, dense_ids = run_route(rows, l.cuda(), 4, False)
    assert torch.equal(w, dense_w) and torch.equal(ids, dense_ids)
    dw = torch.randn(37, 4, generator=gen(3)).cuda()
    d = strided(torch.zeros_like(l), extra, shift)
    rows.route_grad(view, w, ids, dw, d)
    dense = torch.zeros_like(l).cuda()
    rows.route_grad(l.cuda(), w, ids, dw, dense)
    assert torch.equal(d, dense)
    around = d._base.clone()
    around[shift:].view(37, E + extra)[:, :E] = 7
    assert (around == 7).all()                              # nothing beside the rows is written


def test_route_ties_go_to_the_lower_expert(rows):
    for E, k in ((8, 8), (40, 7), (128, 8), (300, 20)):
        l = torch.zeros(5, E)
        l[1, E // 2:] = 1.0
        l[2] = torch.arange(E) % 2 * 1.0
        l[3, 1] = -0.0
        w, ids = run_route(rows, l.cuda(), k, True)
        assert (ids.cpu().numpy() == ref.route(l.double().numpy(), k, True)[1]).all()


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("chosen", [False, True])
def test_route_barred_and_lowest(rows, kind, chosen):
    t = TYPES[kind]
    l = torch.randn(8, 20, generator=gen(5)).to(t)
    l[0] = -math.inf                                        # nobody
    l[1, 2:] = -math.inf                                    # fewer than k
    l[2] = torch.finfo(t).min                               # all at the type's lowest value: an ordinary tie
    l[3, 1:] = torch.finfo(t).min                           # one far above the others
    l[4] = torch.finfo(t).max                               # the largest finite value
    l[5, ::2] = -math.inf
    w, ids = run_route(rows, l.cuda(), 4, chosen)
    want_w, want_ids = ref.route(f64(l), 4, chosen)
    assert (ids.cpu().numpy() == want_ids).all()
    np.testing.assert_allclose(f64(w), want_w, rtol=route_tolerance(10, 20), atol=1e-37)
    dw = torch.randn(8, 4, generator=gen(6))
    d = torch.full((8, 20), 3.0, dtype=t, device="cuda")
    rows.route_grad(l.cuda(), w, ids, dw.cuda(), d, over_chosen=chosen)
    assert torch.isfinite(d).all() and (d[0] == 0).all()
    assert (d[1, 2:] == 0).all() and (d[5, ::2] == 0).all()
    assert rows.sync() == 0


def test_route_reports_nan_and_infinity(rows):
    l = torch.randn(6, 12, generator=gen(7))
    clean = l.clone()
    for t, e, v in ((1, 3, math.nan), (2, 0, math.inf), (4, 11, -math.nan)):
        l[t, e] = v
        clean[t, e] = -math.inf
    w, ids = run_route(rows, l.cuda(), 5, False)
    assert rows.sync() == BAD_SCORE and rows.sync() == 0
    want_w, want_ids = run_route(rows, clean.cuda(), 5, False)
    assert torch.equal(w, want_w) and torch.equal(ids, want_ids) and rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("chosen", [False, True])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 8, 2), (31, 33, 4), (64, 128, 8), (9, 257, 3), (3, 1024, 32)])
def test_route_grad(rows, kind, chosen, T, E, k):
    l = (torch.randn(T, E, generator=gen(8, T, E, k)) * 1.5).clamp(-5, 5).to(TYPES[kind])
    dw = torch.randn(T, k, generator=gen(9, T, E, k))
    w, ids = run_route(rows, l.cuda(), k, chosen)
    d = torch.full((T, E), 3.0, dtype=TYPES[kind], device="cuda")
    rows.route_grad(None if chosen else l.cuda(), w, ids, dw.cuda(), d, over_chosen=chosen)
    exact_w, at = ref.route(f64(l), k, chosen)
    want = ref.route_grad(f64(l), exact_w, at, dw.double().numpy(), chosen, E)
    # p (g - mean): p and w within the router's tolerance, the mean's k products and additions; magnitudes up to p (|g| + sum |w dw|)
    size = (np.abs(dw.double().numpy()).max(1, keepdims=True) * 2) * np.ones((T, E))
    p = np.exp(f64(l) - f64(l).max(1, keepdims=True))
    p /= p.sum(1, keepdims=True) if not chosen else np.maximum(p.max(1, keepdims=True), 1e-300)
    tol = (route_tolerance(10, E) * 2 + (k + 4) * U) * size * (p if not chosen else 1.0)
    assert (np.abs(f64(d) - want) <= tol + ref.HALF_STEP[kind] * np.abs(want) * 1.01 + 2.0 ** -24 * (kind == "fp16")).all()
    assert rows.sync() == 0


def test_route_grad_same_expert_twice_and_bad_ids(rows):
    """Ids that did not come from the router: a repeated one gets both gradients, one out of range is left out and reported."""
    l = torch.randn(3, 10, generator=gen(10))
    ids = torch.tensor([[4, 4, 1], [9, 10, 2], [-1, -2, 0]], dtype=torch.int32)
    w, dw = torch.rand(3, 3, generator=gen(11)), torch.randn(3, 3, generator=gen(12))
    d = torch.zeros(3, 10, device="cuda")
    for chosen in (True, False):
        rows.route_grad(l.cuda(), w.cuda(), ids.cuda(), dw.cuda(), d, over_chosen=chosen)
        want = ref.route_grad(f64(l), f64(w), ids.numpy(), f64(dw), chosen, 10)
        np.testing.assert_allclose(f64(d), want, rtol=0, atol=40 * U * 4)
        assert rows.sync() == BAD_INDEX


# ---- the sort --------------------------------------------------------------------------------------------------------

def run_sort(rows, ids, E, with_order=True):
    n = ids.numel()
    offsets = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda") if with_order else None
    place = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    rows.sort(ids.cuda(), E, offsets, order, place)
    return offsets.cpu().numpy(), None if order is None else order.cpu().numpy(), place.cpu().numpy()


@pytest.mark.parametrize("n", [0, 1, 31, 32, 33, 127, 1000, 4096, 8191, 70001, 300000])
@pytest.mark.parametrize("E", [1, 2, 7, 64, 257, 1024])
def test_sort(rows, n, E):
    ids = torch.randint(-1 if n % 2 else 0, E, (n,), generator=gen(20, n, E), dtype=torch.int32)
    offsets, order, place = run_sort(rows, ids, E)
    want_offsets, want_order, want_place = ref.sort(ids.numpy(), E)
    assert (offsets == want_offsets).all() and (place == want_place).all()
    assert (order[:len(want_order)] == want_order).all()
    assert (order[len(want_order):] == -7).all()            # what lies behind the last row is left as it was
    assert rows.sync() == 0


@pytest.mark.parametrize("case", ["one expert", "none", "last only", "alternating", "falling"])
def test_sort_skewed(rows, case):
    n, E = 20011, 100
    ids = {"one expert": torch.full((n,), 37), "none": torch.full((n,), -1), "last only": torch.full((n,), E - 1),
           "alternating": torch.arange(n) % 2 * 99, "falling": (E - 1 - torch.arange(n) * E // n)}[case].to(torch.int32)
    offsets, order, place = run_sort(rows, ids, E)
    want_offsets, want_order, want_place = ref.sort(ids.numpy(), E)
    assert (offsets == want_offsets).all() and (place == want_place).all() and (order[:len(want_order)] == want_order).all()
    assert (run_sort(rows, ids, E, with_order=False)[2] == want_place).all()


def test_sort_reports_bad_ids(rows):
    ids = torch.tensor([3, -1, 8, 2, -5, 0, 2147483647], dtype=torch.int32)
    offsets, order, place = run_sort(rows, ids, 8)
    assert rows.sync() == BAD_INDEX
    assert place.tolist() == [2, -1, -1, 1, -1, 0, -1] and offsets.tolist() == [0, 1, 1, 2, 3, 3, 3, 3, 3] and order[:3].tolist() == [5, 3, 0]


# ---- rows to the experts and back ------------------------------------------------------------------------------------

def places(T, k, dropped, seed):
    """Places as a sort gives them: a permutation, with some slots left out."""
    g = gen(30, T, k, seed)
    n = T * k
    keep = torch.rand(n, generator=g) >= dropped
    place = torch.full((n,), -1, dtype=torch.int64)
    at = torch.nonzero(keep).squeeze(1)
    place[at] = torch.randperm(len(at), generator=g)
    return place.view(T, k).to(torch.int32)


ROWS = [(1, 1, 1), (1, 8, 4096), (3, 2, 17), (64, 2, 17), (5, 3, 8), (10, 4, 1000), (33, 8, 264), (7, 9, 100), (40, 1, 513), (2, 17, 2056),
        (257, 5, 33), (6, 2, 8200), (5, 4, 2047), (3, 7, 4098), (130, 2, 65), (2, 1, 12289)]


@pytest.mark.parametrize("T,k,D", ROWS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.uint8, torch.int64])
def test_dispatch(rows, T, k, D, dtype):
    x = torch.randint(0, 256, (T, D * torch.empty((), dtype=dtype).element_size()), generator=gen(31, T, k, D), dtype=torch.uint8)
    x = x.view(dtype) if dtype != torch.uint8 else x
    place = places(T, k, 0.25, 1)
    n = int((place >= 0).sum())
    for view in (x.cuda(), strided(x, 3, 1), strided(x, 16, 0)):
        xs = torch.zeros((T * k, D), dtype=dtype, device="cuda")
        xs.view(torch.uint8).fill_(0xA5)
        want = xs.cpu().clone()
        rows.dispatch(view, place.cuda(), xs)
        for t, j in itertools.product(range(T), range(k)):
            if place[t, j] >= 0:
                want[place[t, j]] = x[t]
        assert torch.equal(xs.cpu().view(torch.uint8), want.view(torch.uint8))
    assert rows.sync() == 0 and n <= T * k


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("T,k,D", ROWS)
def test_combine(rows, kind, T, k, D):
    t = TYPES[kind]
    place = places(T, k, 0.3, 2)
    z = torch.randn(T * k, D, generator=gen(32, T, k, D)).to(t)
    w = torch.rand(T, k, generator=gen(33, T, k, D))
    for weights in (w, None):
        want, size = ref.combine(f64(z), place.numpy(), None if weights is None else f64(w))
        for y in (torch.full((T, D), 9.0, dtype=t, device="cuda"), strided(torch.zeros(T, D, dtype=t), 5, 3), strided(torch.zeros(T, D, dtype=t), 8, 8)):
            rows.combine(z.cuda(), place.cuda(), None if weights is None else w.cuda(), y)
            # k additions (a fused product each) in 32 bits, then one rounding; half steps below fp16's normal range are absolute
            tol = k * U * size + ref.HALF_STEP[kind] * (np.abs(want) + k * U * size) + (2.0 ** -25 if kind == "fp16" else 0)
            assert (np.abs(f64(y) - want) <= tol).all()
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("T,k,D", ROWS)
def test_combine_grad(rows, kind, T, k, D):
    t = TYPES[kind]
    place = places(T, k, 0.3, 3)
    z, dy = torch.randn(T * k, D, generator=gen(34, T, k, D)).to(t), torch.randn(T, D, generator=gen(35, T, k, D)).to(t)
    w = torch.rand(T, k, generator=gen(36, T, k, D))
    want_dz, want_dw, size = ref.combine_grad(f64(dy), f64(z), place.numpy(), f64(w))
    unit = torch.finfo(t).tiny * torch.finfo(t).eps / 2
    for g in (dy.cuda(), strided(dy, 5, 3), strided(dy, 8, 8)):
        dz = torch.full((T * k, D), 9.0, dtype=t, device="cuda")
        dw = torch.full((T, k), 9.0, device="cuda")
        rows.combine_grad(g, z.cuda(), place.cuda(), w.cuda(), dz, dw)
        named = np.zeros(T * k, bool)
        named[place[place >= 0].numpy()] = True
        assert (f64(dz)[~named] == 9.0).all()               # rows that no slot names are left as they were
        # one product in 32 bits, one rounding
        assert (np.abs(f64(dz) - want_dz)[named] <= (ref.HALF_STEP[kind] + 1.01 * U) * np.abs(want_dz)[named] + unit).all()
        # D fused products and additions (fewer in a row, but at most D)
        assert (np.abs(f64(dw) - want_dw) <= D * U * size).all()
        only_dz, only_dw = torch.full_like(dz, 9.0), torch.full_like(dw, 9.0)
        rows.combine_grad(g, None, place.cuda(), w.cuda(), only_dz, None)
        rows.combine_grad(g, z.cuda(), place.cuda(), None, None, only_dw)
        assert torch.equal(only_dz, dz) and torch.equal(only_dw, dw)
    # weights of 1: the gradient of dispatch's answer is the row itself
    ones = torch.full((T * k, D), 9.0, dtype=t, device="cuda")
    rows.combine_grad(dy.cuda(), None, place.cuda(), None, ones, None)
    for tt, j in itertools.product(range(T), range(k)):
        if place[tt, j] >= 0:
            assert torch.equal(ones[int(place[tt, j])].cpu(), dy[tt])
    assert rows.sync() == 0


def test_rows_report_bad_places(rows):
    """A place beyond the sorted rows, or below -1, is skipped and reported by each call."""
    place = torch.tensor([[0, 4], [-2, 1], [5, -1], [2147483647, 3]], dtype=torch.int32)
    x, z = torch.randn(4, 40, generator=gen(40)), torch.randn(4, 40, generator=gen(41))
    good = torch.where((place >= 0) & (place < 4), place, torch.full_like(place, -1))
    xs = torch.zeros(4, 40, device="cuda")
    rows.dispatch(x.cuda(), place.cuda(), xs)
    assert rows.sync() == BAD_INDEX
    assert torch.equal(xs.cpu(), torch.stack([x[0], x[1], torch.zeros(40), x[3]]))
    y, want = torch.zeros(4, 40, device="cuda"), torch.zeros(4, 40, device="cuda")
    rows.combine(z.cuda(), place.cuda(), None, y)
    assert rows.sync() == BAD_INDEX
    rows.combine(z.cuda(), good.cuda(), None, want)
    assert rows.sync() == 0 and torch.equal(y, want)
    out = [(torch.zeros(4, 40, device="cuda"), torch.zeros(4, 2, device="cuda")) for _ in range(2)]
    rows.combine_grad(x.cuda(), z.cuda(), place.cuda(), None, *out[0])
    assert rows.sync() == BAD_INDEX
    rows.combine_grad(x.cuda(), z.cuda(), good.cuda(), None, *out[1])
    assert rows.sync() == 0 and all(torch.equal(a, b) for a, b in zip(*out))


def test_combine_infinities_and_nan_stay_in_their_rows(rows):
    z = torch.randn(6, 50, generator=gen(42))
    z[1, 7], z[2, 8], z[5] = math.inf, math.nan, math.nan
    place = torch.tensor([[0, 1], [2, 3], [4, -1]], dtype=torch.int32)        # row 5 is named by nobody
    y = torch.zeros(3, 50, device="cuda")
    rows.combine(z.cuda(), place.cuda(), torch.ones(3, 2, device="cuda"), y)
    y = y.cpu()
    assert y[0, 7] == math.inf and torch.isfinite(y[0, :7]).all() and math.isnan(y[1, 8]) and torch.isfinite(y[2]).all()


# ---- beam search: selection ------------------------------------------------------------------------------------------

def run_select(rows, logits, scores, C, done=None, end=2):
    G = logits.shape[0]
    out = (torch.full((G, C), 5.0, device="cuda"), torch.full((G, C), 77, dtype=torch.int32, device="cuda"),
           torch.full((G, C), 77, dtype=torch.int32, device="cuda"))
    rows.beam_select(logits, scores.cuda(), *out, done=None if done is None else done.cuda(), end_token=end)
    return tuple(o.cpu().numpy() for o in out)


def check_select(rows, logits, scores, C, done=None, end=2, view=None):
    got = run_select(rows, logits.cuda() if view is None else view, scores, C, done, end)
    for g in range(logits.shape[0]):
        ref.check_selection(got[0][g], got[1][g], got[2][g], f64(logits[g]), f64(scores[g]), None if done is None else done[g].numpy(), end, C)
    return got


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("G,W,V,C", [(1, 1, 1, 1), (1, 1, 1, 4), (2, 3, 2, 5), (1, 4, 300, 8), (3, 5, 1001, 10), (2, 1, 32003, 4), (1, 8, 20000, 16),
                                     (2, 2, 50001, 64), (1, 17, 2047, 34), (1, 32, 4099, 64), (5, 4, 2056, 1), (1, 1, 131072, 2), (40, 3, 777, 6)])
def test_beam_select(rows, kind, G, W, V, C):
    logits = (torch.randn(G, W, V, generator=gen(50, G, W, V, C)) * 2.5).to(TYPES[kind])
    scores = -20 * torch.rand(G, W, generator=gen(51, G, W, V, C))
    check_select(rows, logits, scores, C)
    done = torch.rand(G, W, generator=gen(52, G, W)) < 0.3
    check_select(rows, logits, scores, C, done.to(torch.uint8), end=11)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("V,extra,shift", [(5000, 0, 1), (5001, 2, 0), (4096, 4, 3), (4097, 1, 5), (20011, 3, 7)])
def test_beam_select_any_alignment(rows, kind, V, extra, shift):
    """Rows at every offset from a 16-byte boundary; equal rows give equal sums wherever they lie, so ties go to the lower beam."""
    W, C = 9, 18
    row = (torch.randn(1, V, generator=gen(53, V)) * 2.5).to(TYPES[kind])
    logits = row.expand(W, V).contiguous().view(1, W, V)
    view = strided(logits[0], extra, shift).unsqueeze(0)
    scores = torch.full((1, W), -1.5)
    got = check_select(rows, logits, scores, C, view=view)
    dense = run_select(rows, logits.cuda(), scores, C)
    assert all((a == b).all() for a, b in zip(got, dense))
    assert got[1][0].tolist() == list(range(W)) * 2 or f64(row)[0].max() == np.sort(f64(row)[0])[-2]
    assert rows.sync() == 0


def test_beam_select_ties(rows):
    for V, W, C in ((10, 3, 8), (5000, 2, 64), (40000, 1, 64), (33333, 4, 20)):
        logits = torch.zeros(1, W, V)
        got = run_select(rows, logits.cuda(), torch.zeros(1, W), C)
        n = min(C, W * V)
        assert got[1][0][:n].tolist() == [i // V for i in range(n)] and got[2][0][:n].tolist() == [i % V for i in range(n)]
        logits = (torch.arange(V) % 3 == 1).float().expand(1, W, V).contiguous()
        scores = torch.arange(W).float().view(1, W) * -0.25
        check_select(rows, logits, scores, C)


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_beam_select_crowded(rows, kind):
    """Rows whose best logits lie where one team of threads reads, in rising and in falling order: more of them reach the first
    bound than are sorted at once."""
    V = 200000
    rising = torch.arange(V).float() / 1000
    for l in (rising, rising.flip(0), torch.where(torch.arange(V) % 2048 < 16, rising + 500, rising * 0.01)):
        logits = l.to(TYPES[kind]).view(1, 1, V)
        for C in (1, 16, 64):
            check_select(rows, logits, torch.zeros(1, 1), C)


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("V", [1500, 60011])
def test_beam_select_magnitudes(rows, kind, V):
    """Logits around values of every size, on both sides of 2^20 (where the sums change their way) among others."""
    t = TYPES[kind]
    bases = [-40.0, -300.0, 300.0, 6e4, -6e4]
    if kind != "fp16":
        bases += [1048576.0 - 20, 1048576.0 + 20, -1048576.0 - 20, -1048576.0 + 20, 1e6, 3e6, -3e6, 1e30, -1e30, 2.5e38, -3e38]
    noise = torch.randn(1, 2, V, generator=gen(59, V))
    for base in bases:
        for spread in (2.0, 1000.0):
            logits = (noise * spread + base).to(t)
            check_select(rows, logits, torch.tensor([[0.0, -0.5]]), 9)
    assert rows.sync() == 0
    # ordinary rows with a few logits that are far above or far below, or not numbers
    for value in (3e4,) if kind == "fp16" else (2e6, 3e38, -3e38):
        for at in ([0], [V - 1], [5, 6, V // 2, V // 2 + 1], list(range(0, V, 700))):
            logits = (noise * 3).to(t)
            logits[0, :, at] = value
            check_select(rows, logits, torch.tensor([[0.0, -0.5]]), 9)
            logits[0, 0, 3::311] = math.nan
            logits[0, 1, 1::411] = math.inf
            assert rows.sync() == 0
            check_select(rows, logits, torch.tensor([[0.0, -0.5]]), 9)
            assert rows.sync() == BAD_SCORE


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_beam_select_equal_long_rows(rows, kind):
    """Equal rows of many accesses have equal sums at every offset from a 16-byte boundary."""
    V, W, C = 60013, 9, 18
    row = (torch.randn(1, V, generator=gen(60)) * 4).to(TYPES[kind])
    row[0, 30000:30100] += 14.0
    logits = row.expand(W, V).contiguous().view(1, W, V)
    scores = torch.full((1, W), -1.5)
    dense = check_select(rows, logits, scores, C)
    for extra, shift in ((1, 0), (3, 5), (0, 3), (8, 7)):
        got = check_select(rows, logits, scores, C, view=strided(logits[0], extra, shift).unsqueeze(0))
        assert all((a == b).all() for a, b in zip(got, dense))
    first = np.sort(f64(row)[0])[::-1]
    assert first[0] == first[1] or dense[1][0].tolist()[:W] == list(range(W))


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
def test_beam_select_mostly_masked(rows, kind):
    """Most of a vocabulary barred or masked with the type's lowest value, in blocks that leave some warps without a logit, and more
    logits at the lowest value than are sorted at once."""
    t, V = TYPES[kind], 60000
    lowest = torch.finfo(t).min
    for barred, some in ((30000, 3), (256, 5), (59000, 2), (8 * 32 * 2, 0), (1000, 7)):
        logits = torch.full((1, 2, V), lowest, dtype=t)
        logits[0, :, :barred] = -math.inf
        for i in range(some):
            logits[0, :, barred + 97 * i] = 0.25 * i - 1
        logits[0, 1, 0::2] = -math.inf
        for C in (1, 8, 64):
            check_select(rows, logits, torch.tensor([[0.0, -0.5]]), C)
    # a grammar that allows a run of tokens
    logits = torch.full((1, 3, V), -math.inf, dtype=t)
    logits[0, :, 20000:27000] = torch.randn(3, 7000, generator=gen(57)).to(t)
    check_select(rows, logits, torch.tensor([[0.0, -0.5, -3.0]]), 12)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
def test_beam_select_barred_beams_and_tokens(rows, kind):
    t = TYPES[kind]
    G, W, V, C = 7, 4, 3000, 8
    logits = (torch.randn(G, W, V, generator=gen(54)) * 2).to(t)
    scores = -5 * torch.rand(G, W, generator=gen(55))
    done = torch.zeros(G, W, dtype=torch.uint8)
    scores[0, 1:] = -math.inf                               # the first step: one beam
    logits[1, :, 3:] = -math.inf                            # three tokens a beam
    logits[2] = -math.inf                                   # nothing at all
    logits[3] = torch.finfo(t).min                          # masked with the lowest value: a tie of all tokens
    logits[4, 0, 1:] = torch.finfo(t).min
    scores[5] = -math.inf                                   # no beam is left
    done[6] = 1                                             # all finished
    scores[6, 2] = -math.inf
    got = check_select(rows, logits, scores, C, done)
    assert (got[1][2] == -1).all() and (got[1][5] == -1).all() and (got[1][6] >= 0).sum() == 3
    assert rows.sync() == 0


def test_beam_select_reports_nan_and_infinity(rows):
    logits = torch.randn(3, 2, 5000, generator=gen(56))
    clean = logits.clone()
    for at, v in (((0, 1, 17), math.nan), ((1, 0, 4999), math.inf), ((1, 1, 0), -math.nan), ((2, 0, 2500), math.inf)):
        logits[at] = v
        clean[at] = -math.inf
    scores = torch.zeros(3, 2)
    got = run_select(rows, logits.cuda(), scores, 6)
    assert rows.sync() == BAD_SCORE
    want = run_select(rows, clean.cuda(), scores, 6)
    assert rows.sync() == 0 and all((a == b).all() for a, b in zip(got, want))
    scores[0, 0], scores[1, 1] = math.nan, math.inf
    got = run_select(rows, clean.cuda(), scores, 6)
    assert rows.sync() == BAD_SCORE and (got[1][0] == 1).all() and (got[1][1] == 0).all()


# ---- beam search: states ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("W", [1, 2, 4, 5, 8, 16, 31, 32])
@pytest.mark.parametrize("dtype,heads,length,room,dim", [(torch.float32, 2, 5, 7, 8), (torch.bfloat16, 3, 9, 9, 33), (torch.uint8, 1, 1, 3, 1),
                                                         (torch.float16, 4, 16, 40, 64), (torch.uint8, 2, 3, 4, 5), (torch.float16, 2, 251, 311, 33),
                                                         (torch.uint8, 3, 1700, 1701, 7), (torch.float32, 1, 100, 101, 3), (torch.int64, 1, 17, 19, 1)])
def test_beam_reorder(rows, W, dtype, heads, length, room, dim):
    blocks, G = 3, 2
    g = gen(60, W, dim)
    cache = torch.randint(0, 256, (blocks, G, W, heads, room, dim * torch.empty((), dtype=dtype).element_size()), generator=g, dtype=torch.uint8)
    cache = cache.view(dtype) if dtype != torch.uint8 else cache
    parent = torch.randint(0, W, (G, W), generator=g, dtype=torch.int32)
    parent[0, W // 2] = -1                                  # left as it was
    want = cache.clone()
    other = torch.zeros_like(cache)
    want_other = other.clone()
    for o, q, i in itertools.product(range(blocks), range(G), range(W)):
        if parent[q, i] >= 0:
            want[o, q, i, :, :length] = cache[o, q, parent[q, i], :, :length]
            want_other[o, q, i, :, :length] = cache[o, q, parent[q, i], :, :length]
    there, second = cache.cuda(), other.cuda()
    rows.beam_reorder(there[:, :, :, :, :length], parent.cuda(), second[:, :, :, :, :length])
    rows.beam_reorder(there[:, :, :, :, :length], parent.cuda())
    assert torch.equal(second.cpu().view(torch.uint8), want_other.view(torch.uint8))
    assert torch.equal(there.cpu().view(torch.uint8), want.view(torch.uint8))
    assert rows.sync() == 0


def test_beam_reorder_at_odd_addresses(rows):
    """States that start at every offset from a 16-byte boundary, longer than a block's tile, in place and across."""
    for shift in range(16):
        length = 9001 + shift
        store = torch.randint(0, 256, (2 * 3 * length + shift,), generator=gen(63, shift), dtype=torch.uint8)
        there = store.cuda()
        states = there[shift:].view(1, 2, 3, length)
        parent = torch.tensor([[1, 2, 0], [2, 2, -1]], dtype=torch.int32)
        was = states.clone()
        other = torch.full((2 * 3 * length + 5,), 9, dtype=torch.uint8, device="cuda")
        out = other[5:].view(1, 2, 3, length)
        rows.beam_reorder(states, parent.cuda(), out)
        rows.beam_reorder(states, parent.cuda())
        for g in range(2):
            for i in range(3):
                want = was[0, g, parent[g, i]] if parent[g, i] >= 0 else None
                assert torch.equal(states[0, g, i], want if want is not None else was[0, g, i])
                assert torch.equal(out[0, g, i], want) if want is not None else (out[0, g, i] == 9).all()
        assert torch.equal(there[:shift].cpu(), store[:shift]) and (other[:5] == 9).all()
    assert rows.sync() == 0


def test_beam_reorder_between_layouts(rows):
    """A dense cache into part of a larger one, and histories of tokens; a state at an odd address."""
    src = torch.randn(2, 3, 4, 5, 6, 8, generator=gen(61)).cuda()
    dst = torch.zeros(2, 3, 4, 5, 11, 8, device="cuda")
    parent = torch.tensor([[3, 3, 0, 1], [0, 1, 2, 3], [2, 2, 2, 2]], dtype=torch.int32)
    rows.beam_reorder(src, parent.cuda(), dst[:, :, :, :, 3:9])
    want = torch.stack([src[:, g][:, parent[g].long()] for g in range(3)], 1)
    assert torch.equal(dst[:, :, :, :, 3:9], want) and (dst[:, :, :, :, :3] == 0).all() and (dst[:, :, :, :, 9:] == 0).all()
    back = torch.zeros_like(src)
    rows.beam_reorder(dst[:, :, :, :, 3:9], torch.arange(4, dtype=torch.int32).expand(3, 4).contiguous().cuda(), back)
    assert torch.equal(back, want)
    tokens = torch.randint(0, 1000, (1, 3, 4, 13), generator=gen(62), dtype=torch.int32)
    there = tokens.cuda()
    rows.beam_reorder(there[..., :9], parent.cuda())
    for g in range(3):
        assert torch.equal(there[0, g, :, :9].cpu(), tokens[0, g, parent[g].long(), :9]) and torch.equal(there[0, g, :, 9:].cpu(), tokens[0, g, :, 9:])


def test_beam_reorder_reports_bad_parents(rows):
    states = torch.arange(24.0).view(1, 2, 4, 3).cuda()
    want = states.clone()
    want[0, 0, 2], want[0, 1, 0] = states[0, 0, 1], states[0, 1, 3]
    rows.beam_reorder(states, torch.tensor([[4, -1, 1, -2], [3, 1, 2, 100]], dtype=torch.int32).cuda())
    assert torch.equal(states, want) and rows.sync() == BAD_INDEX


# ---- arguments, streams, graphs --------------------------------------------------------------------------------------

def test_binding_refuses(rows):
    f, i = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    w, p = torch.zeros(4, 2, device="cuda"), torch.zeros(8, 8, device="cuda")
    bad = [lambda: rows.route(f.cpu(), w, i), lambda: rows.route(f.t(), w, i), lambda: rows.route(f, w.double(), i), lambda: rows.route(f, w, i.long()),
           lambda: rows.route(f, w[:, :1], i), lambda: rows.route(f.double(), w, i), lambda: rows.route(f[:1].expand(4, 8), w, i),
           lambda: rows.route_grad(f, w, i, w, torch.zeros(4, 9, device="cuda")), lambda: rows.route_grad(f, w, i, w, f.half()),
           lambda: rows.sort(i, 8, torch.zeros(8, dtype=torch.int32, device="cuda"), i, i), lambda: rows.sort(i.float(), 8, i, i, i),
           lambda: rows.dispatch(f, i[:3], p), lambda: rows.dispatch(f, i, p.half()), lambda: rows.dispatch(f, i, torch.zeros(8, 9, device="cuda")),
           lambda: rows.dispatch(f, i, torch.zeros(8, 16, device="cuda")[:, :8]), lambda: rows.combine(p, i, w[:3], f), lambda: rows.combine(p, i, w, f.half()),
           lambda: rows.combine_grad(f, None, i, w, p, w), lambda: rows.combine_grad(f, p[:7], i, w, p, w), lambda: rows.combine_grad(f, p, i, w, p, w.half()),
           lambda: rows.beam_select(f, w, w, i, i), lambda: rows.beam_select(f.view(2, 2, 8), w, w, i, i),
           lambda: rows.beam_reorder(f.view(1, 2, 2, 8), i), lambda: rows.beam_reorder(f.view(1, 2, 2, 8), i[:2], f.view(1, 2, 2, 8).half()),
           lambda: rows.beam_reorder(f, i)]
    for n, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("not refused:", n)
    from paper_2311_09445_b200 import PearlError
    for call, code in ((lambda: rows.route(f, torch.zeros(4, 9, device="cuda"), torch.zeros(4, 9, dtype=torch.int32, device="cuda")), -7),
                       (lambda: rows.sort(i, 0, torch.zeros(1, dtype=torch.int32, device="cuda"), i, i), -7),
                       (lambda: rows.beam_reorder(p.view(1, 4, 2, 8)[:, 1:3], i[:2].contiguous(), p.view(1, 4, 2, 8)[:, 2:]), -7)):
        with pytest.raises(PearlError) as e:
            call()
        assert e.value.code == code
    assert rows.sync() == 0


def test_empty_batches(rows):
    e = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t, device="cuda")      # noqa: E731
    rows.route(e(0, 8), e(0, 2), e(0, 2, t=torch.int32))
    rows.route_grad(e(0, 8), e(0, 2), e(0, 2, t=torch.int32), e(0, 2), e(0, 8))
    rows.dispatch(e(0, 8), e(0, 2, t=torch.int32), e(0, 8))
    rows.combine(e(0, 8), e(0, 2, t=torch.int32), e(0, 2), e(0, 8))
    rows.combine_grad(e(0, 8), e(0, 8), e(0, 2, t=torch.int32), e(0, 2), e(0, 8), e(0, 2))
    rows.beam_select(e(0, 4, 100), e(0, 4), e(0, 8), e(0, 8, t=torch.int32), e(0, 8, t=torch.int32))
    rows.beam_reorder(e(2, 0, 4, 9), e(0, 4, t=torch.int32))
    # rows, but no sorted rows: every slot was dropped
    y = torch.full((3, 8), 4.0, device="cuda")
    rows.combine(e(0, 8), torch.full((3, 2), -1, dtype=torch.int32, device="cuda"), e(3, 2), y)
    assert (y == 0).all() and rows.sync() == 0


def expert_pass(r, x, wr, experts, k):
    """A layer of experts (one matrix each) with its gradients: outputs and gradients of sum(y * dy)."""
    T, D = x.shape
    i32 = dict(dtype=torch.int32, device=x.device)
    o = {"w": torch.empty(T, k, device=x.device), "ids": torch.empty(T, k, **i32), "offsets": torch.empty(len(experts) + 1, **i32),
         "order": torch.zeros(T * k, **i32), "place": torch.empty(T, k, **i32), "xs": torch.empty(T * k, D, device=x.device),
         "y": torch.empty(T, D, device=x.device), "dz": torch.empty(T * k, D, device=x.device), "dw": torch.empty(T, k, device=x.device),
         "dlogits": torch.empty(T, len(experts), device=x.device), "dx": torch.empty(T, D, device=x.device)}
    o["logits"] = x @ wr
    r.route(o["logits"], o["w"], o["ids"], over_chosen=True)
    r.sort(o["ids"], len(experts), o["offsets"], o["order"], o["place"])
    r.dispatch(x, o["place"], o["xs"])
    return o


def test_experts_on_a_sampled_batch_with_gradients(rows):
    """A learner's pass over a batch drawn from the replay buffer: route, sort, dispatch, the experts, combine, the TD errors back
    into the buffer -- and every gradient against the same layer written densely in 64 bits."""
    from paper_2311_09445_b200 import PrioritizedReplay
    N, B, D, E, k = 2048, 100, 17, 6, 2
    g = gen(70)
    prb = PrioritizedReplay(N, 16, 4 * D, 4, 512)
    for _ in range(4):
        obs = torch.randn(512, D, generator=g).cuda()
        prb.insert(obs.view(torch.uint8), torch.zeros(512, 4, dtype=torch.uint8, device="cuda"), torch.randn(512, generator=g).cuda(),
                   obs.view(torch.uint8), torch.zeros(512, dtype=torch.uint8, device="cuda"), torch.rand(512, generator=g).cuda() + 0.1)
    idx, isw = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
    x, rew = torch.zeros(B, D, device="cuda"), torch.zeros(B, device="cuda")
    prb.sample(B, 0.4, 7, idx, isw, x.view(torch.uint8), rew=rew)
    wr = torch.randn(D, E, generator=g).cuda()
    experts = torch.randn(E, D, D, generator=g).cuda() / D ** 0.5
    o = expert_pass(rows, x, wr, experts, k)
    offsets = o["offsets"].tolist()
    assert offsets[-1] == B * k
    z = torch.cat([o["xs"][a:b] @ experts[e] for e, (a, b) in enumerate(zip(offsets, offsets[1:]))])
    rows.combine(z, o["place"], o["w"], o["y"])
    td = o["y"].mean(1) - rew
    prb.update(idx, td.contiguous(), 0.6, 1e-6)
    assert prb.sync() == 0
    # loss = sum(isw * td^2) / 2
    dy = ((isw * td) / D).unsqueeze(1).expand(B, D).contiguous()
    rows.combine_grad(dy, z, o["place"], o["w"], o["dz"], o["dw"])
    dxs = torch.cat([o["dz"][a:b] @ experts[e].t() for e, (a, b) in enumerate(zip(offsets, offsets[1:]))])
    rows.dispatch_grad(dxs, o["place"], o["dx"])
    rows.route_grad(None, o["w"], o["ids"], o["dw"], o["dlogits"], over_chosen=True)
    dx = o["dx"] + o["dlogits"] @ wr.t()
    dwr = x.t() @ o["dlogits"]
    assert rows.sync() == 0

    x64, wr64, ex64 = x.double().requires_grad_(), wr.double().requires_grad_(), experts.double()
    l = x64 @ wr64
    mask = torch.zeros_like(l).scatter_(1, o["ids"].long(), 1.0)
    p = torch.softmax(l.masked_fill(mask == 0, -math.inf), 1)
    y = torch.einsum("te,td,edf->tf", p, x64, ex64)
    loss = (isw.double() * (y.mean(1) - rew.double()) ** 2).sum() / 2
    loss.backward()
    # sums of at most D * E products of entries of a few units in 32 bits, through four stages
    tol = 4 * D * E * U
    assert (o["y"].double() - y).abs().max() <= tol * y.abs().max()
    assert (dx.double() - x64.grad).abs().max() <= tol * x64.grad.abs().max() * 4
    assert (dwr.double() - wr64.grad).abs().max() <= B * U * 40 * wr64.grad.abs().max()
    prb.close()


def test_beam_search_into_the_buffer(rows):
    """A search of several steps with states that follow the beams, against the same search in 64 bits; the best sequences go into a
    replay buffer with their scores."""
    from paper_2311_09445_b200 import PrioritizedReplay
    G, W, V, S, steps = 3, 4, 501, 24, 6
    g = gen(71)
    table, mix = torch.randn(V, S, generator=g), torch.randn(S, V, generator=g) * 1.3
    state = torch.randn(1, G, 1, S, generator=g).expand(1, G, W, S).contiguous().cuda()
    tokens = torch.zeros(1, G, W, steps, dtype=torch.int32, device="cuda")
    scores = torch.full((G, W), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    done = torch.zeros(G, W, dtype=torch.uint8, device="cuda")
    best = (torch.empty(G, W, device="cuda"), torch.empty(G, W, dtype=torch.int32, device="cuda"), torch.empty(G, W, dtype=torch.int32, device="cuda"))
    end = 0
    paths = [[((), 0.0, state[0, q, 0].cpu().double(), False)] for q in range(G)]
    for step in range(steps):
        logits = (torch.tanh(state[0]) @ mix.cuda()).contiguous()
        before = (f64(logits), f64(scores), done.cpu().numpy())
        rows.beam_select(logits, scores, *best, done=done, end_token=end)
        for q in range(G):
            ref.check_selection(best[0][q].cpu().numpy(), best[1][q].cpu().numpy(), best[2][q].cpu().numpy(), before[0][q], before[1][q],
                                before[2][q], end, W)
        rows.beam_reorder(state, best[1])
        rows.beam_reorder(tokens[..., :step], best[1])
        done = done.gather(1, best[1].long())
        tokens[0, :, :, step] = best[2]
        done |= (best[2] == end).to(torch.uint8)
        state = torch.where(done.view(1, G, W, 1).bool(), state, state * 0.5 + table.cuda()[best[2].long()].unsqueeze(0))
        scores = best[0].clone()
        # the states are those that the tokens so far lead to
        new = []
        for q in range(G):
            new.append([])
            for i in range(W):
                path, s, st, over = paths[q][int(best[1][q, i])] if int(best[1][q, i]) < len(paths[q]) else paths[q][0]
                tok = int(best[2][q, i])
                over = over or tok == end
                new[q].append((path + (tok,), s, st if over else st * 0.5 + table[tok].double(), over))
                assert tuple(tokens[0, q, i, :step + 1].tolist()) == new[q][i][0]
                assert (state[0, q, i].cpu().double() - new[q][i][2]).abs().max() < 1e-5
        paths = new
    assert (np.diff(f64(scores), axis=1) <= 0).all() and rows.sync() == 0
    prb = PrioritizedReplay(64, 4, 4 * steps, 4, 16)
    n = G * W
    prio = torch.exp(scores / steps).view(-1).contiguous()
    prb.insert(tokens.view(n, steps).view(torch.uint8), torch.zeros(n, 4, dtype=torch.uint8, device="cuda"), scores.view(-1).contiguous(),
               tokens.view(n, steps).view(torch.uint8), torch.ones(n, dtype=torch.uint8, device="cuda"), prio)
    assert prb.sync() == 0 and prb.info()[0] == n
    prb.close()


def test_calls_in_a_captured_graph_replayed_with_new_inputs():
    """Two graphs of one handle, replayed in turn on new inputs: nothing is kept from one replay for the next."""
    from paper_2311_09445_b200 import RowRouter
    stream = torch.cuda.Stream()
    g = gen(72)
    with torch.cuda.stream(stream):
        r = RowRouter(stream=stream)
        x, wr = torch.randn(200, 40, generator=g).cuda(), torch.randn(40, 12, generator=g).cuda()
        logits = torch.randn(2, 4, 9001, generator=g).cuda()
        scores = torch.zeros(2, 4, device="cuda")
        states = torch.randn(3, 2, 4, 55, generator=g).cuda()
        best = (torch.empty(2, 4, device="cuda"), torch.empty(2, 4, dtype=torch.int32, device="cuda"), torch.empty(2, 4, dtype=torch.int32, device="cuda"))
        stream.synchronize()
        a, b = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(a, stream=stream):
            o = expert_pass(r, x, wr, range(12), 3)
            r.combine(o["xs"], o["place"], o["w"], o["y"])
            r.combine_grad(x, o["xs"], o["place"], o["w"], o["dz"], o["dw"])
            r.route_grad(o["logits"], o["w"], o["ids"], o["dw"], o["dlogits"], over_chosen=True)
        with torch.cuda.graph(b, stream=stream):
            r.beam_select(logits, scores, *best)
            r.beam_reorder(states, best[1])
        for _ in range(3):
            x.copy_(torch.randn(200, 40, generator=g))
            logits.copy_(torch.randn(2, 4, 9001, generator=g))
            before = states.clone()
            a.replay()
            b.replay()
            stream.synchronize()
            # the weights add up to 1 and the rows come back as they went
            assert (o["y"] - x).abs().max() <= 8 * U * x.abs().max()
            want = expert_pass(r, x, wr, range(12), 3)
            assert all(torch.equal(o[n], want[n]) for n in ("w", "ids", "offsets", "order", "place", "xs"))
            got = [t.cpu().numpy() for t in best]
            for q in range(2):
                ref.check_selection(got[0][q], got[1][q], got[2][q], f64(logits[q]), f64(scores[q]), None, 0, 4)
                assert torch.equal(states[:, q], before[:, q][:, best[1][q].long()])
        assert r.sync() == 0
        a.reset()
        b.reset()
        r.close()


def test_handle_on_its_own_stream_and_two_handles_at_once():
    from paper_2311_09445_b200 import RowRouter
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    handles = [RowRouter(stream=s) for s in streams]
    ids = torch.randint(0, 50, (100000,), generator=gen(73), dtype=torch.int32)
    dev = ids.cuda()
    torch.cuda.synchronize()
    out = []
    for r, s in zip(handles, streams):
        with torch.cuda.stream(s):
            out.append([torch.empty(51, dtype=torch.int32, device="cuda"), torch.empty_like(dev), torch.empty_like(dev)])
    for _ in range(5):
        for r, o in zip(handles, out):
            r.sort(dev, 50, *o)                             # (the current stream is another one: the handle's is used)
    want = ref.sort(ids.numpy(), 50)
    for r, o in zip(handles, out):
        assert r.sync() == 0 and r.kernel_launches() == 5
        assert all((a.cpu().numpy() == b).all() for a, b in zip(o, want))
        r.close()


def test_offsets_past_32_bits(rows):
    """A cache and a matrix of sorted rows of more than 4 GB: the last rows and states are reached."""
    D = 1 << 20
    z = torch.empty(4500, D, dtype=torch.uint8, device="cuda").view(torch.bfloat16)          # 4.7 GB
    z[4400:].normal_()
    place = torch.tensor([[4499, 4400], [4499, -1], [0, 4498]], dtype=torch.int32)
    z[0].fill_(1.0)
    y = torch.empty(3, D // 2, dtype=torch.bfloat16, device="cuda")
    rows.combine(z, place.cuda(), None, y)
    assert torch.equal(y[1], z[4499])
    assert torch.equal(y[0], (z[4499].float() + z[4400].float()).bfloat16())
    x = torch.randn(3, D // 2, generator=gen(74)).bfloat16().cuda()
    rows.dispatch(x, place.cuda(), z)
    assert torch.equal(z[4400], x[0]) and torch.equal(z[4498], x[2]) and torch.equal(z[0], x[2])
    states = z[:4496].view(4, 281, 4, D // 2)
    last, other = states[3, 280].clone(), states[3, 279].clone()
    parent = torch.arange(4, dtype=torch.int32).repeat(281, 1)
    parent[280] = torch.tensor([2, 3, 3, 0])
    rows.beam_reorder(states, parent.cuda())
    assert torch.equal(states[3, 280], last[[2, 3, 3, 0]]) and torch.equal(states[3, 279], other)
    assert rows.sync() == 0


def test_other_device_than_the_current_one():
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    from paper_2311_09445_b200 import RowRouter
    r = RowRouter(device="cuda:1")
    ids = torch.randint(0, 5, (1000,), generator=gen(75), dtype=torch.int32)
    o = [torch.empty(n, dtype=torch.int32, device="cuda:1") for n in (6, 1000, 1000)]
    r.sort(ids.to("cuda:1"), 5, *o)
    assert r.sync() == 0 and torch.cuda.current_device() == 0
    assert all((a.cpu().numpy() == b).all() for a, b in zip(o, ref.sort(ids.numpy(), 5)))
    r.close()


@pytest.mark.parametrize("B", [64, 1000])
def test_rows_right_behind_a_sample(rows, B):
    """The buffer's kernels let the next kernel of the stream start early; what they gather, and the indices and weights that they draw, are
    operands here with nothing in between.  Every pass draws others, so a row, a place or a weight read too early is one of the pass before."""
    from paper_2311_09445_b200 import PrioritizedReplay
    N, D, E = 2048, 17, 5
    g = gen(76)
    prb = PrioritizedReplay(N, 16, 4 * D, 4, 1024)
    obs = torch.randn(N, D, generator=g).cuda()
    for part in obs.split(512):
        prb.insert(part.view(torch.uint8), torch.zeros(512, 4, dtype=torch.uint8, device="cuda"), torch.zeros(512, device="cuda"),
                   part.view(torch.uint8), torch.zeros(512, dtype=torch.uint8, device="cuda"), torch.rand(512, generator=g).cuda() + 0.1)
    idx, isw, x = torch.zeros(B, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, 1, device="cuda"), torch.zeros(B, D, device="cuda")
    place = torch.randperm(B, generator=g).to(torch.int32).view(B, 1).cuda()
    xs, y, w, ids = torch.zeros(B, D, device="cuda"), torch.zeros(B, D, device="cuda"), torch.zeros(B, E, device="cuda"), torch.zeros(B, E, dtype=torch.int32, device="cuda")
    seed = 0

    def draw():
        nonlocal seed
        seed += 1
        prb.sample(B, 0.4, seed, idx.view(-1), isw.view(-1), x.view(torch.uint8))

    for _ in range(25):
        draw()
        rows.dispatch(x, place, xs)
        assert torch.equal(x, obs[idx.view(-1).long()]) and torch.equal(xs[place.view(-1).long()], x)
        draw()
        rows.combine(obs, idx, isw, y)
        assert torch.equal(y, isw * obs[idx.view(-1).long()])
        draw()
        rows.route(x, w, ids, over_chosen=True)
        assert torch.equal(ids.long(), x.topk(E, dim=1).indices)
    assert rows.sync() == 0 and prb.sync() == 0
    prb.close()


def test_beam_select_waits_for_rows_that_are_searched_long(rows):
    """Rows of one value, but for a thread's share, whose bound has to be searched over nearly all logits, in one CTA of a group
    whose other CTAs have finished beams alone and nothing to do but wait."""
    W, V, C = 32, 1 << 22, 64
    logits = torch.zeros(1, W, V, dtype=torch.bfloat16, device="cuda")
    share = logits.view(W, V // 2048, 256, 8)[:4, :-1, 255]                 # the 16-byte accesses of the last of 256 threads, but for its last one
    share.fill_(-1.0)
    scores, done = torch.zeros(1, W), torch.ones(1, W, dtype=torch.uint8)
    scores[0, 4:] = -math.inf
    done[0, :4] = 0
    score, beam, token = run_select(rows, logits, scores, C, done=done)
    lower = int((logits[0, 0] < 0).sum())
    lse = math.log(V - lower + lower * math.exp(-1.0))
    assert (beam[0] == 0).all() and token[0].tolist() == list(range(C))       # four equal beams: the lowest one's lowest tokens
    assert np.abs(score[0] + lse).max() <= 25 * U + 2.0 ** -26 + lse * U
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("E,k", [(8, 8), (64, 6), (128, 8), (500, 8), (60, 20), (1024, 32)])
def test_route_small_weights_keep_their_digits(rows, kind, E, k):
    """One logit far above the others: a row's sum is 1, and a weight is the exponential itself, of a difference that is exact."""
    far = torch.randint(0, 33, (70, E), generator=gen(77, E)).double() / 4            # 27 to 35 below the largest
    l = -23.0 - far
    l[torch.arange(70), torch.randint(0, E, (70,), generator=gen(78, E))] = 4.0
    logits = l.to(TYPES[kind])
    assert torch.equal(logits.double(), l)
    for chosen in (False, True):
        w, ids = run_route(rows, logits.cuda(), k, chosen)
        want_w, want_ids = ref.route(l.numpy(), k, chosen)
        assert (ids.cpu().numpy() == want_ids).all()
        # expf is within 2 units of the last place, 2 * 2^-23 of the value at most: 4 half steps; the sum is 1 + E e^-27 (2^-28); the division 1
        np.testing.assert_allclose(f64(w), want_w, rtol=5.1 * U, atol=0)


@pytest.mark.parametrize("E,k", [(8, 2), (64, 6), (128, 8), (129, 3), (500, 8), (1024, 32)])
def test_route_grad_small_parts_keep_their_digits(rows, E, k):
    """The same rows with dw = 1 for the first choice, whose weight is 1: the gradient of every other expert is -p, its exponential."""
    l = -23.0 - torch.randint(0, 33, (70, E), generator=gen(79, E)).float() / 4
    top = torch.randint(0, E, (70,), generator=gen(80, E))
    l[torch.arange(70), top] = 4.0
    w, ids = run_route(rows, l.cuda(), k, False)
    dw = torch.zeros(70, k)
    dw[:, 0] = 1.0
    d = torch.zeros(70, E, device="cuda")
    rows.route_grad(l.cuda(), w, ids, dw.cuda(), d)
    p = torch.softmax(l.double(), 1).numpy()
    others = np.ones((70, E), bool)
    others[np.arange(70), top.numpy()] = False
    # expf 4 half steps, the sum (1) and its reciprocal and the first weight 1 each, two products 1 each
    np.testing.assert_allclose(f64(d)[others], -p[others], rtol=8.1 * U, atol=0)


def test_no_status_bit_is_lost_between_streams():
    """A graph of the handle, replayed on another stream, raises its bit at any moment of sync(): this answer or the next one has it."""
    from paper_2311_09445_b200 import RowRouter
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(a):
        r = RowRouter(stream=a)
        logits = torch.full((1, 4), math.nan, device="cuda")
        w, ids = torch.zeros(1, 1, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda")
        bad, offsets, place = torch.full((1,), 9, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        r.route(logits, w, ids)
        r.sort(bad, 4, offsets, None, place)
        assert r.sync() == BAD_SCORE | BAD_INDEX
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=a):
            r.route(logits, w, ids)
    assert r.sync() == 0
    for delay in range(0, 120000, 400):                     # (cycles: from before the copy of the word to behind its clearing)
        with torch.cuda.stream(b):
            torch.cuda._sleep(delay)
            graph.replay()
        r.sort(bad, 4, offsets, None, place)
        first = r.sync()
        b.synchronize()
        second = r.sync()
        assert first & BAD_INDEX and not second & BAD_INDEX
        assert (first | second) == BAD_SCORE | BAD_INDEX, delay
        assert r.sync() == 0
    graph.reset()
    r.close()


# ---- loops that only larger calls reach ------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["fp32", "fp16", "bf16"])
@pytest.mark.parametrize("T,k,D", [(3, 2, 8200), (2, 1, 12289), (2, 3, 4097), (5, 2, 2047), (2, 9, 1031), (1, 1, 40000)])
def test_combine_grad_sums_every_element(rows, kind, T, k, D):
    """Small whole numbers: every product and every sum is exact, in any order, so a left out or doubled element shows."""
    z = torch.randint(1, 5, (T * k, D), generator=gen(81, T, k, D)).to(TYPES[kind])
    dy = torch.randint(1, 5, (T, D), generator=gen(82, T, k, D)).to(TYPES[kind])
    place = places(T, k, 0.0, 4)
    want = torch.einsum("td,tkd->tk", dy.double(), z.double()[place.long()])
    assert want.max() < 2 ** 24
    for g in (dy.cuda(), strided(dy, 5, 3), strided(dy, 8, 8)):
        dw = torch.zeros(T, k, device="cuda")
        rows.combine_grad(g, z.cuda(), place.cuda(), None, None, dw)
        assert torch.equal(dw.double().cpu(), want)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("T,E,k,chosen", [(20011, 40, 20, True), (20011, 40, 20, False), (12011, 600, 2, False), (12011, 1024, 8, True), (330011, 8, 2, False),
                                          (330011, 16, 1, True), (90011, 128, 8, False)])
def test_router_with_more_rows_than_the_gpu_holds_at_once(rows, kind, T, E, k, chosen):
    """The gradient's warps take several groups of rows each, one after the other, through the same shared memory; the choice has that
    many blocks.  Against the definition in 64 bits, and the same rows in smaller calls."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(83)
    l = (torch.randn(T, E, device=dev, generator=g) * 1.5).clamp(-5, 5).to(TYPES[kind])
    l.masked_fill_(torch.rand(T, E, device=dev, generator=g) < 0.1, -math.inf)
    l[T // 2] = -math.inf                                   # a row without experts
    dw = torch.randn(T, k, device=dev, generator=g)
    w, ids = run_route(rows, l, k, chosen)
    d = torch.full((T, E), 3.0, dtype=TYPES[kind], device=dev)
    rows.route_grad(None if chosen else l, w, ids, dw, d, over_chosen=chosen)
    step = 1009
    for a in list(range(0, T, step))[::7] + [T - step]:
        part = l[a:a + step].contiguous()
        part_w, part_ids = run_route(rows, part, k, chosen)
        assert torch.equal(part_w, w[a:a + step]) and torch.equal(part_ids, ids[a:a + step])
        part_d = torch.full_like(part, 3.0)
        rows.route_grad(None if chosen else part, part_w, part_ids, dw[a:a + step].contiguous(), part_d, over_chosen=chosen)
        assert torch.equal(part_d, d[a:a + step])

    x = l.double()
    left, at, best = x.clone(), [], []
    for _ in range(k):                                      # the largest that is left, the first of equal ones
        top = left.amax(1, keepdim=True)
        first = torch.where(left == top, torch.arange(E, device=dev), E).amin(1, keepdim=True)
        at.append(torch.where(top == -math.inf, -1, first))
        best.append(top)
        left.scatter_(1, first, -math.inf)
    at, best = torch.cat(at, 1), torch.cat(best, 1)
    assert torch.equal(ids.long(), at)
    top = torch.where(best[:, :1] == -math.inf, 0.0, best[:, :1])
    e = (x - top).exp()
    member = torch.zeros_like(x).scatter_add_(1, at.clamp_min(0), (at >= 0).double())
    p = e * member if chosen else e
    p = p / p.sum(1, keepdim=True).clamp_min(1e-300)
    want_w = torch.where(at < 0, 0.0, p.gather(1, at.clamp_min(0)))
    # two exponentials within 2 units of the last place (4 half steps) of differences (|x| <= 10 half steps), additions, the division
    rel = (2 * (4 + 10) + E + 1) * U
    assert ((w.double() - want_w).abs() <= rel * want_w).all()
    part = want_w * dw.double()
    mean, size = part.sum(1, keepdim=True), part.abs().sum(1, keepdim=True)
    grad = torch.zeros_like(x).scatter_add_(1, at.clamp_min(0), dw.double() * (at >= 0))
    want = p * (grad - mean)
    # p and the weights within that, and the mean's products and additions: k + 1 half steps of its magnitude; the difference, the product and
    # the reciprocal one each; a rounding to the type
    tol = p * ((2 * rel + (k + 5) * U) * (grad.abs() + size))
    small = 2.0 ** -25 if kind == "fp16" else 0.0
    assert ((d.double() - want).abs() <= tol + ref.HALF_STEP[kind] * (want.abs() + tol) + small).all()
    assert rows.sync() == 0
