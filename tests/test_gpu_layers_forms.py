"""The forms of a layer's kernels that the sizes of test_gpu_layers.py do not take: many rows at odd places, matrices whose rows start at different places,
wide and long rows in number, dropout of many 16-bit rows.  Tolerances: layer_reference.py."""
import pytest
import torch

import layer_reference as ref
from test_gpu_layers import (KINDS, LINES, TYPES, expected_dropout, f64, gen, layer_inputs, norm_inputs, rows, run_layer, run_norm,  # noqa: F401
                             strided, untouched_beside)

pytestmark = pytest.mark.gpu


def norm_both_ways(rows, T, D, kind, places, params="fp32", dx_wanted=True):  # noqa: F811
    """The norm and its gradient; places: (elements between rows, elements before the first one) of x, y, dy and dx."""
    x, gamma, beta, dy = norm_inputs(T, D, kind, params, 80)
    at_x, at_y, at_dy, at_dx = places
    X, Y = strided(x, *at_x), strided(torch.zeros_like(x), *at_y)
    got = run_norm(rows, X, gamma.cuda(), beta.cuda(), y=Y)
    want, off = ref.norm(f64(x), f64(gamma), f64(beta), 1e-5)
    for a, b, c, k in zip(got, want, off, (kind, "fp32", "fp32")):
        ref.within(f64(a), b, c, k)
    assert untouched_beside(Y, *at_y)
    mean, rstd = torch.from_numpy(want[1]).float(), torch.from_numpy(want[2]).float()
    DX = strided(torch.zeros_like(x), *at_dx) if dx_wanted else None
    dgamma, dbeta = torch.full((D,), 5.0, device="cuda"), torch.full((D,), 5.0, device="cuda")
    rows.layer_norm_grad(strided(dy, *at_dy), X, mean.cuda(), rstd.cuda(), gamma.cuda(), DX, dgamma, dbeta, rows.layer_norm_grad_work(T, D).fill_(0xFF))
    want, off = ref.norm_grad(f64(dy), f64(x), f64(mean), f64(rstd), f64(gamma), LINES)
    for a, b, c, k in zip((DX, dgamma, dbeta), want, off, (kind, "fp32", "fp32")):
        if a is not None:
            ref.within(f64(a), b, c, k)
    assert DX is None or untouched_beside(DX, *at_dx)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind,T,D,extra,shift", [
    ("bf16", 20011, 33, 0, 0), ("fp16", 4001, 501, 0, 0), ("fp16", 2001, 4001, 0, 0), ("fp32", 5003, 1001, 0, 0), ("bf16", 2500, 2047, 0, 0), ("fp16", 6001, 33, 2, 3),
    ("bf16", 4001, 500, 12, 1), ("fp16", 4001, 500, 12, 2), ("fp32", 3001, 500, 4, 2), ("bf16", 5001, 500, 2, 0), ("fp32", 20011, 17, 0, 1)])
def test_norm_of_many_rows_at_odd_places(rows, kind, T, D, extra, shift):  # noqa: F811
    """More rows than there are teams: the next row is fetched, rings are filled again, a team's rows start at one place in a word."""
    norm_both_ways(rows, T, D, kind, [(extra, shift)] * 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("places", [((0, 0), (0, 1), (0, 0), (0, 0)), ((0, 0), (3, 0), (1, 2), (5, 3)), ((8, 0), (8, 0), (8, 0), (8, 1)), ((0, 0), (0, 0), (1, 0), (0, 0))])
def test_norm_of_matrices_that_start_differently(rows, kind, places):  # noqa: F811
    norm_both_ways(rows, 701, 332, kind, places)


@pytest.mark.parametrize("kind,T,D,extra,shift", [
    ("bf16", 331, 12289, 0, 0), ("fp16", 331, 16384, 0, 0), ("fp16", 331, 12290, 6, 2), ("fp32", 331, 6145, 0, 0), ("fp32", 331, 8192, 0, 0), ("fp32", 331, 7000, 4, 3),
    ("bf16", 331, 20000, 0, 0), ("fp16", 331, 24001, 0, 0), ("fp32", 331, 9000, 0, 0), ("fp32", 331, 12001, 0, 0)])
def test_norm_of_wide_rows_in_number(rows, kind, T, D, extra, shift):  # noqa: F811
    """A block of up to 1024 threads has several rows one after the other; the forward kernel's widest rows."""
    norm_both_ways(rows, T, D, kind, [(extra, shift)] * 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,extra,shift", [(37, 3, 0), (300, 0, 0), (501, 0, 1), (1001, 7, 2)])
@pytest.mark.parametrize("which", ["gamma", "beta"])
def test_norm_with_one_parameter(rows, kind, D, extra, shift, which):  # noqa: F811
    """A weight without a bias, and a bias without a weight."""
    x, gamma, beta, _ = norm_inputs(70, D, kind, "fp32", 81)
    gamma, beta = (gamma, None) if which == "gamma" else (None, beta)
    on = [None if p is None else p.cuda() for p in (gamma, beta)]
    for other in (0, 1):
        got = run_norm(rows, strided(x, extra, shift), *on, y=strided(torch.zeros_like(x), extra, shift + other))
        want, off = ref.norm(f64(x), None if gamma is None else f64(gamma), None if beta is None else f64(beta), 1e-5)
        for a, b, c, k in zip(got, want, off, (kind, "fp32", "fp32")):
            ref.within(f64(a), b, c, k)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind,T,D", [("bf16", 700, 33000), ("fp16", 601, 25001), ("fp32", 601, 12801)])
@pytest.mark.parametrize("dx_wanted", [True, False], ids=["all", "sums only"])
def test_norm_of_long_rows_in_number(rows, kind, T, D, dx_wanted):  # noqa: F811
    norm_both_ways(rows, T, D, kind, [(0, 0)] * 4, dx_wanted=dx_wanted)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D,extra", [(2047, 40, 0), (2048, 40, 0), (2049, 40, 0), (4101, 64, 0), (2049, 44, 4), (2051, 3, 5), (2049, 2056, 0), (30001, 8, 0), (259, 4096, 0), (4101, 264, 0), (70001, 20, 4),
                                     (9001, 249, 0), (5003, 501, 0)])
def test_dropout_of_many_rows(rows, kind, T, D, extra):  # noqa: F811
    x, res = torch.randn(T, D, generator=gen(90, T, D)).to(TYPES[kind]), torch.randn(T, D, generator=gen(91, T, D)).to(TYPES[kind])
    for residual in (res, None):
        y = strided(torch.zeros_like(x), extra)
        rows.dropout(strided(x, extra), y, 0.3, 12, 5, residual=None if residual is None else strided(res, extra))
        assert torch.equal(y.cpu(), expected_dropout(x, residual, 0.3, 12, 5)) and untouched_beside(y, extra)
    assert rows.sync() == 0


# ---- the expert layer's ends, and calls side by side -------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D,H,E,k", [(2, 65536, 24, 2, 1), (2, 65535, 9, 2, 1), (2, 24, 65536, 2, 2), (2, 9, 65535, 2, 2), (64, 16, 8, 1024, 32), (64, 24, 40, 1, 1),
                                       (64, 200, 72, 2, 2), (64, 72, 200, 3, 2)])
def test_expert_layer_at_the_ends_of_its_sizes(rows, kind, T, D, H, E, k):  # noqa: F811
    """The widest rows, the most experts and choices, experts with more slots than are multiplied at once."""
    for gated, chosen in ((True, False), (False, True)):
        x, router, up, down = layer_inputs(T, D, H, E, k, kind, gated, 96)
        w, ids = torch.full((T, k), 5.0, device="cuda"), torch.full((T, k), 99, dtype=torch.int32, device="cuda")
        y = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, gated, chosen)
        want_w, want_ids, off_w = ref.choose(f64(x), f64(router), k, chosen)
        assert (ids.cpu().numpy() == want_ids).all()
        want, off = ref.experts(f64(x), f64(up), f64(down), want_w, want_ids, kind, gated, off_w)
        ref.within(f64(y), want, off, kind)
    assert rows.sync() == 0


def test_calls_side_by_side(rows):  # noqa: F811
    """Two streams with handles and scratch of their own, whose calls are in the GPU at the same time: each has the results that it has alone."""
    from paper_2311_09445_b200 import RowLayers
    T, D, H, E, k = 48, 2048, 1000, 24, 4
    sides = []
    for i, kind in enumerate(("bf16", "fp16")):
        x, router, up, down = (t.cuda() for t in layer_inputs(T, D, H, E, k, kind, True, 97 + i))
        w, ids, y = torch.zeros(T, k, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda"), torch.zeros_like(x)
        norm, mean, rstd = torch.zeros_like(x), torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
        dx, dg, db = torch.zeros_like(x), torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
        stream = torch.cuda.Stream()
        r = RowLayers(stream=stream)
        work, sums = r.expert_layer_work(T, D, H, E, k), r.layer_norm_grad_work(T, D)

        def step(r=r, x=x, router=router, up=up, down=down, y=y, w=w, ids=ids, work=work, norm=norm, mean=mean, rstd=rstd, dx=dx, dg=dg, db=db, sums=sums):
            r.layer_norm(x, norm, None, None, 1e-5, mean, rstd)
            r.expert_layer(norm, router, up, down, y, w, ids, work)
            r.layer_norm_grad(y, x, mean, rstd, None, dx, dg, db, sums)

        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        outs = (norm, mean, rstd, y, w, ids, dx, dg, db)
        sides.append((r, stream, step, outs, [t.clone() for t in outs]))
    for _ in range(30):
        for _, _, step, _, _ in sides:
            step()
    torch.cuda.synchronize()
    graphs = []
    for r, stream, step, outs, alone in sides:
        for a, b in zip(outs, alone):
            assert torch.equal(a, b)
            a.zero_()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                step()
        graphs.append(graph)
    for _ in range(5):
        for graph, (_, stream, _, _, _) in zip(graphs, sides):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for r, _, _, outs, alone in sides:
        for a, b in zip(outs, alone):
            assert torch.equal(a, b)
        assert r.sync() == 0
    graphs.clear()
    for r, *_ in sides:
        r.close()
