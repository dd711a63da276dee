"""A layer's operators on the GPU against their definitions in 64 bits (layer_reference.py, where the tolerances are counted)."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
KINDS = list(TYPES)
BAD_INDEX, BAD_SCORE = 1, 64
LINES = 296


@pytest.fixture(scope="module")
def rows():
    from paper_2311_09445_b200 import RowLayers
    r = RowLayers()
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


def untouched_beside(view, extra, shift=0):
    T, D = view.shape
    around = view._base.clone()
    around[shift:].view(T, D + extra)[:, :D] = 7
    return bool((around == 7).all())


# ---- layer norm ------------------------------------------------------------------------------------------------------

def norm_inputs(T, D, kind, params, seed=1):
    g = gen(seed, T, D)
    x = (torch.randn(T, D, generator=g) * (0.5 + torch.rand(T, 1, generator=g)) + 0.4).to(TYPES[kind])
    gamma = (1 + 0.3 * torch.randn(D, generator=g)).to(TYPES[params])
    beta = torch.randn(D, generator=g).to(TYPES[params])
    return x, gamma, beta, torch.randn(T, D, generator=g).to(TYPES[kind])


def run_norm(rows, x, gamma, beta, eps=1e-5, y=None):
    T = x.shape[0]
    y = torch.full_like(x, 3) if y is None else y
    mean, rstd = torch.full((T,), 9.0, device="cuda"), torch.full((T,), 9.0, device="cuda")
    rows.layer_norm(x, y, gamma, beta, eps, mean, rstd)
    return y, mean, rstd


NORM_SIZES = [(1, 1), (2, 2), (3, 7), (5, 17), (257, 33), (70, 128), (9, 129), (33, 500), (6, 1000), (11, 1024), (5, 1025), (7, 2046), (4, 4096),
              (3, 5000), (2, 12289), (3, 16384), (2, 33000), (1, 65536)]


MANY_ROWS = [(1000, 40), (700, 600), (301, 2048), (20011, 512), (40001, 256), (3001, 1000)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D", NORM_SIZES + MANY_ROWS)
def test_norm(rows, kind, T, D):
    for params in {kind, "fp32"}:
        x, gamma, beta, _ = norm_inputs(T, D, kind, params)
        got = run_norm(rows, x.cuda(), gamma.cuda(), beta.cuda())
        want, off = ref.norm(f64(x), f64(gamma), f64(beta), 1e-5)
        for a, b, c, k in zip(got, want, off, (kind, "fp32", "fp32")):
            ref.within(f64(a), b, c, k)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D", NORM_SIZES + MANY_ROWS)
def test_norm_grad(rows, kind, T, D):
    for params in {kind, "fp32"}:
        x, gamma, _, dy = norm_inputs(T, D, kind, params, 2)
        (_, mean, rstd), _ = ref.norm(f64(x), None, None, 1e-5)
        mean, rstd = torch.from_numpy(mean).float(), torch.from_numpy(rstd).float()
        dx, dgamma, dbeta = torch.full((T, D), 3.0, dtype=x.dtype, device="cuda"), torch.full((D,), 5.0, device="cuda"), torch.full((D,), 5.0, device="cuda")
        work = rows.layer_norm_grad_work(T, D).fill_(0xFF)               # (its contents do not matter)
        rows.layer_norm_grad(dy.cuda(), x.cuda(), mean.cuda(), rstd.cuda(), gamma.cuda(), dx, dgamma, dbeta, work)
        want, off = ref.norm_grad(f64(dy), f64(x), f64(mean), f64(rstd), f64(gamma), LINES)
        for a, b, c, k in zip((dx, dgamma, dbeta), want, off, (kind, "fp32", "fp32")):
            ref.within(f64(a), b, c, k)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind,D,extra,shift", [("fp32", 60, 3, 1), ("bf16", 128, 1, 1), ("fp16", 200, 8, 2), ("bf16", 64, 4, 4), ("fp32", 2000, 4, 4),
                                                ("fp16", 3001, 15, 0), ("bf16", 999, 9, 8)])
def test_norm_rows_apart(rows, kind, D, extra, shift):
    """Rows at other distances and places: the same numbers, and nothing beside the rows is written."""
    x, gamma, beta, dy = norm_inputs(37, D, kind, kind, 3)
    dense = run_norm(rows, x.cuda(), gamma.cuda(), beta.cuda())
    y = strided(torch.zeros_like(x), extra, shift)
    got = run_norm(rows, strided(x, extra, shift), gamma.cuda(), beta.cuda(), y=y)
    want, off = ref.norm(f64(x), f64(gamma), f64(beta), 1e-5)
    for a, b, c, k in zip(got, want, off, (kind, "fp32", "fp32")):
        ref.within(f64(a), b, c, k)
    assert untouched_beside(y, extra, shift)
    dx, dgamma, dbeta = strided(torch.zeros_like(x), extra, shift), torch.zeros(D, device="cuda"), torch.zeros(D, device="cuda")
    rows.layer_norm_grad(strided(dy, extra, shift), strided(x, extra, shift), dense[1], dense[2], gamma.cuda(), dx, dgamma, dbeta,
                         rows.layer_norm_grad_work(37, D))
    want, off = ref.norm_grad(f64(dy), f64(x), f64(dense[1]), f64(dense[2]), f64(gamma), LINES)
    for a, b, c, k in zip((dx, dgamma, dbeta), want, off, (kind, "fp32", "fp32")):
        ref.within(f64(a), b, c, k)
    assert untouched_beside(dx, extra, shift)
    assert rows.sync() == 0


def test_norm_outputs_that_are_not_wanted(rows):
    x, gamma, beta, dy = (t.cuda() for t in norm_inputs(50, 300, "bf16", "fp32", 4))
    y, mean, rstd = run_norm(rows, x, gamma, beta)
    alone = torch.zeros_like(x)
    rows.layer_norm(x, alone, gamma, beta, 1e-5)
    assert torch.equal(alone, y)
    plain = torch.zeros_like(x)
    rows.layer_norm(x, plain, None, None, 1e-5)
    ones = run_norm(rows, x, torch.ones(300, device="cuda"), torch.zeros(300, device="cuda"))[0]
    assert torch.equal(plain, ones)
    work = rows.layer_norm_grad_work(50, 300)
    dx, dg, db = torch.zeros_like(x), torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    rows.layer_norm_grad(dy, x, mean, rstd, gamma, dx, dg, db, work)
    for which in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        outs = [torch.zeros_like(t) if want else None for t, want in zip((dx, dg, db), which)]
        rows.layer_norm_grad(dy, x, mean, rstd, gamma, *outs, work if any(which[1:]) else None)
        for a, b in zip(outs, (dx, dg, db)):
            assert a is None or torch.equal(a, b)
    assert rows.sync() == 0


def test_norm_of_no_rows(rows):
    x = torch.zeros(0, 40, device="cuda")
    run_norm(rows, x, None, None)
    dg, db = torch.full((40,), 5.0, device="cuda"), torch.full((40,), 5.0, device="cuda")
    rows.layer_norm_grad(x, x, x[:, 0].contiguous(), x[:, 0].contiguous(), None, torch.zeros_like(x), dg, db, rows.layer_norm_grad_work(0, 40))
    assert (dg == 0).all() and (db == 0).all() and rows.sync() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [5, 500, 3000])
def test_norm_special_rows(rows, kind, D):
    """A constant row, rows with infinity or NaN, the type's largest values: only their own results are touched."""
    x, gamma, beta, dy = norm_inputs(9, D, kind, "fp32", 5)
    plain = run_norm(rows, x.cuda(), gamma.cuda(), beta.cuda())[0]
    x[1] = 2.5
    x[3, D // 2] = math.inf
    x[5, 0] = math.nan
    x[7] = 0
    y, mean, rstd = run_norm(rows, x.cuda(), gamma.cuda(), beta.cuda())
    for t in (0, 2, 4, 6, 8):
        assert torch.equal(y[t], plain[t])
    for t in (1, 7):
        ref.within(f64(y[t]), f64(beta), 0.0, kind)                # (an exactly constant row: its mean is exact, its differences zero)
        assert float(rstd[t]) == pytest.approx(1e-5 ** -0.5, rel=1e-6)
    assert y[3].isnan().all() and y[5].isnan().all()


# ---- dropout ---------------------------------------------------------------------------------------------------------

def expected_dropout(x, residual, p, seed, call):
    mask, scale = ref.kept(*x.shape, p, seed, call)
    y = torch.where(torch.from_numpy(mask), x.float() * np.float32(scale), torch.zeros(()))
    return (y + (residual.float() if residual is not None else 0.0)).to(x.dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D", [(1, 1), (3, 7), (5, 8), (256, 17), (9, 500), (4, 2047), (5, 2046), (3, 4096), (2, 20000), (700, 64)])
def test_dropout(rows, kind, T, D):
    """Every bit: the mask by the generator's definition, a product and a sum in binary32, one rounding."""
    x, res = torch.randn(T, D, generator=gen(6, T, D)).to(TYPES[kind]), torch.randn(T, D, generator=gen(7, T, D)).to(TYPES[kind])
    for p, seed, call in ((0.1, 3, 0), (0.5, 1 << 40, 7), (0.93, (1 << 64) - 1, (1 << 64) - 5), (0.0, 5, 1), (1.0, 5, 1)):
        y = torch.full_like(x, 3).cuda()
        rows.dropout(x.cuda(), y, p, seed, call, residual=res.cuda())
        assert torch.equal(y.cpu(), expected_dropout(x, res, p, seed, call)), (p, seed, call)
        rows.dropout_grad(x.cuda(), y, p, seed, call)
        assert torch.equal(y.cpu(), expected_dropout(x, None, p, seed, call)), (p, seed, call)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind,D,extra,shift", [("fp32", 60, 3, 1), ("bf16", 128, 1, 1), ("fp16", 200, 8, 2), ("bf16", 61, 3, 4), ("fp32", 2000, 4, 4)])
def test_dropout_rows_apart_and_in_place(rows, kind, D, extra, shift):
    x, res = torch.randn(37, D, generator=gen(8, D)).to(TYPES[kind]), torch.randn(37, D, generator=gen(9, D)).to(TYPES[kind])
    want = expected_dropout(x, res, 0.3, 11, 2)
    y = strided(torch.zeros_like(x), extra, shift)
    rows.dropout(strided(x, extra, shift), y, 0.3, 11, 2, residual=strided(res, extra, shift))
    assert torch.equal(y.cpu(), want) and untouched_beside(y, extra, shift)
    a = strided(x, extra, shift)
    rows.dropout(a, a, 0.3, 11, 2, residual=res.cuda())
    assert torch.equal(a.cpu(), want) and untouched_beside(a, extra, shift)
    b = strided(res, extra, shift)
    rows.dropout(x.cuda(), b, 0.3, 11, 2, residual=b)
    assert torch.equal(b.cpu(), want) and untouched_beside(b, extra, shift)


def test_dropped_elements_do_not_matter(rows):
    x = torch.randn(40, 100, generator=gen(10))
    mask = torch.from_numpy(ref.kept(40, 100, 0.4, 9, 9)[0])
    y = torch.zeros(40, 100, device="cuda")
    rows.dropout(torch.where(mask, x, torch.full((), math.nan)).cuda(), y, 0.4, 9, 9)
    assert torch.equal(y.cpu(), expected_dropout(x, None, 0.4, 9, 9))


def test_dropout_counts_calls_in_a_captured_graph(rows):
    """A graph that counts its calls in device memory draws a new mask in each replay."""
    from paper_2311_09445_b200 import RowLayers
    x = torch.randn(30, 72, generator=gen(11))
    calls, y, d = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(30, 72, device="cuda"), x.cuda()
    stream = torch.cuda.Stream()
    r = RowLayers(stream=stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        r.dropout(d, y, 0.25, 77, 5, calls=calls)
        calls.add_(1)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.cpu(), expected_dropout(x, None, 0.25, 77, 5 + i))
    del graph
    r.close()


# ---- the expert layer for a few rows ---------------------------------------------------------------------------------

def layer_inputs(T, D, H, E, k, kind, gated, seed=20):
    g = gen(seed, T, D, H, E)
    t = TYPES[kind]
    x = torch.randn(T, D, generator=g).to(t)
    router = (1.5 * D ** -0.5 * torch.randn(E, D, generator=g)).to(t)
    up = (D ** -0.5 * torch.randn(E, (2 if gated else 1) * H, D, generator=g)).to(t)
    down = (H ** -0.5 * torch.randn(E, D, H, generator=g)).to(t)
    return x, router, up, down


def run_layer(rows, x, router, up, down, w, ids, gated, chosen, work=None, y=None):
    T, D = x.shape
    E, H, k = down.shape[0], down.shape[2], ids.shape[1]
    work = rows.expert_layer_work(T, D, H, E, k) if work is None else work
    y = torch.full_like(x, 3) if y is None else y
    rows.expert_layer(x, router, up, down, y, w, ids, work, gated=gated, over_chosen=chosen)
    return y


LAYERS = [(1, 16, 16, 2, 1), (1, 1, 1, 1, 1), (3, 17, 5, 3, 2), (2, 64, 64, 8, 2), (9, 500, 333, 16, 4), (64, 128, 96, 4, 2), (5, 256, 40, 130, 8),
          (33, 72, 200, 5, 5), (64, 65, 63, 2, 1), (17, 1024, 128, 6, 3), (8, 40, 1000, 4, 2), (64, 32, 32, 40, 32), (1, 2048, 512, 16, 8),
          (12, 66, 34, 7, 2), (40, 520, 264, 3, 2), (6, 256, 130, 5, 2), (6, 250, 128, 5, 2), (64, 512, 77, 3, 2)]


# enough pieces of 128 weight rows for every SM
LARGE_LAYERS = [(33, 1024, 520, 24, 3), (64, 1088, 648, 16, 16), (5, 2048, 1000, 40, 4), (1, 4096, 1024, 12, 8)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D,H,E,k", LAYERS + LARGE_LAYERS)
def test_expert_layer(rows, kind, T, D, H, E, k):
    for gated, chosen in ((True, True), (False, False)):
        x, router, up, down = layer_inputs(T, D, H, E, k, kind, gated)
        w, ids = torch.full((T, k), 5.0, device="cuda"), torch.full((T, k), 99, dtype=torch.int32, device="cuda")
        y = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, gated, chosen)
        want_w, want_ids, off_w = ref.choose(f64(x), f64(router), k, chosen)
        assert (ids.cpu().numpy() == want_ids).all()
        np.testing.assert_allclose(f64(w), want_w, rtol=off_w, atol=0)
        want, off = ref.experts(f64(x), f64(up), f64(down), want_w, want_ids, kind, gated, off_w)
        ref.within(f64(y), want, off, kind)
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,D,H,E,k", [(1, 64, 32, 8, 2), (20, 100, 60, 6, 3), (64, 256, 128, 8, 4), (64, 64, 64, 1, 1), (64, 1024, 512, 16, 4)])
def test_expert_layer_with_given_choices(rows, kind, T, D, H, E, k):
    """Slots without an expert, rows without any, a row that names an expert twice, all rows at one expert."""
    x, _, up, down = layer_inputs(T, D, H, E, k, kind, True, 21)
    g = gen(22, T, E)
    ids = torch.randint(0, E, (T, k), generator=g, dtype=torch.int32)
    w = torch.rand(T, k, generator=g) + 0.1
    for case in ("random", "barred", "none", "one"):
        if case == "barred":
            ids[torch.rand(T, k, generator=g) < 0.5] = -1
            ids[T // 2] = -1
        elif case == "none":
            ids = torch.full_like(ids, -1)
        elif case == "one":
            ids = torch.full_like(ids, E - 1)
        wd, idd = w.cuda(), ids.cuda()
        y = run_layer(rows, x.cuda(), None, up.cuda(), down.cuda(), wd, idd, True, True)
        assert torch.equal(idd.cpu(), ids) and torch.equal(wd.cpu(), w)
        want, off = ref.experts(f64(x), f64(up), f64(down), f64(w), ids.numpy(), kind, True)
        ref.within(f64(y), want, off, kind)
    assert rows.sync() == 0


def test_expert_layer_reports_bad_choices(rows):
    x, _, up, down = layer_inputs(4, 32, 16, 3, 2, "fp32", True, 23)
    ids = torch.tensor([[0, 3], [-2, 1], [1 << 30, -1], [2, 0]], dtype=torch.int32)
    w = torch.ones(4, 2)
    y = run_layer(rows, x.cuda(), None, up.cuda(), down.cuda(), w.cuda(), ids.cuda(), True, True)
    assert rows.sync() == BAD_INDEX
    want, off = ref.experts(f64(x), f64(up), f64(down), f64(w), ids.numpy(), "fp32", True)
    ref.within(f64(y), want, off, "fp32")


@pytest.mark.parametrize("kind", KINDS)
def test_expert_layer_rows_apart_at_odd_places(rows, kind):
    for D, H, extra, shift in ((60, 36, 3, 1), (64, 64, 4, 4), (33, 31, 0, 1), (128, 40, 8, 8)):
        x, router, up, down = layer_inputs(7, D, H, 5, 2, kind, True, 24)
        w, ids = torch.zeros(7, 2, device="cuda"), torch.zeros(7, 2, dtype=torch.int32, device="cuda")

        def odd(t):
            store = torch.zeros(t.numel() + shift, dtype=t.dtype, device="cuda")
            store[shift:] = t.flatten().cuda()
            return store[shift:].view(t.shape)

        y = strided(torch.zeros_like(x), extra, shift)
        run_layer(rows, strided(x, extra, shift), odd(router), odd(up), odd(down), w, ids, True, True, y=y)
        want_w, want_ids, off_w = ref.choose(f64(x), f64(router), 2, True)
        assert (ids.cpu().numpy() == want_ids).all()
        want, off = ref.experts(f64(x), f64(up), f64(down), want_w, want_ids, kind, True, off_w)
        ref.within(f64(y), want, off, kind)
        assert untouched_beside(y, extra, shift)


def test_expert_layer_bad_logits(rows):
    """NaN or infinity in a router's row bars that expert; a row of x that is not finite is its own affair."""
    x, router, up, down = layer_inputs(6, 48, 32, 5, 2, "fp32", True, 25)
    router[3, 7] = math.nan
    w, ids = torch.zeros(6, 2, device="cuda"), torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    y = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, True, False)
    assert rows.sync() == BAD_SCORE and not (ids == 3).any()
    want_w, want_ids, off_w = ref.choose(f64(x), f64(router), 2, False)
    assert (ids.cpu().numpy() == want_ids).all()
    want, off = ref.experts(f64(x), f64(up), f64(down), want_w, want_ids, "fp32", True, off_w)
    ref.within(f64(y), want, off, "fp32")
    router[3, 7] = 0.1
    y = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, True, False)
    broken = x.clone()
    broken[2, 5] = math.nan
    z = run_layer(rows, broken.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, True, False)
    assert rows.sync() == BAD_SCORE
    keep = [0, 1, 3, 4, 5]
    assert torch.equal(y[keep], z[keep]) and (z[2] == 0).all() and (ids[2] == -1).all()


def test_expert_layer_nan_weights_of_other_experts_do_not_matter(rows):
    x, router, up, down = layer_inputs(3, 64, 32, 9, 2, "bf16", True, 26)
    w, ids = torch.zeros(3, 2, device="cuda"), torch.zeros(3, 2, dtype=torch.int32, device="cuda")
    y = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, True, True)
    rest = [e for e in range(9) if e not in ids.flatten().tolist()]
    up[rest], down[rest] = math.nan, math.nan
    z = run_layer(rows, x.cuda(), router.cuda(), up.cuda(), down.cuda(), w, ids, True, True)
    assert torch.equal(y, z)


def test_expert_layer_one_workspace_for_many_sizes(rows):
    """A workspace serves call after call, of any sizes it has room for."""
    work = rows.expert_layer_work(64, 520, 264, 64, 8)
    for i, (T, D, H, E, k) in enumerate([(64, 520, 264, 64, 8), (1, 64, 32, 4, 2), (33, 500, 100, 7, 3), (2, 520, 264, 64, 8), (64, 64, 264, 64, 1)] * 2):
        x, router, up, down = (t.cuda() for t in layer_inputs(T, D, H, E, k, "bf16", True, 27))
        w, ids = torch.zeros(T, k, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda")
        fresh = run_layer(rows, x, router, up, down, w, ids, True, True)
        assert torch.equal(run_layer(rows, x, router, up, down, w, ids, True, True, work=work), fresh), i
    assert rows.sync() == 0


def test_expert_layer_captured(rows):
    """Replays with new inputs, and two graphs with workspaces of their own side by side."""
    from paper_2311_09445_b200 import RowLayers
    x, router, up, down = (t.cuda() for t in layer_inputs(5, 256, 128, 16, 4, "bf16", True, 28))
    runs = []
    for i in range(2):
        stream = torch.cuda.Stream()
        r = RowLayers(stream=stream)
        a, y = x.clone(), torch.zeros_like(x)
        w, ids = torch.zeros(5, 4, device="cuda"), torch.zeros(5, 4, dtype=torch.int32, device="cuda")
        work = r.expert_layer_work(5, 256, 128, 16, 4)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(4):
                r.expert_layer(a, router, up, down, y, w, ids, work)
        runs.append((r, stream, graph, a, y, work))
    for trial in range(3):
        inputs = [torch.randn(5, 256, generator=gen(29, trial, i)).bfloat16().cuda() for i in range(2)]
        for (_, stream, graph, a, _, _), new in zip(runs, inputs):
            a.copy_(new)
        torch.cuda.synchronize()
        for _, stream, graph, _, _, _ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (_, _, _, _, y, _), new in zip(runs, inputs):
            w, ids = torch.zeros(5, 4, device="cuda"), torch.zeros(5, 4, dtype=torch.int32, device="cuda")
            assert torch.equal(y, run_layer(rows, new, router, up, down, w, ids, True, True))
    for r, _, graph, *_ in runs:
        del graph
    rs = [r for r, *_ in runs]
    runs.clear()
    for r in rs:
        assert r.sync() == 0
        r.close()


# ---- together --------------------------------------------------------------------------------------------------------

def test_layer_trained_and_acted_with(rows):
    """x + dropout(experts(norm(x))) through the row operators with every gradient, against differences; and the same layer as a policy
    runs it, in one call."""
    T, D, H, E, k, p, seed = 24, 32, 24, 4, 2, 0.2, 5
    g = gen(40)
    d64 = dict(generator=g, dtype=torch.float64)
    x0, gamma0, beta0 = torch.randn(T, D, **d64), 1 + 0.2 * torch.randn(D, **d64), 0.1 * torch.randn(D, **d64)
    up0, down0, router0 = torch.randn(E, 2 * H, D, **d64) * D ** -0.5, torch.randn(E, D, H, **d64) * H ** -0.5, torch.randn(E, D, **d64) * D ** -0.5
    dout0 = torch.randn(T, D, **d64)
    x, gamma, beta, up, down, router, dout = (t.float().cuda() for t in (x0, gamma0, beta0, up0, down0, router0, dout0))
    zeros = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    i32 = torch.int32
    n, mean, rstd = zeros(T, D), zeros(T), zeros(T)
    rows.layer_norm(x, n, gamma, beta, 1e-5, mean, rstd)
    logits = n @ router.t()
    w, ids, offsets, order, place = zeros(T, k), zeros(T, k, dtype=i32), zeros(E + 1, dtype=i32), zeros(T * k, dtype=i32), zeros(T, k, dtype=i32)
    xs, y, out = zeros(T * k, D), zeros(T, D), zeros(T, D)
    rows.route(logits, w, ids, over_chosen=True)
    rows.sort(ids, E, offsets, order, place)
    rows.dispatch(n, place, xs)
    # the experts' products of a training batch: the caller's (here with torch's own gradient)
    cuts = offsets.tolist()
    leaf = xs.detach().requires_grad_()
    zs = []
    for e in range(E):
        both = leaf[cuts[e]:cuts[e + 1]] @ up[e].t()
        zs.append((torch.nn.functional.silu(both[:, :H]) * both[:, H:]) @ down[e].t())
    z = torch.cat(zs)
    rows.combine(z.detach().contiguous(), place, w, y)
    rows.dropout(y, out, p, seed, 1, residual=x)
    # the acting form gives the same layer
    act_y, act_w, act_ids = zeros(T, D), zeros(T, k), zeros(T, k, dtype=i32)
    rows.expert_layer(n, router, up, down, act_y, act_w, act_ids, rows.expert_layer_work(T, D, H, E, k))
    assert torch.equal(act_ids, ids) and torch.allclose(act_w, w, rtol=1e-5) and torch.allclose(act_y, y, rtol=1e-3, atol=1e-4)
    # backward
    dy, dz, dw, dxs, dn, dlogits, dx = zeros(T, D), zeros(T * k, D), zeros(T, k), zeros(T * k, D), zeros(T, D), zeros(T, E), zeros(T, D)
    dgamma, dbeta = zeros(D), zeros(D)
    rows.dropout_grad(dout, dy, p, seed, 1)
    rows.combine_grad(dy, z.detach().contiguous(), place, w, dz, dw)
    dxs = torch.autograd.grad(z, leaf, dz)[0].contiguous()
    rows.dispatch_grad(dxs, place, dn)
    rows.route_grad(logits, w, ids, dw, dlogits, over_chosen=True)
    dn += dlogits @ router
    rows.layer_norm_grad(dn, x, mean, rstd, gamma, dx, dgamma, dbeta, rows.layer_norm_grad_work(T, D))
    dx += dout
    assert rows.sync() == 0
    mask, scale = ref.kept(T, D, p, seed, 1)
    mask = torch.from_numpy(mask)
    chosen = ids.cpu().long()

    def loss(x, gamma, beta):
        n = torch.nn.functional.layer_norm(x, (D,), gamma, beta, 1e-5)
        l = (n @ router0.t()).gather(1, chosen)
        w = torch.softmax(l, 1)
        y = 0
        for j in range(k):
            both = torch.einsum("trd,td->tr", up0[chosen[:, j]], n)
            y = y + w[:, j:j + 1] * torch.einsum("tdh,th->td", down0[chosen[:, j]], torch.nn.functional.silu(both[:, :H]) * both[:, H:])
        return float(((x + torch.where(mask, y * scale, torch.zeros((), dtype=y.dtype))) * dout0).sum())

    for name, at, grad in (("x", 0, dx), ("gamma", 1, dgamma), ("beta", 2, dbeta)):
        for trial in range(3):
            args = [x0, gamma0, beta0]
            v = torch.randn(args[at].shape, generator=gen(41, trial), dtype=torch.float64)
            h = 1e-5
            ends = []
            for sign in (1, -1):
                moved = list(args)
                moved[at] = args[at] + sign * h * v
                ends.append(loss(*moved))
            slope = (ends[0] - ends[1]) / (2 * h)
            mine = float((grad.double().cpu() * v).sum())
            # binary32 throughout: some 1e-6 of the magnitudes that are summed
            size = float((grad.double().cpu().abs() * v.abs()).sum())
            assert abs(slope - mine) <= 2e-5 * size + 1e-4 * abs(slope) + 1e-6, (name, slope, mine)
