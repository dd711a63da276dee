"""A layer's operators on the GPU where values are special: NaN and infinity in what is chosen, numbers that need all of binary32, constant rows."""
import math
import time

import numpy as np
import pytest
import torch

import layer_reference as ref
from test_gpu_layers import KINDS, TYPES, f64, gen, layer_inputs, norm_inputs, rows, run_layer, run_norm, strided  # noqa: F401

pytestmark = pytest.mark.gpu
INTERNAL = 16


def given(T, k, E, *seed):
    """Weights and experts of T rows; the last row asks for none."""
    g = gen(*seed)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    ids[-1] = -1
    return torch.rand(T, k, generator=g) + 0.5, ids


# ---- NaN and infinity in what the experts' products take -------------------------------------------------------------

# (the last ones in binary32: NaNs that arithmetic on a GPU gives, with a sign, with the lowest bit alone, and next to what rounds to them)
VALUES = {"nan": math.nan, "+inf": math.inf, "-inf": -math.inf, "all ones": 0x7FFFFFFF, "all ones and sign": 0xFFFFFFFF, "upper ones": 0x7FFFF000,
          "lowest bit": 0x7F800001, "below the upper ones": 0x7FFFEFFF}


def special(value, kind):
    if isinstance(value, float):
        return torch.tensor(value, dtype=TYPES[kind])
    return torch.from_numpy(np.array([value], np.uint32).view(np.float32))[0].to(TYPES[kind])


def not_finite(rows, kind, gated, where, D, H):  # noqa: F811
    T, E, k, row, e = 7, 5, 2, 2, 3
    x, _, up, down = layer_inputs(T, D, H, E, k, kind, gated, 50)
    w, ids = given(T, k, E, 51)
    ids[row, 0], ids[row, 1] = e, (e + 1) % E
    plain = run_layer(rows, x.cuda(), None, up.cuda(), down.cuda(), w.cuda(), ids.cuda(), gated, True).cpu()
    for name, value in VALUES.items():
        if kind != "fp32" and not isinstance(value, float):
            continue
        parts = {"x": x.clone(), "up": up.clone(), "down": down.clone()}
        at = {"x": (row, 5), "up": (e, H - 2, D - 1), "down": (e, D - 3, H - 1)}[where]
        parts[where][at] = special(value, kind)
        y = run_layer(rows, parts["x"].cuda(), None, parts["up"].cuda(), parts["down"].cuda(), w.cuda(), ids.cuda(), gated, True).cpu()
        with np.errstate(all="ignore"):
            want = ref.experts(f64(parts["x"]), f64(parts["up"]), f64(parts["down"]), f64(w), ids.numpy(), kind, gated)[0]
        touched = torch.zeros(T, D, dtype=torch.bool)
        meets = torch.arange(T) == row if where == "x" else (ids == e).any(1)
        touched[meets, D - 3 if where == "down" else slice(None)] = True
        assert touched.any() and torch.equal(y[~touched], plain[~touched]), name
        want = torch.from_numpy(want)
        if kind == "fp32":
            assert y[touched].isnan().all(), (name, y[touched])
        else:
            assert torch.equal(y[touched].isnan(), want[touched].isnan()), name
            infinite = touched & want.isinf()
            assert torch.equal(y[infinite].double(), want[infinite]), name
    assert rows.sync() == 0


@pytest.mark.parametrize("gated", [True, False], ids=["gated", "relu"])
@pytest.mark.parametrize("where", ["x", "up", "down"])
@pytest.mark.parametrize("D,H", [(48, 32), (47, 31)])
def test_expert_layer_in_binary32_keeps_what_is_not_finite(rows, gated, where, D, H):  # noqa: F811
    """A NaN or an infinity among the factors gives NaN where it is used, and no other bit changes."""
    not_finite(rows, "fp32", gated, where, D, H)


@pytest.mark.parametrize("kind", ["fp16", "bf16"])
@pytest.mark.parametrize("gated", [True, False], ids=["gated", "relu"])
@pytest.mark.parametrize("where", ["x", "up", "down"])
@pytest.mark.parametrize("D,H", [(48, 32), (47, 31)])
def test_expert_layer_in_16_bits_keeps_what_is_not_finite(rows, kind, gated, where, D, H):  # noqa: F811
    """It reaches the results as the definition has it, and no other bit changes."""
    not_finite(rows, kind, gated, where, D, H)


# ---- sums and products to the digits that binary32 has ----------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
def test_expert_layer_adds_blocks_rounding_to_nearest(rows, kind):  # noqa: F811
    """A large number and then, block after block of 64 numbers, three quarters of the last place of it.  A matrix instruction may cut off up to a place
    where its own sum has the large number; the sums of some blocks are added with half a place each.  So most of the terms are there."""
    T, D, H, E = 24, 2048, 520, 24                                # (enough pieces for every SM, so that one warp has a whole row)
    large = 2.0 ** (15 if kind == "fp16" else 24)
    place = large * 2.0 ** -23
    x, up, down = torch.ones(T, D), torch.zeros(E, H, D), torch.zeros(E, D, H)
    first = torch.arange(64) % 16 < 4                             # (the columns of one instruction's step, in each of a block's four parts)
    up[:, :2, :64][:, :, first] = large / 16
    up[:, 0, 64::64] = 0.75 * place
    down[:, :, 0], down[:, :, 1] = 1, -1
    ids = torch.arange(T, dtype=torch.int32).view(T, 1)
    t = TYPES[kind]
    y = f64(run_layer(rows, x.to(t).cuda(), None, up.to(t).cuda(), down.to(t).cuda(), torch.ones(T, 1).cuda(), ids.cuda(), False, True))
    blocks = D // 64 - 1
    want = 0.75 * place * blocks
    # a place for each of three blocks beside the large number, half a place for each block, and for h's own rounding and two of the second product
    limit = (3 + 0.5 * blocks + 1.5) * place
    assert limit < want
    ref.within(y, np.full_like(y, want), limit, kind)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,H,most,most16,times", [(8, 8, 255, 90, 2), (64, 2, 255, 31, 1), (512, 256, 255, 90, 2), (501, 123, 255, 90, 2)])
def test_expert_layer_on_whole_numbers(rows, kind, D, H, most, most16, times):  # noqa: F811
    """Whole numbers of up to 22 bits between the products (16 in binary16) whose differences are the results: every sum is exact in binary32."""
    g = gen(60, D, H)
    T, E, terms, pairs = 9, 4, min(D, 64 if H == 2 else 8), min(H // 2, 4)
    most = most16 if kind == "fp16" else most
    x, up, down = torch.zeros(T, D), torch.zeros(E, H, D), torch.zeros(E, D, H)
    at = torch.randperm(D, generator=g)[:terms]
    x[:, at] = torch.randint(0, most + 1, (T, terms), generator=g).float()
    x[:, at[0]] = 1
    for e in range(E):
        for i in (torch.randperm(H // 2, generator=g)[:pairs] * 2).tolist():
            up[e, i, at] = torch.randint(0, most - 2, (terms,), generator=g).float()
            up[e, i + 1] = up[e, i]
            up[e, i + 1, at[0]] += int(torch.randint(1, 4, (1,), generator=g))
            f = torch.randint(-times, times + 1, (D,), generator=g).float()
            down[e, :, i], down[e, :, i + 1] = -f, f
    ids = torch.randint(0, E, (T, 1), generator=g, dtype=torch.int32)
    t = TYPES[kind]
    y = run_layer(rows, x.to(t).cuda(), None, up.to(t).cuda(), down.to(t).cuda(), torch.ones(T, 1).cuda(), ids.cuda(), False, True)
    want = torch.stack([down[e].double() @ (up[e].double() @ row.double()) for row, e in zip(x, ids[:, 0].tolist())])
    assert want.abs().max() > 0 and torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("size", [1e-2, 1e-4, 1e-6])
def test_expert_layer_binary16_of_small_numbers_between_the_products(rows, size):  # noqa: F811
    """An h of the given size against large weights: it is kept to 2^-22 of it, give or take 2^-36."""
    T, D, H, E, k = 9, 64, 96, 4, 2
    g = gen(61)
    x = (0.05 * torch.randn(T, D, generator=g)).half()
    up = (size / 0.05 * D ** -0.5 * torch.randn(E, H, D, generator=g)).half()
    down = (min(0.3 / size, 2000.0) * torch.randn(E, D, H, generator=g)).half()
    w, ids = given(T, k, E, 62)
    y = f64(run_layer(rows, x.cuda(), None, up.cuda(), down.cuda(), w.cuda(), ids.cuda(), False, True))
    X, U, V = f64(x), f64(up), f64(down)
    want, off = np.zeros((T, D)), np.zeros((T, D))
    for t in range(T):
        for j in range(k):
            e = int(ids[t, j])
            if e < 0:
                continue
            h = np.maximum(U[e] @ X[t], 0)
            # additions: of a product's terms at most as many, each with two half steps where an instruction cuts off
            dh = 2 * D * ref.U * (np.abs(U[e]) @ np.abs(X[t])) + 2.0 ** -22 * h + 2.0 ** -36
            want[t] += float(w[t, j]) * (V[e] @ h)
            off[t] += float(w[t, j]) * (np.abs(V[e]) @ dh + 2 * (H + k + 4) * ref.U * (np.abs(V[e]) @ h))
    ref.within(y, want, off, "fp16")
    assert np.abs(want).mean() > 1e-4


# ---- constant rows of the norm -----------------------------------------------------------------------------------------

CONSTANT = [(41, 4096.0), (83, 1000.0), (83, 30000.0), (1000, 1000.0), (2047, 1000.0), (4099, 24.0)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,value", CONSTANT)
def test_norm_of_constant_rows(rows, kind, D, value):  # noqa: F811
    """Their sum is exact, so the mean is the value itself: the result is the bias, and 1 / sqrt(eps)."""
    _, gamma, beta, _ = norm_inputs(3, D, kind, "fp32", 70)
    for extra, shift, other in ((0, 0, 0), (3, 1, 1), (0, 0, 1)):          # (`other`: rows of y at another place than those of x)
        x = torch.full((3, D), value).to(TYPES[kind])
        y = strided(torch.zeros_like(x), extra + other, shift + other)
        got = run_norm(rows, strided(x, extra, shift), gamma.cuda(), beta.cuda(), y=y)
        assert torch.equal(got[1].cpu(), x[:, 0].float())
        np.testing.assert_allclose(f64(got[2]), 1e-5 ** -0.5, rtol=4 * ref.U)
        assert torch.equal(got[0].cpu(), beta.to(TYPES[kind]).expand(3, D))
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,value", CONSTANT)
def test_norm_grad_of_constant_rows(rows, kind, D, value):  # noqa: F811
    """A constant gradient of a constant row is taken out of it whole."""
    for extra, shift, other in ((0, 0, 0), (3, 1, 1), (0, 0, 1)):
        dy = torch.full((3, D), value).to(TYPES[kind])
        x = torch.full((3, D), 2.0).to(TYPES[kind])
        dx = strided(torch.ones_like(x), extra + other, shift + other)
        rows.layer_norm_grad(strided(dy, extra, shift), strided(x, extra, shift), torch.full((3,), 2.0, device="cuda"),
                             torch.full((3,), 300.0, device="cuda"), None, dx)
        assert (dx == 0).all()
    assert rows.sync() == 0


@pytest.mark.parametrize("kind", ["fp32", "bf16"])
@pytest.mark.parametrize("D,shift", [(48, 0), (333, 1)])
def test_norm_of_rows_beyond_the_range_of_binary32(rows, kind, D, shift):  # noqa: F811
    """Squared differences that are infinite give the bias, an infinite sum gives NaN; other rows are as they are alone."""
    x, gamma, beta, _ = norm_inputs(5, D, kind, "fp32", 71)
    for other in (0, 1):
        plain = run_norm(rows, strided(x, 0, shift), gamma.cuda(), beta.cuda(), y=strided(torch.zeros_like(x), 0, shift + other))
        far = x.clone()
        far[1] *= 1e25
        far[3] = 3e38
        got = run_norm(rows, strided(far, 0, shift), gamma.cuda(), beta.cuda(), y=strided(torch.zeros_like(x), 0, shift + other))
        assert float(got[2][1]) == 0 and torch.equal(got[0][1].cpu(), beta.to(TYPES[kind]))
        assert got[0][3].isnan().all()
        for t in (0, 2, 4):
            assert all(torch.equal(a[t], b[t]) for a, b in zip(got, plain))


# ---- a scratch that does not fit ---------------------------------------------------------------------------------------

def test_expert_layer_with_a_scratch_that_was_not_zero_ends(rows):  # noqa: F811
    """A count in it says that some first products are already in work, so nobody tells of them.  The call gives up after a limit, says so, and leaves the
    scratch fit for the next."""
    T, D, H, E, k = 64, 512, 256, 64, 4
    x, router, up, down = (t.cuda() for t in layer_inputs(T, D, H, E, k, "bf16", True, 95))
    w, ids, work = torch.zeros(T, k, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda"), rows.expert_layer_work(T, D, H, E, k)
    want = run_layer(rows, x, router, up, down, w, ids, True, True, work=work)
    assert rows.sync() == 0
    work[:4].view(torch.int32)[0] = 64
    start = time.monotonic()
    run_layer(rows, x, router, up, down, w, ids, True, True, work=work)
    assert rows.sync() == INTERNAL
    assert time.monotonic() - start < 20
    assert torch.equal(run_layer(rows, x, router, up, down, w, ids, True, True, work=work), want)
    assert rows.sync() == 0
