"""A layer's operators in 64 bits, plainly: what tests of the CUDA kernels compare with.  Shares no code with the library.

Each answers with how far a kernel's result may be off before it is rounded to the output's type: roundings counted, one half step of
binary32 (U) each, relative to what is rounded."""
import math

import numpy as np

from rows_reference import HALF_STEP

U = 2.0 ** -24


# additions one after the other in a sum over a row: 64 in a thread, 5 in a warp, 5 over the warps; and the scaling
ROW_CHAIN = 64 + 5 + 5 + 1


def norm(x, gamma, beta, eps):
    """(y, mean, rstd) and how far each may be off."""
    D = x.shape[1]
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    g = np.ones(D) if gamma is None else gamma
    b = np.zeros(D) if beta is None else beta
    n = (x - mean) * rstd
    y = n * g + b
    off_mean = ROW_CHAIN * U * np.abs(x).mean(1, keepdims=True)
    # the differences from a mean that is off by d: var + d^2; each difference and its square rounded; then 1 / sqrt: three roundings
    part = var / (var + eps)
    off_rstd = rstd * (0.5 * part * (ROW_CHAIN + 3) * U + 0.5 * off_mean ** 2 * rstd ** 2 + 3 * U + 0.5 * U)
    off = np.abs(g) * (off_mean * rstd + np.abs(x - mean) * off_rstd + 2 * U * np.abs(n)) + U * np.abs(y)
    return (y, mean[:, 0], rstd[:, 0]), (off, off_mean[:, 0], off_rstd[:, 0])


def norm_grad(dy, x, mean, rstd, gamma, lines):
    """(dx, dgamma, dbeta) and how far each may be off; lines: the partial sums over rows that there are at most."""
    T, D = x.shape
    g = np.ones(D) if gamma is None else gamma
    m, r = mean[:, None], rstd[:, None]
    n = (x - m) * r
    w = dy * g
    off_n = 2 * U * np.abs(n)
    a, b = w.mean(1, keepdims=True), (w * n).mean(1, keepdims=True)
    off_a = (ROW_CHAIN + 1) * U * np.abs(w).mean(1, keepdims=True)
    off_b = (ROW_CHAIN + 4) * U * np.abs(w * n).mean(1, keepdims=True)
    dx = r * (w - a - n * b)
    inner = 2 * U * np.abs(w) + off_a + U * np.abs(a) + np.abs(n) * off_b + 4 * U * np.abs(n * b)
    off_dx = np.abs(r) * (inner + 2 * U * (np.abs(w) + np.abs(a) + np.abs(n * b)))
    # rows a thread adds up one after the other (there are 148 blocks at least where there are as many rows), the teams of a block (15 at
    # most), the lines (32 sums of them, then 5 steps); two roundings of n
    chain = math.ceil(T / max(1, min(T, 148))) + 15 + math.ceil(lines / 32) + 5
    return (dx, (dy * n).sum(0), dy.sum(0)), (off_dx, (chain + 3) * U * np.abs(dy * n).sum(0), chain * U * np.abs(dy).sum(0))


def philox(counter, key):
    """Philox4x32-10 on arrays of whole numbers: counter [4, n], key (k0, k1) -> [4, n]."""
    c = [np.asarray(v, np.uint64) for v in counter]
    k0, k1 = int(key[0]), int(key[1])
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c)


def kept(T, D, p, seed, call):
    """The mask [T, D], and the factor of what is kept."""
    groups = -(-D // 8)
    t, g = np.meshgrid(np.arange(T), np.arange(groups), indexing="ij")
    call %= 1 << 64
    words = philox([g.ravel(), t.ravel(), np.full(T * groups, call & 0xFFFFFFFF), np.full(T * groups, call >> 32)],
                   (seed & 0xFFFFFFFF, seed >> 32)).T.reshape(T, groups, 4)
    bits = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], 3).reshape(T, groups * 8)[:, :D]
    below = math.floor(65536 * p + 0.5)
    return bits >= np.uint64(below), (65536 / (65536 - below) if below < 65536 else 0.0)


def choose(x, router, k, over_chosen):
    """(w, ids, how far w may be off, relative)."""
    from rows_reference import route
    with np.errstate(over="ignore", invalid="ignore"):
        logits = (x @ router.T).astype(np.float32).astype(np.float64)
    w, ids = route(logits, k, over_chosen)
    spread = max(1.0, float(np.nanmax(np.where(np.isfinite(logits), np.abs(logits), 0.0))) * 2)
    one = (2 + 1.2 * spread) * 2 * U + spread * U
    return w, ids, 2 * one + (router.shape[0] + 3) * U


def act(both, H, gated):
    if not gated:
        return np.maximum(both, 0.0)
    g = both[..., :H]
    return g / (1 + np.exp(-g)) * both[..., H:]


def experts(x, up, down, w, ids, kind, gated, off_w=0.0):
    """y and how far it may be off before its own rounding."""
    T, D = x.shape
    E, H = down.shape[0], down.shape[2]
    # additions in a row: an eighth of the terms one after the other and the joining of parts at most; a matrix instruction may cut off
    # where an addition rounds: two half steps each
    c1, c2 = 2 * (D / 8 + 32), 2 * (H / 8 + 32)
    split = {"fp32": 2.0 ** -22, "fp16": 2.0 ** -21, "bf16": 2.0 ** -17}[kind]     # h as the sum of two of the type
    least = 2.0 ** -24 if kind == "fp16" else 0.0                                  # (and the smallest number of it)
    y, off = np.zeros((T, D)), np.zeros((T, D))
    for t in range(T):
        for j in range(ids.shape[1]):
            e = ids[t, j]
            if not 0 <= e < E:
                continue
            both = up[e] @ x[t]
            size = (c1 * U + (2.0 ** -21 if kind == "fp32" else 0.0)) * (np.abs(up[e]) @ np.abs(x[t]))
            h = act(both, H, gated)
            if gated:
                g, v = both[:H], both[H:]
                # |silu'| <= 1.1; the exponential, the division and the product: 8 half steps
                dh = 1.1 * size[:H] * (np.abs(v) + size[H:]) + np.abs(g / (1 + np.exp(-g))) * size[H:] + 8 * U * np.abs(h)
            else:
                dh = size
            dh = dh + split * np.abs(h) + least
            z, mags = down[e] @ h, np.abs(down[e]) @ np.abs(h)
            y[t] += w[t, j] * z
            off[t] += abs(w[t, j]) * (np.abs(down[e]) @ dh + (c2 + 4) * U * mags + (2.0 ** -21 if kind == "fp32" else 0.0) * mags)
            off[t] += (off_w + (ids.shape[1] + 2) * U) * np.abs(w[t, j] * z)
    return y, off


def within(got, want, off, kind):
    """Asserts that got is want rounded to the type, give or take off."""
    got = np.asarray(got, np.float64)
    limit = off + HALF_STEP[kind] * (np.abs(want) + off) + (2.0 ** -25 if kind == "fp16" else 1e-45)
    bad = ~(np.abs(got - want) <= limit)
    assert not bad.any(), "%d of %d, worst %.3g at %s: %.9g for %.9g" % (
        bad.sum(), bad.size, np.max(np.abs(got - want) / limit), np.argwhere(bad)[0], got[bad][0], np.broadcast_to(want, got.shape)[bad][0])
