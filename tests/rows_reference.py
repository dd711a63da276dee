"""The row operators in 64 bits, plainly: what tests of the CUDA kernels compare with.  Shares no code with the library."""
import math

import numpy as np

HALF_STEP = {"fp32": 2.0 ** -24, "fp16": 2.0 ** -11, "bf16": 2.0 ** -8}     # a rounding, relative to the value


def route(logits, k, over_chosen):
    """[T, E] float64 -> (w [T, k], ids [T, k])."""
    T, E = logits.shape
    w, ids = np.zeros((T, k)), np.full((T, k), -1, np.int64)
    for t in range(T):
        row = np.where(np.isfinite(logits[t]), logits[t], -math.inf)
        best = [e for e in sorted(range(E), key=lambda e: (-row[e], e)) if row[e] > -math.inf][:k]
        if not best:
            continue
        top = row[best[0]]
        total = math.fsum(math.exp(row[e] - top) for e in (best if over_chosen else range(E)))
        for j, e in enumerate(best):
            ids[t, j], w[t, j] = e, math.exp(row[e] - top) / total
    return w, ids


def route_grad(logits, w, ids, dw, over_chosen, experts):
    T, k = ids.shape
    out = np.zeros((T, experts))
    for t in range(T):
        use = [j for j in range(k) if 0 <= ids[t, j] < experts]
        mean = sum(w[t, j] * dw[t, j] for j in use)
        if over_chosen:
            for j in use:
                out[t, ids[t, j]] += w[t, j] * (dw[t, j] - mean)
            continue
        row = np.where(np.isfinite(logits[t]), logits[t], -math.inf)
        if not np.any(row > -math.inf):
            continue
        p = np.exp(row - row.max())
        p /= p.sum()
        g = np.zeros(experts)
        for j in use:
            g[ids[t, j]] += dw[t, j]
        out[t] = p * (g - mean)
    return out


def sort(ids, experts):
    """ids [slots] -> (offsets [E + 1], order of the slots that ask, place [slots])."""
    offsets, order, place = [0], [], np.full(len(ids), -1, np.int64)
    for e in range(experts):
        for s in np.nonzero(ids == e)[0]:
            place[s] = len(order)
            order.append(int(s))
        offsets.append(len(order))
    return np.array(offsets), np.array(order, np.int64), place


def combine(z, place, w):
    T, k = place.shape
    y, size = np.zeros((T, z.shape[1])), np.zeros((T, z.shape[1]))
    for j in range(k):
        has = place[:, j] >= 0
        term = z[place[has, j]] * (w[has, j, None] if w is not None else 1.0)
        y[has] += term
        size[has] += np.abs(term)
    return y, size                       # (size: the sum of the terms' magnitudes)


def combine_grad(dy, z, place, w):
    T, k = place.shape
    dz, dw, size = np.zeros_like(z), np.zeros((T, k)), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            if place[t, j] >= 0:
                dz[place[t, j]] = dy[t] * (w[t, j] if w is not None else 1.0)
                dw[t, j] = dy[t] @ z[place[t, j]]
                size[t, j] = np.abs(dy[t]) @ np.abs(z[place[t, j]])
    return dz, dw, size


def offers(logits, scores, done, end_token):
    """One group's offers: a list over the beams of (total, token) best first, each beam by (larger logit, lower token)."""
    out = []
    for b in range(logits.shape[0]):
        s = scores[b]
        if not s < math.inf or s == -math.inf:
            out.append([])
        elif done is not None and done[b]:
            out.append([(float(s), end_token)])
        else:
            row = np.where(logits[b] < math.inf, logits[b], -math.inf)
            open_ = np.nonzero(row > -math.inf)[0]
            if not len(open_):
                out.append([])
                continue
            top = row.max()
            lse = top + math.log(math.fsum(np.exp(row[open_] - top)))
            order = open_[np.argsort(-row[open_], kind="stable")]
            out.append([(float(s) + (float(row[v]) - lse), int(v)) for v in order])
    return out


def check_selection(got_score, got_beam, got_token, logits, scores, done, end_token, C):
    """One group's selection against the definition.  Sums of different beams that are nearer to each other than the
    32-bit terms of the row sums allow (see below) may stand in either order."""
    lists = offers(logits, scores, done, end_token)
    best = sorted(((-total, b, r, token) for b, l in enumerate(lists) for r, (total, token) in enumerate(l[:C])))[:C]
    n = len(best)
    assert (got_beam[n:] == -1).all() and (got_token[n:] == -1).all() and np.isneginf(got_score[n:]).all()
    # a row's sum, in half steps of 2^-24 relative to it: a term is an exponential within 2 units of its last place (4) of a
    # product (1) of a difference (x e^-x of one: 0.4), four additions in 32 bits (4), and three factors that bring sums to a
    # common reference, each an exponential of a product with a product (3 * 5 + 0.6 for the differences): 25; the whole
    # numbers that warps add up are off by 2^-26 at most.  Two rows are compared.
    near = 2 * (25 * 2.0 ** -24 + 2.0 ** -26)
    taken = [0] * len(lists)
    for i in range(n):
        b = int(got_beam[i])
        total, token = lists[b][taken[b]]        # within a beam the order has no freedom
        assert got_token[i] == token, (i, b)
        taken[b] += 1
        want = -best[i][0]
        assert abs(total - want) <= near, (i, total, want)
        alone = (i == 0 or -best[i - 1][0] - want > near) and (i + 1 >= n or want + best[i + 1][0] > near)
        same_rows = [q for q in (i - 1, i + 1) if 0 <= q < n and best[q][0] == best[i][0]]
        if alone or same_rows:
            assert (b, token) == (best[i][1], best[i][3]) or (same_rows and not alone and abs(total - want) <= near
                                                                and total != want), (i, b, token, best[i])
        assert abs(float(got_score[i]) - total) <= near + abs(total) * 2.0 ** -24, (i, got_score[i], total)
