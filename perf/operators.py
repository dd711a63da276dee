"""The row operators that are timed: what a learner with expert layers and a policy that searches with beams
do to a batch, next to drawing it from the replay buffer.

Fields of a case
  op        "route"     the router: the k best of E experts for each of `rows` rows, with softmax weights
            "dispatch"  rows sorted by expert: the plan from the expert ids, then the rows' copy
            "combine"   the experts' answers brought back to their rows, weighted
            "gradient"  the gradients of "combine" (answers and weights) and of "dispatch" (rows)
            "select"    one step of a beam search: the best continuations of each group of beams
            "reorder"   the beams' states moved to where that choice says
  rows, experts, k, width    T, E, k and the elements of a row
  dropped   part of the slots that go to no expert (a capacity limit did that)
  barred    part of the logits that are -inf (experts that are off, tokens that are not allowed)
  chosen    the router's softmax runs over the chosen experts (else over all)
  grad      the router's gradient is part of the pass
  groups, beams, vocab, best    G, W, V, and the candidates kept for a group
  done      part of the beams that are finished
  blocks, heads, length, room, dim     a cache [blocks, G, W, heads, room, dim] of which `length` positions are used
  kept      beams of a group that survive the choice (the others' states are read by nobody)
  inplace   the states are moved within the cache, else into a second one
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def route(name, dtype, rows, experts, k, barred=0.0, chosen=True, grad=False):
    return {"name": name, "op": "route", "dtype": dtype, "rows": rows, "experts": experts, "k": k, "barred": barred,
            "chosen": chosen, "grad": grad}


def expert(name, op, dtype, rows, experts, k, width, dropped=0.0):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "experts": experts, "k": k, "width": width,
            "dropped": dropped}


def select(name, dtype, groups, beams, vocab, best, barred=0.0, done=0.0):
    return {"name": name, "op": "select", "dtype": dtype, "groups": groups, "beams": beams, "vocab": vocab, "best": best,
            "barred": barred, "done": done}


def reorder(name, dtype, blocks, groups, beams, kept, heads, length, room, dim, inplace):
    return {"name": name, "op": "reorder", "dtype": dtype, "blocks": blocks, "groups": groups, "beams": beams,
            "kept": kept, "heads": heads, "length": length, "room": room, "dim": dim, "inplace": inplace}


def listed():
    return [
        # a classic-control learner's batch before a small expert layer: launches are the whole cost
        route("route_step", "fp32", 64, 8, 2, chosen=False),
        # a training batch of a large layer: forward and gradient, some experts off
        route("route_train", "bf16", 65521, 128, 8, barred=0.02, grad=True),
        # the observations of a continuous-control batch (rows of 68 bytes) sent to their experts
        expert("dispatch_step", "dispatch", "fp32", 256, 8, 2, 17),
        # a training batch's hidden states
        expert("dispatch_train", "dispatch", "bf16", 16381, 64, 8, 2048),
        # a policy step: few rows, many experts
        expert("combine_step", "combine", "bf16", 64, 128, 8, 4096),
        # a training batch, a tenth of its slots over the experts' capacity
        expert("combine_train", "combine", "fp16", 32768, 64, 4, 2048, dropped=0.1),
        # a small learner's gradient in full precision
        expert("gradient_step", "gradient", "fp32", 1000, 16, 2, 500, dropped=0.25),
        # a training batch's gradient
        expert("gradient_train", "gradient", "bf16", 8192, 256, 8, 4096),
        # planning for a single environment: latency
        select("select_step", "fp32", 1, 4, 32003, 8, barred=0.01),
        # many plans at once over a large vocabulary, some beams finished
        select("select_batch", "bf16", 64, 8, 131072, 16, done=0.1),
        # a short history's states into the other of two caches
        reorder("reorder_step", "fp16", 2, 4, 4, 3, 4, 33, 64, 64, False),
        # a long history's states within one cache that is nearly full
        reorder("reorder_cache", "bf16", 16, 8, 8, 5, 8, 500, 512, 128, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "dispatch", "combine", "gradient", "select", "reorder"])
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    size = BYTES[dtype]
    if op == "route":
        experts = _log(rng, 2, 512)
        rows = _log(rng, 1, min(65536, (1 << 23) // experts))
        return route("", dtype, rows, experts, rng.randint(1, min(8, experts)), barred=rng.choice([0.0, 0.0, 0.05, 0.3]),
                     chosen=rng.random() < 0.5, grad=rng.random() < 0.5)
    if op in ("dispatch", "combine", "gradient"):
        experts = _log(rng, 2, 512)
        k = rng.randint(1, min(8, experts))
        width = rng.choice([17, _log(rng, 8, 8192), 8 * _log(rng, 8, 1024), 8 * _log(rng, 8, 1024)])
        rows = _log(rng, 1, max(2, min(65536, (1 << 28) // (k * width * size))))
        return expert("", op, dtype, rows, experts, k, width, dropped=rng.choice([0.0, 0.0, round(rng.uniform(0.02, 0.6), 2)]))
    beams = rng.choice([1, 2, 3, 4, 5, 8, 16])
    if op == "select":
        vocab = _log(rng, 300, 262144)
        groups = _log(rng, 1, max(1, min(256, (1 << 26) // (beams * vocab))))
        best = min(vocab, rng.choice([beams, 2 * beams, 2 * beams]))
        return select("", dtype, groups, beams, vocab, best, barred=rng.choice([0.0, 0.0, 0.02]), done=rng.choice([0.0, 0.0, 0.2]))
    heads, dim, blocks = rng.choice([1, 2, 4, 8]), rng.choice([33, 64, 64, 128]), 2 * rng.randint(1, 12)
    room = _log(rng, 4, max(8, min(4096, (1 << 28) // (blocks * beams * heads * dim * size))))
    groups = _log(rng, 1, max(1, min(64, (1 << 28) // (blocks * beams * heads * room * dim * size))))
    return reorder("", dtype, blocks, groups, beams, rng.randint(1, beams), heads, rng.randint(max(1, room // 2), room), room, dim,
                   rng.random() < 0.5)


def _open_logits(gen, shape, c, spread):
    """Normal logits in the case's type, some of them barred."""
    x = (torch.randn(shape, device=gen.device, generator=gen) * spread).to(TYPES[c["dtype"]])
    if c["barred"]:
        x.masked_fill_(torch.rand(shape, device=gen.device, generator=gen) < c["barred"], -math.inf)
    return x


def _ids(gen, c):
    """Experts as a router gives them: k different ones a row, some more wanted than others; -1 for a dropped slot."""
    T, E, k = c["rows"], c["experts"], c["k"]
    want = torch.rand((T, E), device=gen.device, generator=gen) + 0.3 * torch.rand(E, device=gen.device, generator=gen)
    ids = want.topk(k, dim=1).indices.to(torch.int32)
    if c["dropped"]:
        ids.masked_fill_(torch.rand((T, k), device=gen.device, generator=gen) < c["dropped"], -1)
    return ids


def _places(ids, experts):
    """The sorted row of every slot, -1 for a dropped one."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, experts), flat)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    return torch.where(flat < 0, torch.full_like(place, -1), place).to(torch.int32).view(ids.shape)


def prepare(c, seed):
    dev = torch.device("cuda:%d" % torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = TYPES[c["dtype"]]
    s = {"case": c}

    def values(*shape, dtype=t):
        return torch.randn(shape, device=dev, generator=gen, dtype=dtype)

    def room(*shape, dtype=t):
        return torch.zeros(shape, device=dev, dtype=dtype)

    if c["op"] == "route":
        T, E, k = c["rows"], c["experts"], c["k"]
        s["logits"] = _open_logits(gen, (T, E), c, 1.5)
        s["w"], s["ids"] = room(T, k, dtype=torch.float32), room(T, k, dtype=torch.int32)
        if c["grad"]:
            s["dw"], s["dlogits"] = values(T, k, dtype=torch.float32), room(T, E)
    elif c["op"] in ("dispatch", "combine", "gradient"):
        T, E, k, D = c["rows"], c["experts"], c["k"], c["width"]
        s["ids"] = _ids(gen, c)
        if c["op"] == "dispatch":
            s["x"], s["xs"] = values(T, D), room(T * k, D)
            s["offsets"] = room(E + 1, dtype=torch.int32)
            s["order"], s["place"] = room(T * k, dtype=torch.int32), room(T, k, dtype=torch.int32)
        else:
            s["place"] = _places(s["ids"], E)
            s["w"] = torch.softmax(values(T, k, dtype=torch.float32), dim=1)
            s["z"] = values(T * k, D)
            if c["op"] == "combine":
                s["y"] = room(T, D)
            else:
                s["dy"], s["dxs"] = values(T, D), values(T * k, D)
                s["dz"], s["dw"], s["dx"] = room(T * k, D), room(T, k, dtype=torch.float32), room(T, D)
    elif c["op"] == "select":
        G, W, V, C = c["groups"], c["beams"], c["vocab"], c["best"]
        s["logits"] = _open_logits(gen, (G, W, V), c, 2.5)
        s["scores"] = -20.0 * torch.rand((G, W), device=dev, generator=gen)
        s["done"] = (torch.rand((G, W), device=dev, generator=gen) < c["done"]).to(torch.uint8)
        s["best"] = (room(G, C, dtype=torch.float32), room(G, C, dtype=torch.int32), room(G, C, dtype=torch.int32))
    else:
        B, G, W = c["blocks"], c["groups"], c["beams"]
        shape = (B, G, W, c["heads"], c["room"], c["dim"])
        s["states"] = values(*shape)
        s["other"] = None if c["inplace"] else room(*shape)
        # `kept` beams survive, each of them at least once, in any order
        kept = torch.rand((G, W), device=dev, generator=gen).argsort(dim=1)[:, :c["kept"]]
        pick = torch.cat([torch.arange(c["kept"], device=dev).expand(G, -1),
                          torch.randint(0, c["kept"], (G, W - c["kept"]), device=dev, generator=gen)], dim=1)
        pick = pick.gather(1, torch.rand((G, W), device=dev, generator=gen).argsort(dim=1))
        s["parent"] = kept.gather(1, pick).to(torch.int32).contiguous()
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _falling(x):
    """Whole numbers that order the last axis of x: larger value first, ties by the lower index; all different."""
    bits = (x.float() + 0.0).view(torch.int32).long()        # (-0 becomes 0)
    rising = torch.where(bits < 0, -2147483648 - bits, bits)
    return rising * 4294967296 + (4294967295 - torch.arange(x.shape[-1], device=x.device))


def _plain_route(c, logits):
    x = logits.float()
    ids = _falling(logits).topk(c["k"], dim=1).indices
    best = x.gather(1, ids)
    top = best[:, :1]
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = (best - top).exp()
    total = e.sum(1, keepdim=True) if c["chosen"] else (x - top).exp().sum(1, keepdim=True)
    shut = best == -math.inf
    w = torch.where(shut, torch.zeros_like(e), e / total)
    return w, torch.where(shut, torch.full_like(ids, -1), ids).to(torch.int32)


def _plain_route_gradient(c, logits, w, ids, dw):
    x = logits.float()
    mean = (w * dw).sum(1, keepdim=True)
    here = (ids >= 0).float()
    at = ids.clamp_min(0).long()
    if c["chosen"]:
        return torch.zeros_like(x).scatter_add_(1, at, w * (dw - mean) * here).to(logits.dtype)
    top = x.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = (x - top).exp()
    p = e / e.sum(1, keepdim=True).clamp_min(1e-30)
    g = torch.zeros_like(x).scatter_add_(1, at, dw * here)
    return (p * (g - mean)).to(logits.dtype)


def _plain_plan(c, ids):
    E, n = c["experts"], ids.numel()
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, torch.full_like(flat, E), flat)
    sorted_key, order = torch.sort(key, stable=True)
    offsets = torch.searchsorted(sorted_key, torch.arange(E + 1, device=ids.device)).to(torch.int32)
    place = torch.empty_like(order)
    place[order] = torch.arange(n, device=ids.device)
    place = torch.where(flat < 0, torch.full_like(place, -1), place)
    order = torch.where(sorted_key < E, order, torch.zeros_like(order))     # rows behind the last one are not written
    return offsets, order.to(torch.int32), place.to(torch.int32).view(ids.shape)


def _plain_gather(z, place):
    """The rows at `place`, in 32 bits; zeros for a slot without one."""
    rows = z[place.clamp_min(0).long()].float()
    return rows.masked_fill_((place < 0).unsqueeze(-1), 0.0)


def _plain_spread(rows, place, like):
    """rows[slot] written to place[slot]; the other rows zero."""
    flat = place.reshape(-1).long()
    out = torch.zeros((like.shape[0] + 1, like.shape[1]), dtype=like.dtype, device=like.device)
    out[torch.where(flat < 0, torch.full_like(flat, like.shape[0]), flat)] = rows
    return out[:-1]


def _plain_select(c, logits, scores, done):
    G, W, V, C = c["groups"], c["beams"], c["vocab"], c["best"]
    x = logits.float()
    token = _falling(logits).topk(C, dim=2).indices                          # the best of each beam ...
    best = x.gather(2, token).double()
    top = best[:, :, :1]
    lse = top + (x - top.float()).exp().sum(2, keepdim=True, dtype=torch.float64).log()
    total = scores.double().unsqueeze(2) + (best - lse)
    over = done.bool().unsqueeze(2)
    first = (torch.arange(C, device=x.device) == 0).view(1, 1, C)
    ended = torch.where(first, scores.double().unsqueeze(2), torch.full_like(total, -math.inf))
    total = torch.where(over, ended, total).view(G, W * C)
    token = torch.where(over, torch.full_like(token, END), token).view(G, W * C)
    total, at = torch.sort(total, dim=1, descending=True, stable=True)       # ... and the best of those
    total, at = total[:, :C], at[:, :C]
    none = total == -math.inf
    parent = torch.where(none, torch.full_like(at, -1), at // C)
    token = torch.where(none, torch.full_like(at, -1), token.gather(1, at))
    return total.float(), parent.to(torch.int32), token.to(torch.int32)


END = 2        # the token that ends a sequence


def _used(c, states):
    return states[:, :, :, :, :c["length"]]


def _plain(s):
    c = s["case"]
    if c["op"] == "route":
        w, ids = _plain_route(c, s["logits"])
        return (w, ids, _plain_route_gradient(c, s["logits"], w, ids, s["dw"])) if c["grad"] else (w, ids)
    if c["op"] == "dispatch":
        offsets, order, place = _plain_plan(c, s["ids"])
        rows = s["x"].unsqueeze(1).expand(-1, c["k"], -1).reshape(-1, c["width"])
        return offsets, order, place, _plain_spread(rows, place, s["xs"])
    if c["op"] == "combine":
        return (_plain_gather(s["z"], s["place"]) * s["w"].unsqueeze(-1)).sum(1).to(s["z"].dtype)
    if c["op"] == "gradient":
        dy = s["dy"].float().unsqueeze(1)
        dw = (_plain_gather(s["z"], s["place"]) * dy).sum(2)
        dz = _plain_spread((dy * s["w"].unsqueeze(-1)).to(s["z"].dtype).reshape(-1, c["width"]), s["place"], s["z"])
        return dz, dw, _plain_gather(s["dxs"], s["place"]).sum(1).to(s["z"].dtype)
    if c["op"] == "select":
        return _plain_select(c, s["logits"], s["scores"], s["done"])
    at = s["parent"].long().view(1, c["groups"], c["beams"], 1, 1, 1)
    used = _used(c, s["states"])
    to = s["states"] if c["inplace"] else s["other"]
    _used(c, to).copy_(torch.gather(used, 2, at.expand_as(used)))
    return to


# ---- the framework's calls ----------------------------------------------------------------------------------------

_routers = {}


def _router(s):
    """The program's handle of the current stream: made once for it, and kept where the program keeps its tensors."""
    device = s.get("device")
    if device is None:
        device = s["device"] = torch.cuda.current_device()
    stream = torch._C._cuda_getCurrentRawStream(device)      # (as a number: a stream object takes as long as a small call)
    if s.get("stream") != stream:
        key = (device, stream)
        if key not in _routers:
            from paper_2311_09445_b200 import RowRouter
            _routers[key] = RowRouter(stream=torch.cuda.current_stream(device))
        s["stream"], s["router"] = stream, _routers[key]
    return s["router"]


def _own(s):
    c, r = s["case"], _router(s)
    if c["op"] == "route":
        r.route(s["logits"], s["w"], s["ids"], over_chosen=c["chosen"])
        if not c["grad"]:
            return s["w"], s["ids"]
        r.route_grad(s["logits"], s["w"], s["ids"], s["dw"], s["dlogits"], over_chosen=c["chosen"])
        return s["w"], s["ids"], s["dlogits"]
    if c["op"] == "dispatch":
        r.sort(s["ids"], c["experts"], s["offsets"], s["order"], s["place"])
        r.dispatch(s["x"], s["place"], s["xs"])
        return s["offsets"], s["order"], s["place"], s["xs"]
    if c["op"] == "combine":
        r.combine(s["z"], s["place"], s["w"], s["y"])
        return s["y"]
    if c["op"] == "gradient":
        r.combine_grad(s["dy"], s["z"], s["place"], s["w"], s["dz"], s["dw"])
        r.dispatch_grad(s["dxs"], s["place"], s["dx"])
        return s["dz"], s["dw"], s["dx"]
    if c["op"] == "select":
        r.beam_select(s["logits"], s["scores"], *s["best"], done=s["done"], end_token=END)
        return s["best"]
    to = s["states"] if c["inplace"] else s["other"]
    r.beam_reorder(_used(c, s["states"]), s["parent"], _used(c, to))
    return to


def run(s):
    return _own(s) if own else _plain(s)


def work(c):
    size = BYTES[c["dtype"]]
    if c["op"] == "route":
        T, E, k = c["rows"], c["experts"], c["k"]
        nbytes = T * E * size + 8 * T * k + (T * E * size + 4 * T * k if c["grad"] else 0)
        return {"bytes": nbytes, "flops": T * E * 4 * (2 if c["grad"] else 1)}
    if c["op"] in ("dispatch", "combine", "gradient"):
        T, k, row = c["rows"], c["k"], c["width"] * size
        slots, routed = T * k, T * k * (1.0 - c["dropped"])
        if c["op"] == "dispatch":
            return {"bytes": T * row + routed * (row + 4) + 8 * slots + 4 * (c["experts"] + 1), "flops": 0}
        if c["op"] == "combine":
            return {"bytes": routed * row + T * row + 8 * slots, "flops": 2 * routed * c["width"]}
        # answers in and out, the rows' gradient in twice (of "combine" and, sorted, of "dispatch") and out
        return {"bytes": 3 * routed * row + 2 * T * row + 12 * slots, "flops": 4 * routed * c["width"]}
    G, W = c["groups"], c["beams"]
    if c["op"] == "select":
        rows = G * W * (1.0 - c["done"])
        return {"bytes": rows * c["vocab"] * size + 5 * G * W + 12 * G * c["best"], "flops": 4 * rows * c["vocab"]}
    row = c["blocks"] * c["heads"] * c["length"] * c["dim"] * size
    moved = W - 1 if c["inplace"] else W                 # (in place a beam stays where it is once in W times)
    return {"bytes": G * row * (c["kept"] + moved) + 4 * G * W, "flops": 0}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "route":
        T, E, k = c["rows"], c["experts"], c["k"]
        x = s["logits"].double()
        left, w, picked = x.clone(), [], []
        shut = torch.zeros(T, dtype=torch.bool, device=x.device)
        for _ in range(k):                       # the largest that is left, the first of equal ones
            best = left.amax(1, keepdim=True)
            at = torch.where(left == best, torch.arange(E, device=x.device), E).amin(1, keepdim=True)
            shut = best.squeeze(1) == -math.inf
            picked.append(torch.where(shut, -1, at.squeeze(1)))
            w.append(torch.where(shut, -math.inf, x.gather(1, at).squeeze(1)))
            left.scatter_(1, at, -math.inf)
        v, at = torch.stack(w, 1), torch.stack(picked, 1)
        over = v if c["chosen"] else x
        lse = torch.logsumexp(over, 1, keepdim=True)
        weight = torch.where(v == -math.inf, 0.0, (v - lse).exp())
        if not c["grad"]:
            return weight, None
        g = s["dw"].double()
        mark = (torch.arange(E, device=x.device).view(1, 1, E) == at.unsqueeze(2)) if T * k * E < 1 << 27 else None
        if mark is not None:
            scattered = (mark * g.unsqueeze(2)).sum(1)
            member = mark.any(1)
        else:
            scattered, member = torch.zeros_like(x), torch.zeros_like(x, dtype=torch.bool)
            for j in range(k):
                one = torch.arange(E, device=x.device).view(1, E) == at[:, j:j + 1]
                scattered += one * g[:, j:j + 1]
                member |= one
        p = torch.where(x == -math.inf, 0.0, (x - lse).exp())
        if c["chosen"]:
            p = p * member
        return weight, None, p * (scattered - (p * scattered).sum(1, keepdim=True))
    if c["op"] in ("dispatch", "combine", "gradient"):
        T, E, k, D = c["rows"], c["experts"], c["k"], c["width"]
        flat = s["ids"].reshape(-1)
        by_expert = [torch.nonzero(flat == e).squeeze(1) for e in range(E)]
        order = torch.cat(by_expert)             # slots in sorted order
        n, step = order.numel(), max(1, (1 << 24) // D)
        if c["op"] == "dispatch":
            xs = torch.zeros((T * k, D), dtype=torch.float64, device=flat.device)
            for a in range(0, n, step):
                xs[a:min(n, a + step)] = s["x"][order[a:a + step] // k].double()
            return None, None, None, xs
        y = torch.zeros((T, D), dtype=torch.float64, device=flat.device)
        w = s["w"].double().reshape(-1)
        if c["op"] == "combine":
            for a in range(0, n, step):
                slot = order[a:a + step]
                y.index_add_(0, slot // k, s["z"][a:min(n, a + step)].double() * w[slot].unsqueeze(1))
            return y
        dz = torch.zeros((T * k, D), dtype=torch.float64, device=flat.device)
        dw = torch.zeros(T * k, dtype=torch.float64, device=flat.device)
        for a in range(0, n, step):
            slot, b = order[a:a + step], min(n, a + step)
            dy = s["dy"][slot // k].double()
            dz[a:b] = dy * w[slot].unsqueeze(1)
            dw[slot] = torch.einsum("rd,rd->r", dy, s["z"][a:b].double())
            y.index_add_(0, slot // k, s["dxs"][a:b].double())
        return dz, dw.view(T, k), y
    if c["op"] == "select":
        G, W, V, C = c["groups"], c["beams"], c["vocab"], c["best"]
        out = torch.full((G, C), -math.inf, dtype=torch.float64, device=s["scores"].device)
        for g in range(G):
            total = torch.log_softmax(s["logits"][g].double(), dim=1) + s["scores"][g].double().unsqueeze(1)
            alone = torch.full((W, V), -math.inf, dtype=torch.float64, device=total.device)
            alone[:, 0] = s["scores"][g].double()
            total = torch.where(s["done"][g].bool().unsqueeze(1), alone, total).reshape(-1)
            best = torch.sort(total.topk(min(C, total.numel())).values, descending=True).values
            out[g, :best.numel()] = best
        return out, None, None
    to = s["states"].clone() if c["inplace"] else s["other"]
    for g in range(c["groups"]):
        for i, b in enumerate(s["parent"][g].tolist()):
            to[:, g, i, :, :c["length"]] = s["states"][:, g, b, :, :c["length"]]
    return to
