"""The operators of a layer that are timed: what a learner and a policy compute around the router and the rows' way to their
experts and back -- the norm before a layer, the dropout behind it, and a whole expert layer for the few rows of a policy step.

Fields of a case
  op        "norm"       the layer norm of each row, with its mean and reciprocal deviation
            "norm_grad"  its gradient: the rows', and the weight's and the bias's, which are sums over all rows
            "dropout"    a branch's rows with elements dropped, added to the residual rows; with `grad` the branch's gradient too
            "experts"    an expert layer: the router's product and choice, the chosen experts' products and their weighted sum
  rows, width            T, and the elements D of a row
  params    the type of the norm's weight and bias
  affine    the norm has a weight and a bias
  ld        elements from a row to the next one (0: the rows are dense)
  p         the probability of dropping an element
  experts, k, hidden     E, the experts chosen for a row, and the elements H between an expert's two products
  gated     an expert's first product has a gate: silu(gate) * value; else relu(value)
  chosen    the router's softmax runs over the chosen experts (else over all)
  barred    part of the slots that have no expert (given choices instead of the router's: -1); 0: the layer has its own router
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5


def norm(name, op, dtype, rows, width, params="fp32", affine=True, ld=0):
    return {"name": name, "op": op, "dtype": dtype, "rows": rows, "width": width, "params": params, "affine": affine, "ld": ld}


def dropout(name, dtype, rows, width, p, grad=False):
    return {"name": name, "op": "dropout", "dtype": dtype, "rows": rows, "width": width, "p": p, "grad": grad}


def experts(name, dtype, rows, width, hidden, number, k, gated=True, chosen=True, barred=0.0):
    return {"name": name, "op": "experts", "dtype": dtype, "rows": rows, "width": width, "hidden": hidden, "experts": number,
            "k": k, "gated": gated, "chosen": chosen, "barred": barred}


def listed():
    return [
        # a continuous-control batch's observations (17 numbers each) before a small network: the call is the whole cost
        norm("norm_step", "norm", "fp32", 256, 17),
        # a training batch's hidden states
        norm("norm_train", "norm", "bf16", 16381, 2048, params="bf16"),
        # the same small learner's gradient
        norm("norm_grad_step", "norm_grad", "fp32", 1000, 500),
        # a training batch's gradient
        norm("norm_grad_train", "norm_grad", "bf16", 16384, 4096),
        # wide rows of an odd length, in a larger matrix
        norm("norm_grad_wide", "norm_grad", "fp16", 2011, 12289, params="fp16", ld=12304),
        # a small learner's branch
        dropout("dropout_step", "fp32", 256, 500, 0.1),
        # a training batch's branch, and its gradient
        dropout("dropout_train", "bf16", 16384, 4096, 0.1, grad=True),
        # one environment's policy step through a small layer: latency
        experts("experts_one", "bf16", 1, 512, 1024, 8, 2, chosen=False),
        # a policy's step in a few environments, full precision, odd sizes, without gates
        experts("experts_odd", "fp32", 9, 500, 333, 16, 4, gated=False),
        # a search for one environment with 4 beams over many experts
        experts("experts_beams", "bf16", 4, 2048, 768, 128, 8),
        # a policy's step in 64 environments, some of their choices over the experts' capacity
        experts("experts_batch", "fp16", 64, 2048, 1408, 64, 6, barred=0.05),
        # the largest layer
        experts("experts_large", "bf16", 64, 4096, 1280, 128, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "dropout", "experts", "experts"])
    dtype = rng.choice(["bf16", "fp16", "fp32"])
    size = BYTES[dtype]
    if op == "experts":
        number = _log(rng, 2, 128)
        k = rng.randint(1, min(8, number))
        width = rng.choice([_log(rng, 16, 4096), 8 * _log(rng, 4, 512), 64 * _log(rng, 1, 64)])
        most = (1 << 30) // (3 * number * width * size)
        hidden = rng.choice([_log(rng, 16, max(17, min(2048, most))), 8 * _log(rng, 2, max(3, min(256, most // 8)))])
        return experts("", dtype, _log(rng, 1, 64), width, hidden, number, k, gated=rng.random() < 0.7, chosen=rng.random() < 0.5,
                       barred=rng.choice([0.0, 0.0, round(rng.uniform(0.02, 0.6), 2)]))
    width = rng.choice([17, _log(rng, 8, 16384), 8 * _log(rng, 1, 2048), 8 * _log(rng, 1, 2048)])
    rows = _log(rng, 1, max(2, min(65536, (1 << 27) // (width * size))))
    if op == "dropout":
        return dropout("", dtype, rows, width, rng.choice([0.1, 0.1, 0.5, round(rng.uniform(0.0, 0.9), 3)]), grad=rng.random() < 0.5)
    return norm("", op, dtype, rows, width, params=rng.choice([dtype, "fp32"]), affine=rng.random() < 0.8,
                ld=rng.choice([0, 0, width + 8 * rng.randint(1, 8), width + rng.randint(1, 8)]))


def prepare(c, seed):
    dev = torch.device("cuda:%d" % torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = TYPES[c["dtype"]]
    T, D = c["rows"], c["width"]
    s = {"case": c}

    def values(*shape, dtype=t, scale=1.0):
        x = torch.randn(shape, device=dev, generator=gen, dtype=dtype)
        return x.mul_(scale) if scale != 1.0 else x

    def room(*shape, dtype=t):
        return torch.zeros(shape, device=dev, dtype=dtype)

    def matrix(x=None):
        """x, or room for it, as rows of the case's distance."""
        m = room(T, c["ld"] or D)[:, :D]
        return m if x is None else m.copy_(x)

    if c["op"] in ("norm", "norm_grad"):
        pt = TYPES[c["params"]]
        # hidden states: rows of different size, off zero, with a few features that are always large
        x = values(T, D, dtype=torch.float32) * (0.5 + 2.0 * torch.rand((T, 1), device=dev, generator=gen)) + 0.3
        x[:, ::97] *= 8.0
        s["x"] = matrix(x.to(t))
        s["gamma"] = (1.0 + 0.1 * values(D, dtype=torch.float32)).to(pt) if c["affine"] else None
        s["beta"] = values(D, dtype=pt, scale=0.1) if c["affine"] else None
        s["mean"], s["rstd"] = room(T, dtype=torch.float32), room(T, dtype=torch.float32)
        if c["op"] == "norm":
            s["y"] = matrix()
        else:
            x = s["x"].double()
            s["mean"].copy_(x.mean(1))
            s["rstd"].copy_((x.var(1, unbiased=False) + EPS).rsqrt())
            s["dy"], s["dx"] = matrix(values(T, D)), matrix()
            s["dgamma"], s["dbeta"] = (room(D, dtype=torch.float32), room(D, dtype=torch.float32)) if c["affine"] else (None, None)
    elif c["op"] == "dropout":
        s["x"], s["residual"], s["y"] = values(T, D), values(T, D), room(T, D)
        if c["grad"]:
            s["dy"], s["dx"] = values(T, D), room(T, D)
        s["seed"], s["call"] = 1000003 * seed + 7, seed & 0xFFFF       # a run's seed, and the number of the call in it
    else:
        E, H, k = c["experts"], c["hidden"], c["k"]
        s["x"], s["y"] = values(T, D), room(T, D)
        s["up"] = values(E, (2 if c["gated"] else 1) * H, D, scale=D ** -0.5)
        s["down"] = values(E, D, H, scale=H ** -0.5)
        s["router"] = None
        s["w"], s["ids"] = room(T, k, dtype=torch.float32), room(T, k, dtype=torch.int32)
        if c["barred"]:
            s["w"].copy_(torch.softmax(values(T, k, dtype=torch.float32), dim=1))
            s["ids"].copy_(torch.rand((T, E), device=dev, generator=gen).topk(k, dim=1).indices)
            s["ids"].masked_fill_(torch.rand((T, k), device=dev, generator=gen) < c["barred"], -1)
        else:
            s["router"] = values(E, D, scale=1.5 * D ** -0.5)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    rstd = ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    y = (x - mean) * rstd
    if s["gamma"] is not None:
        y = y * s["gamma"].float() + s["beta"].float()
    return y.to(s["x"].dtype), mean.squeeze(1), rstd.squeeze(1)


def _plain_norm_grad(s):
    rstd = s["rstd"].unsqueeze(1)
    normed = (s["x"].float() - s["mean"].unsqueeze(1)) * rstd
    dy = s["dy"].float()
    g = dy * s["gamma"].float() if s["gamma"] is not None else dy
    dx = rstd * (g - g.mean(1, keepdim=True) - normed * (g * normed).mean(1, keepdim=True))
    if s["gamma"] is None:
        return (dx.to(s["x"].dtype),)
    return dx.to(s["x"].dtype), (dy * normed).sum(0), dy.sum(0)


def _times(a, b):
    """The high and the low half of the product of 32-bit numbers a (a tensor of 64-bit integers) and b."""
    low, high = a & 0xFFFF, a >> 16
    middle = high * (b & 0xFFFF) + ((low * (b & 0xFFFF)) >> 16)
    upper = low * (b >> 16) + (middle & 0xFFFF)
    return high * (b >> 16) + (middle >> 16) + (upper >> 16), ((upper & 0xFFFF) << 16) | ((low * (b & 0xFFFF)) & 0xFFFF)


def _philox_round(c, k0, k1):
    h0, l0 = _times(c[0], 0xD2511F53)
    h1, l1 = _times(c[2], 0xCD9E8D57)
    return h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0


def _kept(s):
    """Which elements stay: 16 bits each of Philox4x32-10 with the counter (column / 8, row, call), compared with p * 2^16."""
    c = s["case"]
    dev = s["x"].device
    groups = -(-c["width"] // 8)
    col = torch.arange(groups, device=dev).expand(c["rows"], groups)
    row = torch.arange(c["rows"], device=dev).unsqueeze(1).expand(c["rows"], groups)
    call = torch.full_like(col, s["call"])
    words = (col, row, call & 0xFFFFFFFF, call >> 32)
    for i in range(10):
        words = _philox_round(words, ((s["seed"] & 0xFFFFFFFF) + i * 0x9E3779B9) & 0xFFFFFFFF, ((s["seed"] >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=2)
    return halves.reshape(c["rows"], groups * 8)[:, :c["width"]] >= _threshold(c["p"])


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _plain_dropout(s):
    c = s["case"]
    kept, scale = _kept(s), 65536.0 / max(1, 65536 - _threshold(c["p"]))
    zero = torch.zeros((), device=kept.device)
    y = (torch.where(kept, s["x"].float() * scale, zero) + s["residual"].float()).to(s["x"].dtype)
    return (y, torch.where(kept, s["dy"].float() * scale, zero).to(s["x"].dtype)) if c["grad"] else (y,)


def _act(c, both):
    if not c["gated"]:
        return both.clamp_min(0.0)
    gate, value = both[..., :c["hidden"]], both[..., c["hidden"]:]
    return gate / (1.0 + torch.exp(-gate)) * value


def _plain_experts(s):
    c = s["case"]
    T, E, k = c["rows"], c["experts"], c["k"]
    x, w, ids = s["x"].float(), s["w"], s["ids"]
    if s["router"] is not None:
        # in 64 bits, rounded to 32: two experts' logits may be near to each other
        logits = (s["x"].double() @ s["router"].double().t()).float()
        order = torch.sort(logits, dim=1, descending=True, stable=True)
        best, ids = order.values[:, :k], order.indices[:, :k].to(torch.int32)
        e = (best - best[:, :1]).exp()
        w = e / (e.sum(1, keepdim=True) if c["chosen"] else (logits - best[:, :1]).exp().sum(1, keepdim=True))
    at = ids.reshape(-1).clamp_min(0).long()
    if T * k <= E:                                             # few slots: the slots' own experts
        rows = x.unsqueeze(1).expand(T, k, -1).reshape(T * k, 1, -1)
        z = torch.bmm(_act(c, torch.bmm(rows, s["up"][at].float().transpose(1, 2))), s["down"][at].float().transpose(1, 2)).view(T, k, -1)
    else:                                                      # else all rows through all experts, of which the slots' are taken
        h = _act(c, torch.matmul(x, s["up"].float().transpose(1, 2)))
        z = torch.bmm(h, s["down"].float().transpose(1, 2))
        z = z[at, torch.arange(T, device=x.device).repeat_interleave(k)].view(T, k, -1)
    y = (z * torch.where(ids < 0, torch.zeros_like(w), w).unsqueeze(2)).sum(1)
    return y.to(s["x"].dtype), w, ids


def _plain(s):
    op = s["case"]["op"]
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "dropout": _plain_dropout, "experts": _plain_experts}[op](s)


# ---- the framework's calls ----------------------------------------------------------------------------------------

_handles = {}


def _handle(s):
    """The program's handle of the current stream: made once for it, and kept where the program keeps its tensors."""
    device = s.get("device")
    if device is None:
        device = s["device"] = torch.cuda.current_device()
    stream = torch._C._cuda_getCurrentRawStream(device)
    if s.get("stream") != stream:
        key = (device, stream)
        if key not in _handles:
            from paper_2311_09445_b200 import RowLayers
            _handles[key] = RowLayers(stream=torch.cuda.current_stream(device))
        s["stream"], s["handle"] = stream, _handles[key]
    return s["handle"]


def _own(s):
    c, r = s["case"], _handle(s)
    if c["op"] == "norm":
        r.layer_norm(s["x"], s["y"], s["gamma"], s["beta"], EPS, s["mean"], s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if c["op"] == "norm_grad":
        if "work" not in s:                                    # a program's workspace
            s["work"] = r.layer_norm_grad_work(c["rows"], c["width"])
        r.layer_norm_grad(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["dx"], s["dgamma"], s["dbeta"], s["work"])
        return (s["dx"], s["dgamma"], s["dbeta"]) if c["affine"] else (s["dx"],)
    if c["op"] == "dropout":
        r.dropout(s["x"], s["y"], c["p"], s["seed"], s["call"], residual=s["residual"])
        if not c["grad"]:
            return (s["y"],)
        r.dropout_grad(s["dy"], s["dx"], c["p"], s["seed"], s["call"])
        return s["y"], s["dx"]
    if "work" not in s:
        s["work"] = r.expert_layer_work(c["rows"], c["width"], c["hidden"], c["experts"], c["k"])
    r.expert_layer(s["x"], s["router"], s["up"], s["down"], s["y"], s["w"], s["ids"], s["work"], gated=c["gated"], over_chosen=c["chosen"])
    return s["y"], s["w"], s["ids"]


def run(s):
    return _own(s) if own else _plain(s)


def _expected_experts(c):
    """How many of the experts are asked for, on average over even choices."""
    asked = c["k"] / c["experts"] * (1.0 - c["barred"])
    return c["experts"] * (1.0 - (1.0 - asked) ** c["rows"])


def work(c):
    size = BYTES[c["dtype"]]
    T, D = c["rows"], c["width"]
    if c["op"] in ("norm", "norm_grad"):
        params = D * BYTES[c["params"]] if c["affine"] else 0
        if c["op"] == "norm":
            return {"bytes": 2 * T * D * size + 8 * T + 2 * params, "flops": 8 * T * D}
        return {"bytes": 3 * T * D * size + 8 * T + params + (8 * D if c["affine"] else 0), "flops": 14 * T * D}
    if c["op"] == "dropout":
        return {"bytes": (5 if c["grad"] else 3) * T * D * size, "flops": (5 if c["grad"] else 3) * T * D}
    E, H, k = c["experts"], c["hidden"], c["k"]
    rows_up = (2 if c["gated"] else 1) * H
    one = (rows_up + H) * D
    router = 0 if c["barred"] else E * D
    return {"bytes": size * (_expected_experts(c) * one + router + 2 * T * D) + 8 * T * k,
            "flops": 2 * T * (k * (1.0 - c["barred"]) * one + router)}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_kept(c, seed, call):
    """The elements that stay, by the generator's definition on 64-bit unsigned numbers."""
    T, D = c["rows"], c["width"]
    groups = (D + 7) // 8
    ctr = np.empty((4, T * groups), np.uint64)
    ctr[0], ctr[1] = np.tile(np.arange(groups), T), np.repeat(np.arange(T), groups)
    ctr[2], ctr[3] = call % (1 << 32), call >> 32
    key = [seed % (1 << 32), seed >> 32]
    mask, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = np.stack([(b >> half) ^ ctr[1] ^ np.uint64(key[0]), b & mask, (a >> half) ^ ctr[3] ^ np.uint64(key[1]), a & mask])
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    bits = np.ascontiguousarray(ctr.T.astype("<u4")).view("<u2").reshape(T, groups * 8)[:, :D]
    return torch.from_numpy(bits >= round(c["p"] * 65536))


def exact(c, seed):
    s = prepare(c, seed)
    T, D = c["rows"], c["width"]
    dev = s["x"].device
    if c["op"] in ("norm", "norm_grad"):
        out = []
        dgamma, dbeta = torch.zeros(D, dtype=torch.float64, device=dev), torch.zeros(D, dtype=torch.float64, device=dev)
        step = max(1, (1 << 24) // D)
        for a in range(0, T, step):
            x = s["x"][a:a + step].double()
            if c["op"] == "norm":
                var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
                rstd = 1.0 / torch.sqrt(var + EPS)
                y = (x - mean) * rstd
                if c["affine"]:
                    y = torch.addcmul(s["beta"].double(), y, s["gamma"].double())
                out.append((y, mean.squeeze(1), rstd.squeeze(1)))
                continue
            dy, r = s["dy"][a:a + step].double(), s["rstd"][a:a + step].double()
            x = torch.einsum("td,t->td", x - s["mean"][a:a + step].double()[:, None], r)
            g = dy * s["gamma"].double() if c["affine"] else dy
            along = torch.einsum("td,td->t", g, x) / D
            out.append(((g - g.sum(1)[:, None] / D - along[:, None] * x) * r[:, None],))
            dgamma += torch.einsum("td,td->d", dy, x)
            dbeta += dy.sum(0)
        out = tuple(torch.cat(part) for part in zip(*out))
        return out + (dgamma, dbeta) if c["op"] == "norm_grad" and c["affine"] else out
    if c["op"] == "dropout":
        kept = _exact_kept(c, s["seed"], s["call"]).to(dev)
        scale = kept.double() / (1.0 - min(round(c["p"] * 65536), 65535) / 65536)
        y = torch.addcmul(s["residual"].double(), s["x"].double(), scale)
        return (y, s["dy"].double() * scale) if c["grad"] else (y,)
    H, E, k = c["hidden"], c["experts"], c["k"]
    x = s["x"].double()
    if s["router"] is not None:
        logits = torch.einsum("td,ed->te", x, s["router"].double())
        v, ids = logits.topk(k, dim=1)
        w = torch.exp(v - torch.logsumexp(v if c["chosen"] else logits, 1, keepdim=True))
    else:
        w, ids = s["w"].double(), s["ids"].long()
    y = torch.zeros((T, D), dtype=torch.float64, device=dev)
    for e in range(E):
        rows, j = torch.nonzero(ids == e, as_tuple=True)
        if rows.numel():
            both = x[rows] @ s["up"][e].double().t()
            h = torch.nn.functional.silu(both[:, :H]) * both[:, H:] if c["gated"] else torch.relu(both)
            y.index_add_(0, rows, (h @ s["down"][e].double().t()) * w[rows, j][:, None])
    return y, w, None
