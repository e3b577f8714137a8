"""The work the dense operators are measured on: products with an epilogue, routing, experts and clipping.

A user of this library who has dense rows (document embeddings, hidden states) scores them against a map's units, routes
each row to its best few units, runs the units' experts on it, and trains these experts. The cases are calls of the entry
points of ``paper_2608_24067_amd.dense`` over the sizes such programs have: a single row in a service's loop, a few rows,
a prompt or mini-batch, a training step. Maps have 8 x 8 to 75 x 75 units, as in this library's tests and benchmark;
widths are generic.
"""
from __future__ import annotations

import math

import torch

own = False  # False: run() computes the plain forms; True: run() calls the library

# What a case holds:
#   kind    "linear" (product, bias, activation, residual), "route", "experts" or "clip"
#   train   forward and backward in one pass (a training step's share of the operator)
#   dtype   the rows' and weights' type (clip: "mixed" draws a type for each tensor)
#   linear  N rows, K features, M units or columns; act; res (with a residual); scores: fp32 result with an fp32 bias
#   route   N rows, E units, k taken; score, renorm, groups, group_top, bias; closed: share of closed (row, unit) pairs
#   experts N rows, D wide, F inner width, E experts, k a row; skew: exponent of the experts' popularity; empty: share
#           of rows that no expert takes
#   clip    n tensors of about `each` elements, sizes spread by a factor of `spread`


def listed():
    return [
        # One row's best units on an 8 x 8 map, in a service's loop.
        dict(name="route_one", kind="route", train=False, dtype="float32", N=1, E=64, k=2, score="softmax", renorm=True,
             groups=1, group_top=1, bias=False, closed=0.0),
        # A prompt's rows over 256 units in 8 regions, four of them open to a row, balanced by a bias.
        dict(name="route_regions", kind="route", train=False, dtype="bfloat16", N=16411, E=256, k=8, score="sigmoid",
             renorm=True, groups=8, group_top=4, bias=True, closed=0.0),
        # A training step's routing over an odd number of units, a part of them closed to each row, some rows to all.
        dict(name="route_train", kind="route", train=True, dtype="float32", N=30011, E=1000, k=4, score="softmax",
             renorm=False, groups=1, group_top=1, bias=False, closed=0.3),
        # One dense row scored against a 64 x 64 map.
        dict(name="scores_one_64", kind="linear", train=False, dtype="float16", N=1, K=1024, M=4096, act="none",
             res=False, scores=True),
        # A mini-batch of odd width scored against a 75 x 75 map: no row of the codebook starts aligned.
        dict(name="scores_75", kind="linear", train=False, dtype="float16", N=2011, K=1003, M=5625, act="none",
             res=False, scores=True),
        # A layer's share of a training step: product, bias, activation and residual, and its three gradients.
        dict(name="linear_train", kind="linear", train=True, dtype="bfloat16", N=8192, K=2048, M=4096, act="gelu",
             res=True, scores=False),
        # A single token through two of 64 experts.
        dict(name="experts_token", kind="experts", train=False, dtype="bfloat16", N=1, D=1024, F=4096, E=64, k=2,
             act="silu", skew=0.5, empty=0.0),
        # Some tens of tokens, which reach most experts with a row or two each.
        dict(name="experts_few", kind="experts", train=False, dtype="float16", N=33, D=1024, F=2048, E=32, k=4,
             act="gelu", skew=0.5, empty=0.0),
        # A prompt through 16 experts of uneven popularity.
        dict(name="experts_prompt", kind="experts", train=False, dtype="bfloat16", N=16384, D=2048, F=4096, E=16, k=2,
             act="silu", skew=0.5, empty=0.0),
        # A training step of 32 experts, ragged everywhere, some rows taken by none.
        dict(name="experts_train", kind="experts", train=True, dtype="bfloat16", N=10007, D=1000, F=2048, E=32, k=2,
             act="gelu", skew=0.7, empty=0.01),
        # A small model's gradients: latency.
        dict(name="clip_small", kind="clip", train=True, dtype="float32", n=12, each=2000, spread=50),
        # Every gradient of a larger model, three types mixed.
        dict(name="clip_large", kind="clip", train=True, dtype="mixed", n=40, each=9000000, spread=200),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A width: three in five a multiple of 64, the others any number."""
    v = _log_int(rng, lo, hi)
    v = max(64, v // 64 * 64) if rng.random() < 0.6 else v
    return v + 64 if v == 3072 else v


def draw(rng):
    """One more case: any kind, sizes spread over their ranges on a logarithmic scale."""
    kind = rng.choice(["linear", "route", "experts", "experts", "clip"])
    train = rng.random() < 0.5
    dtype = rng.choice(["float16", "bfloat16"])
    if kind == "linear":
        K, M = _width(rng, 64, 4096), _width(rng, 64, 5625)
        N = _log_int(rng, 1, min(16384, 6e10 / (K * M)))
        scores = not train and rng.random() < 0.5
        return dict(kind=kind, train=train, dtype=dtype, N=N, K=K, M=M,
                    act="none" if scores else rng.choice(["none", "relu", "gelu", "silu"]),
                    res=not scores and rng.random() < 0.5, scores=scores)
    if kind == "route":
        groups = rng.choice([1, 1, 4, 8])
        E = groups * max(2, _log_int(rng, 16, 2048) // groups)
        top = rng.randint(max(1, groups // 2), groups)
        return dict(kind=kind, train=train, dtype=rng.choice(["float32", dtype]), N=_log_int(rng, 1, 3.2e7 / E), E=E,
                    k=min(rng.choice([1, 2, 4, 8]), E // groups), score=rng.choice(["softmax", "sigmoid"]),
                    renorm=rng.random() < 0.5, groups=groups, group_top=top, bias=rng.random() < 0.5,
                    closed=rng.choice([0.0, 0.3]))
    if kind == "experts":
        D, F, E = _width(rng, 256, 2048), _width(rng, 256, 4096), rng.choice([4, 8, 13, 16, 32, 64])
        k = rng.choice([1, 2, 4])
        most = (5e10 if train else 1.2e11) / (k * D * F)
        return dict(kind=kind, train=train, dtype=dtype, N=_log_int(rng, 1, min(16384, most)), D=D, F=F, E=E, k=k,
                    act=rng.choice(["relu", "gelu", "silu"]), skew=rng.choice([0.0, 0.5, 1.0]),
                    empty=rng.choice([0.0, 0.02]))
    n = rng.randint(1, 60)
    return dict(kind=kind, train=True, dtype=rng.choice(["float32", "bfloat16", "float16", "mixed"]), n=n,
                each=_log_int(rng, 100, 3e8 / n), spread=rng.choice([1, 20, 200]))


# ------------------------------------------------------------------ inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, device="cuda", generator=g).mul_(scale).to(dtype)


def _clip_sizes(case):
    """The tensors' sizes: `each` on average (over their logarithm), spread evenly, the sizes odd as they fall."""
    n, s = case["n"], math.log(case["spread"])
    return [max(1, int(case["each"] * math.exp(s * ((i * 7 % n + 0.5) / n - 0.5)))) for i in range(n)]


def _clip_types(case):
    kinds = [torch.float32, torch.bfloat16, torch.float16]
    return [kinds[i % 3] if case["dtype"] == "mixed" else getattr(torch, case["dtype"]) for i in range(case["n"])]


def prepare(case, seed):
    g, s = _generator(seed), {"case": case}
    dt = getattr(torch, case["dtype"]) if case["dtype"] != "mixed" else None
    if case["kind"] == "linear":
        N, K, M = case["N"], case["K"], case["M"]
        s["x"] = _normal(g, N, K, dtype=dt)
        s["W"] = _normal(g, K, M, dtype=dt, scale=K ** -0.5)
        if case["scores"]:  # -|w|^2 / 2: the score x.w - |w|^2 / 2 ranks units as their distance does
            s["bias"] = -0.5 * s["W"].float().square().sum(0)
        else:
            s["bias"] = _normal(g, M, dtype=dt, scale=0.1)
        s["res"] = _normal(g, N, M, dtype=dt) if case["res"] else None
        s["y"] = torch.empty(N, M, dtype=torch.float32 if case["scores"] else dt, device="cuda")
        if case["train"]:
            s["dy"] = _normal(g, N, M, dtype=dt)
            s["pre"] = torch.empty(N, M, dtype=dt, device="cuda") if case["act"] != "none" else None
            s["grads"] = tuple(torch.empty_like(s[n]) for n in ("x", "W", "bias"))
            s["scratch"] = torch.empty(N * M * 2 + (1 << 24), dtype=torch.uint8, device="cuda")
    elif case["kind"] == "route":
        N, E, k = case["N"], case["E"], case["k"]
        s["logits"] = _normal(g, N, E, dtype=dt, scale=1.5)
        if case["closed"]:
            shut = torch.rand(N, E, device="cuda", generator=g) < case["closed"]
            shut |= torch.rand(N, 1, device="cuda", generator=g) < 0.01  # rows that every unit is closed to
            s["logits"].masked_fill_(shut, -math.inf)
        s["bias"] = _normal(g, E, scale=0.3) if case["bias"] else None
        s["idx"] = torch.empty(N, k, dtype=torch.int32, device="cuda")
        s["w"] = torch.empty(N, k, dtype=dt, device="cuda")
        s["counts"] = torch.empty(E, dtype=torch.int32, device="cuda")
        if case["train"]:
            s["dw"] = _normal(g, N, k, dtype=dt)
            s["dlogits"] = torch.empty(N, E, dtype=dt, device="cuda")
    elif case["kind"] == "experts":
        N, D, F, E, k = (case[n] for n in ("N", "D", "F", "E", "k"))
        s["x"] = _normal(g, N, D, dtype=dt)
        s["W1"], s["b1"] = _normal(g, E, D, F, dtype=dt, scale=D ** -0.5), _normal(g, E, F, dtype=dt, scale=0.1)
        s["W2"], s["b2"] = _normal(g, E, F, D, dtype=dt, scale=F ** -0.5), _normal(g, E, D, dtype=dt, scale=0.1)
        liking = -case["skew"] * torch.arange(1, E + 1, device="cuda").float().log()
        noise = -(-torch.rand(N, E, device="cuda", generator=g).clamp_(1e-7, 1 - 1e-7).log()).log()
        s["idx"] = (liking + noise).topk(min(k, E)).indices.int()
        if case["empty"]:
            s["idx"][torch.rand(N, device="cuda", generator=g) < case["empty"]] = -1
        w = torch.rand(N, k, device="cuda", generator=g) + 0.2
        s["w"] = (w / w.sum(1, keepdim=True)).to(dt)
        s["most"] = max(1, int(torch.bincount(s["idx"].reshape(-1).long() + 1, minlength=E + 1)[1:].max()))
        s["res"] = s["x"]
        s["out"] = torch.empty(N, D, dtype=dt, device="cuda")
        if case["train"]:
            s["dout"] = _normal(g, N, D, dtype=dt)
            s["grads"] = tuple(torch.empty_like(s[n]) for n in ("x", "w", "W1", "b1", "W2", "b2"))
        P = N * k  # scratch: the pairs' inner rows and results, and the order of the pairs
        s["scratch"] = torch.empty(P * (8 * F + 8 * D) + 64 * (P + N) + (1 << 25), dtype=torch.uint8, device="cuda")
    else:
        s["grads"] = [_normal(g, n, scale=0.01).to(t) for n, t in zip(_clip_sizes(case), _clip_types(case))]
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
        s["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
        s["max_norm"] = 1.0
        s["scratch"] = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------ the plain forms


def _act(a, z):
    """The activation and its derivative at z."""
    if a == "none":
        return z, torch.ones_like(z)
    if a == "relu":
        return z * (z > 0), (z > 0).to(z.dtype)
    if a == "silu":
        q = 1 / (1 + (-z).exp())
        return z * q, q * (1 + z * (1 - q))
    q = 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
    return z * q, q + z * (-0.5 * z * z).exp() * (2 * math.pi) ** -0.5


def _plain_linear(s, case):
    x, W, dt = s["x"].float(), s["W"].float(), s["x"].dtype
    y, slope = _act(case["act"], x @ W + s["bias"].float())
    y = (y + s["res"].float() if case["res"] else y).to(s["y"].dtype)
    if not case["train"]:
        return y
    dz = s["dy"].float() * slope
    return y, (dz @ W.t()).to(dt), (x.t() @ dz).to(dt), dz.sum(0).to(s["bias"].dtype)


def _plain_route(s, case):
    k, E, dt = case["k"], case["E"], s["logits"].dtype
    l = s["logits"].float()
    key = l + s["bias"] if case["bias"] else l
    shut = (key == -math.inf) | torch.isnan(key)
    if case["groups"] > 1:
        best = key.masked_fill(shut, -math.inf).reshape(-1, case["groups"], E // case["groups"]).amax(2)
        rank = best.sort(dim=1, descending=True, stable=True).indices
        kept = torch.zeros_like(best).scatter_(1, rank[:, :case["group_top"]], 1.0)
        key = key.masked_fill(kept.repeat_interleave(E // case["groups"], 1) == 0, -math.inf)
    first = key.masked_fill(shut, -math.inf).sort(dim=1, descending=True, stable=True)
    none = first.values[:, :k] == -math.inf
    at = first.indices[:, :k]
    if case["score"] == "softmax":
        z = (l - l.masked_fill(shut, -math.inf).amax(1, keepdim=True)).exp().masked_fill(shut, 0.0)
        p = z / z.sum(1, keepdim=True).clamp_min(1e-30)
    else:
        p = (1 / (1 + (-l).exp())).masked_fill(shut, 0.0)
    took = p.gather(1, at).masked_fill(none, 0.0)
    total = took.sum(1, keepdim=True).clamp_min(1e-30)
    w = took / total if case["renorm"] else took
    idx = at.masked_fill(none, -1).int()
    counts = torch.zeros(E + 1, dtype=torch.int32, device=l.device).index_add_(
        0, idx.reshape(-1).long() + 1, torch.ones(idx.numel(), dtype=torch.int32, device=l.device))[1:]
    if not case["train"]:
        return idx, w.to(dt), counts
    dw = s["dw"].float().masked_fill(none, 0.0)
    if case["renorm"]:
        dw = (dw - (dw * w).sum(1, keepdim=True)) / total
    dp = torch.zeros_like(l).scatter_add_(1, at, dw.masked_fill(none, 0.0))
    dl = p * (dp - (dp * p).sum(1, keepdim=True)) if case["score"] == "softmax" else dp * p * (1 - p)
    return idx, w.to(dt), counts, dl.to(dt)


def _plain_experts(s, case):
    N, D, E, k, dt = case["N"], case["D"], case["E"], case["k"], s["x"].dtype
    x, w, flat = s["x"].float(), s["w"].float().reshape(-1, 1), s["idx"].reshape(-1).long()
    row = torch.arange(N * k, device=x.device) // k
    shut = (flat < 0).unsqueeze(1)
    if N * k <= E and not case["train"]:  # a few rows: only the weights they meet
        e = flat.clamp_min(0)
        h, _ = _act(case["act"], torch.bmm(x[row].unsqueeze(1), s["W1"][e].float()) + s["b1"][e].float().unsqueeze(1))
        y = (torch.bmm(h, s["W2"][e].float()).squeeze(1) + s["b2"][e].float()).masked_fill(shut, 0.0)
        return (s["res"].float() + (w * y).reshape(N, k, D).sum(1)).to(dt)
    most = s["most"]  # every expert's rows in a block of its own
    order = flat.sort(stable=True)
    start = torch.zeros(E + 2, dtype=torch.long, device=x.device)
    start[1:] = torch.zeros(E + 1, dtype=torch.long, device=x.device).index_add_(0, flat + 1, torch.ones_like(flat)).cumsum(0)
    place = torch.empty_like(flat)
    place[order.indices] = torch.arange(N * k, device=x.device) - start[order.values + 1]
    slot = torch.where(flat < 0, E * most, flat * most + place)

    def spread(v):  # a value for each pair to its expert's block; the last place takes what no expert has
        return torch.zeros(E * most + 1, v.shape[1], device=x.device).index_copy_(0, slot, v)[:-1].reshape(E, most, -1)

    def back(v):  # and from there
        return v.reshape(E * most, -1)[slot.clamp_max(E * most - 1)].masked_fill(shut, 0.0)

    W1, W2 = s["W1"].float(), s["W2"].float()
    xs = spread(x[row])
    h, slope = _act(case["act"], torch.bmm(xs, W1) + s["b1"].float().unsqueeze(1))
    y = back(torch.bmm(h, W2) + s["b2"].float().unsqueeze(1))
    out = (s["res"].float() + (w * y).reshape(N, k, D).sum(1)).to(dt)
    if not case["train"]:
        return out
    dout = s["dout"].float()[row]
    dys = spread(w * dout)
    dz = torch.bmm(dys, W2.transpose(1, 2)) * slope
    dx = back(torch.bmm(dz, W1.transpose(1, 2))).reshape(N, k, D).sum(1)
    return (out, dx.to(dt), (y * dout).sum(1).reshape(N, k).to(dt), torch.bmm(xs.transpose(1, 2), dz).to(dt),
            dz.sum(1).to(dt), torch.bmm(h.transpose(1, 2), dys).to(dt), dys.sum(1).to(dt))


def _plain_clip(s, case):
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    scale = (s["max_norm"] / norm).clamp_max(1.0)
    return [norm.reshape(1)] + [(t.float() * scale).to(t.dtype) for t in s["grads"]]


# ------------------------------------------------------------------ the library's calls


def _routing(case):
    return {n: case[n] for n in ("score", "renorm", "groups", "group_top")}


def _own(s, case):
    import paper_2608_24067_amd.dense as dense

    if case["kind"] == "linear":
        pre = s["pre"] if case["train"] else None
        y = dense.linear(s["x"], s["W"], s["bias"], residual=s["res"], act=case["act"], out=s["y"], pre=pre)
        if not case["train"]:
            return y
        return (y,) + dense.linear_bwd(s["x"], s["W"], s["dy"], pre=pre, act=case["act"], out=s["grads"],
                                       workspace=s["scratch"])
    if case["kind"] == "route":
        got = dense.route(s["logits"], case["k"], bias=s["bias"], out=(s["idx"], s["w"]), counts=s["counts"],
                          **_routing(case))
        if not case["train"]:
            return got + (s["counts"],)
        return got + (s["counts"], dense.route_bwd(s["logits"], s["idx"], s["dw"], bias=s["bias"], out=s["dlogits"],
                                                   **_routing(case)))
    if case["kind"] == "experts":
        out = dense.experts(s["x"], s["idx"], s["w"], s["W1"], s["b1"], s["W2"], s["b2"], act=case["act"],
                            residual=s["res"], out=s["out"], keep=case["train"], workspace=s["scratch"])
        if not case["train"]:
            return out
        return (out,) + dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], s["dout"],
                                          act=case["act"], out=s["grads"], workspace=s["scratch"])
    out, norm = dense.clip(s["grads"], s["max_norm"], out=s["out"], norm=s["norm"], workspace=s["scratch"])
    return [norm] + list(out)


_PLAIN = {"linear": _plain_linear, "route": _plain_route, "experts": _plain_experts, "clip": _plain_clip}


def run(state):
    case = state["case"]
    return _own(state, case) if own else _PLAIN[case["kind"]](state, case)


def work(case):
    """What one pass cannot do without: every input read once, every output written once, every product term."""
    size = 4 if case["dtype"] == "float32" else 2
    t = 1 if case["train"] else 0
    if case["kind"] == "linear":
        N, K, M = case["N"], case["K"], case["M"]
        out = (4 if case["scores"] else size) * N * M
        moved = size * (N * K + K * M + M + (N * M if case["res"] else 0)) + out
        return {"bytes": moved + t * size * (N * M + N * K + K * M + M), "flops": 2 * N * K * M * (1 + 2 * t)}
    if case["kind"] == "route":
        N, E, k = case["N"], case["E"], case["k"]
        return {"bytes": size * N * E * (1 + t) + N * k * (4 + size * (1 + t)) + 4 * E, "flops": 8 * N * E * (1 + t)}
    if case["kind"] == "experts":
        N, D, F, E, k = (case[n] for n in ("N", "D", "F", "E", "k"))
        met = E * (1 - (1 - 1 / E) ** (N * k)) if N * k > 1 else 1  # experts that any row meets, taken evenly
        weights = met * (2 * D * F + D + F)
        return {"bytes": size * (weights + t * (E * (2 * D * F + D + F)) + N * D * (2 + 2 * t) + N * k * (1 + t)) + 4 * N * k,
                "flops": 4 * N * k * (1 - case["empty"]) * D * F * (1 + 2 * t)}
    sizes, types = _clip_sizes(case), _clip_types(case)
    moved = sum(n * (4 if t == torch.float32 else 2) for n, t in zip(sizes, types))
    return {"bytes": 2 * moved, "flops": 3 * sum(sizes)}


# ------------------------------------------------------------------ the definitions in 64 bits


def _wide_act(a, z):
    if a == "relu":
        return torch.relu(z)
    if a == "silu":
        return z * torch.sigmoid(z)
    return z * torch.special.ndtr(z) if a == "gelu" else z


def _wide(t, grad=True):
    return t.double().requires_grad_(grad)


def exact(case, seed):
    s, train = prepare(case, seed), case["train"]
    with torch.enable_grad():
        if case["kind"] == "linear":
            x, W, b = (_wide(s[n], train) for n in ("x", "W", "bias"))
            y = _wide_act(case["act"], torch.addmm(b, x, W))
            y = y + s["res"].double() if case["res"] else y
            if not train:
                return y
            return (y.detach(),) + torch.autograd.grad(y, (x, W, b), s["dy"].double())
        if case["kind"] == "route":
            return _exact_route(s, case)
        if case["kind"] == "experts":
            return _exact_experts(s, case)
    total = math.sqrt(math.fsum(float(t.double().pow(2).sum()) for t in s["grads"]))
    scale = min(1.0, s["max_norm"] / total)
    return [torch.tensor([total], dtype=torch.float64)] + [t.double() * scale for t in s["grads"]]


def _exact_route(s, case):
    """The k largest keys one after the other (the key, logit + bias, is held in fp32 by definition)."""
    N, E, k, G = case["N"], case["E"], case["k"], case["groups"]
    l = s["logits"].double().requires_grad_(case["train"])
    key = s["logits"].double().detach()
    key = (key + s["bias"].double()).float() if case["bias"] else key.float()
    key = torch.where(torch.isnan(key), -math.inf, key)
    open_ = key > -math.inf
    number = torch.arange(E, device=key.device).expand(N, E)
    if G > 1:
        region, size = number // (E // G), E // G
        left, keep = key.clone(), torch.zeros(N, E, dtype=torch.bool, device=key.device)
        for _ in range(case["group_top"]):
            top = left.max(1, keepdim=True).values
            which = torch.where(left == top, number, E).min(1, keepdim=True).values // size
            mine = region == which
            keep |= mine
            left = left.masked_fill(mine, -math.inf)
        key = key.masked_fill(~keep, -math.inf)
    idx = torch.empty(N, k, dtype=torch.long, device=key.device)
    for j in range(k):
        top = key.max(1, keepdim=True).values
        at = torch.where(key == top, number, E).min(1, keepdim=True).values
        idx[:, j:j + 1] = torch.where(top > -math.inf, at, -1)
        key = key.masked_fill(number == at, -math.inf)
    some = idx >= 0
    if case["score"] == "softmax":
        z = l.masked_fill(~open_, -1e300)
        p = torch.softmax(z, 1)
    else:
        p = torch.sigmoid(l.masked_fill(~open_, -1e300))
    w = p.gather(1, idx.clamp_min(0)) * some
    if case["renorm"]:
        w = w / (w.sum(1, keepdim=True) + (~some.any(1, keepdim=True)).double())
    counts = torch.bincount(idx[some], minlength=E)
    if not case["train"]:
        return idx, w.detach(), counts
    return idx, w.detach(), counts, torch.autograd.grad(w, l, s["dw"].double())[0]


def _exact_experts(s, case):
    """Expert after expert on the rows that it takes."""
    N, D, E, train = case["N"], case["D"], case["E"], case["train"]
    x, w = _wide(s["x"], train), _wide(s["w"], train)
    out, dx = torch.zeros(N, D, dtype=torch.float64, device="cuda"), torch.zeros(N, D, dtype=torch.float64, device="cuda")
    dw, parts = torch.zeros_like(w, requires_grad=False), []
    for e in range(E):
        rows, slots = (s["idx"] == e).nonzero(as_tuple=True)
        if not train and not rows.numel():
            continue
        own_ = [_wide(s[n][e], train) for n in ("W1", "b1", "W2", "b2")]
        xe, we = x.detach()[rows].requires_grad_(train), w.detach()[rows, slots].requires_grad_(train)
        y = we.unsqueeze(1) * (_wide_act(case["act"], xe @ own_[0] + own_[1]) @ own_[2] + own_[3])
        out.index_add_(0, rows, y.detach())
        if train:
            got = torch.autograd.grad(y, [xe, we] + own_, s["dout"].double()[rows])
            dx.index_add_(0, rows, got[0])
            dw[rows, slots] = got[1]
            parts.append([t.to(torch.float32 if t.dim() == 2 else torch.float64) for t in got[2:]])
    out = out + s["res"].double()
    if not train:
        return out
    return (out, dx, dw) + tuple(torch.stack([p[i] for p in parts]) for i in range(4))
