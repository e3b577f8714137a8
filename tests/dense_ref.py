"""Plain 64-bit forms of the dense operators (include/som_dense.h), on the CPU, and the error bounds the tests use.

Bounds. A result rounded to a type of p significant bits is off by at most u |y|, u = 2^-p, plus half the smallest
subnormal. A product summed in fp32 in any order over n terms is off by at most n 2^-24 times the sum of the terms'
magnitudes (twice that is taken: the products of 16-bit values are exact in fp32, each addition rounds once). An
activation's slope is at most 1.13, and the fp32 activations are good to 2^-20 of max(|z|, 1), which covers erf and exp
at a few units in the last place.
"""
import math

import torch

U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
LIP = 1.13


def wide(t):
    return t.detach().cpu().double()


def act(name, z):
    if name == "relu":
        return torch.relu(z)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
    return z


def slope(name, z):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def curve(name):
    """The largest second derivative: how far a rounded z moves the slope (relu's jump is left to the caller)."""
    return {"none": 0.0, "relu": 0.0, "gelu": 0.8, "silu": 0.5}[name]


def check(got, ref, bound, what):
    """|got - ref| within the rounding of got's type and the given bound of what was computed before it."""
    assert tuple(got.shape) == tuple(ref.shape), f"{what}: {tuple(got.shape)} vs {tuple(ref.shape)}"
    got, dt = wide(got), got.dtype
    lim = U[dt] * (ref.abs() + bound) + bound + TINY[dt]
    bad = ~((got - ref).abs() <= lim)
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst "
                                 f"{float(((got - ref).abs() - lim)[bad].max()) if bad.any() else 0:.3g}, first at "
                                 f"{bad.nonzero()[0].tolist()}: {float(got[bad][0])} vs {float(ref[bad][0])}")


def sums(n, magnitude):
    """The bound of an fp32 sum over n terms."""
    return 2 * (n + 2) * 2.0 ** -24 * magnitude


def route(logits, k, bias=None, score="softmax", renorm=True, groups=1, group_top=0):
    """(idx, weights in 64 bits) row by row."""
    l32 = logits.detach().cpu().float()
    N, E = l32.shape
    key = l32 + (bias.cpu() if bias is not None else 0.0)
    idx = torch.full((N, k), -1, dtype=torch.int32)
    w = torch.zeros(N, k, dtype=torch.float64)
    width = E // groups
    for n in range(N):
        open_ = [e for e in range(E) if float(l32[n, e]) > -math.inf and float(key[n, e]) > -math.inf]
        ranked = sorted(open_, key=lambda e: (-float(key[n, e]), e))
        if groups > 1:
            best = []
            for e in ranked:  # a group's best unit is its first in the ranking
                if e // width not in [g for g, _ in best]:
                    best.append((e // width, float(key[n, e])))
            best.sort(key=lambda g: (-g[1], g[0]))
            kept = {g for g, _ in best[:group_top or groups]}
            ranked = [e for e in ranked if e // width in kept]
        taken = ranked[:k]
        if not taken:
            continue
        idx[n, :len(taken)] = torch.tensor(taken, dtype=torch.int32)
        v = l32[n].double().clamp(max=torch.finfo(torch.float32).max)
        if score == "sigmoid":
            s = torch.sigmoid(v[taken])
            if renorm:  # scaled alike, so that not all underflow: exp(log sigmoid - its largest)
                s = torch.nn.functional.logsigmoid(v[taken])
                s = (s - s.max()).exp()
        else:
            among = taken if renorm else open_
            top = max(float(v[e]) for e in among)
            z = sum(math.exp(float(v[e]) - top) for e in among)
            s = torch.tensor([math.exp(float(v[e]) - top) / z for e in taken], dtype=torch.float64)
        if renorm:
            s = s / s.sum()
        w[n, :len(taken)] = s
    return idx, w


def route_grad(logits, idx, dw, bias=None, score="softmax", renorm=True):
    """The logits' gradient by autograd in 64 bits (the choice idx held fixed)."""
    l32 = logits.detach().cpu().float()
    key = l32 + (bias.cpu() if bias is not None else 0.0)
    open_ = (l32 > -math.inf) & (key > -math.inf)
    l = l32.double().clamp(max=torch.finfo(torch.float32).max).masked_fill(~open_, 0.0).requires_grad_(True)
    idx = idx.cpu().long()
    some = (idx >= 0) & (idx < l.shape[1])
    at = idx.clamp(0, l.shape[1] - 1)
    if score == "sigmoid":
        p = torch.sigmoid(l)
    else:
        z = l.masked_fill(~open_, -1e300)
        p = torch.softmax(z, 1)
    took = p.gather(1, at) * some * open_.gather(1, at)
    if renorm and score == "sigmoid":  # shares of exp(log sigmoid), which do not underflow
        took = torch.softmax(torch.nn.functional.logsigmoid(l).gather(1, at).masked_fill(
            ~(some & open_.gather(1, at)), -1e300), 1) * some
    elif renorm:
        total = took.sum(1, keepdim=True)
        took = torch.where(total > 0, took / torch.where(total > 0, total, torch.ones_like(total)), took)
    (g,) = torch.autograd.grad((took * wide(dw) * some).sum(), l)
    return g * open_
