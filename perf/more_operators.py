"""The work that layer norm, AdamW and the products with 4-bit matrices are measured on.

A user of this library who trains layers on a map's dense rows normalises the rows in front of a layer, and steps the
weights with the gradients that ``dense.clip`` leaves; who serves them holds codebooks and layers in 4 bits (microscaled:
blocks of 32 values share a power of two), and multiplies rows with them. The cases are calls of the entry points of
``paper_2608_24067_amd.dense`` over the sizes such programs have. Maps have 8 x 8 to 75 x 75 units, as in this library's
tests and benchmark; widths are generic.
"""
from __future__ import annotations

import math

import torch

own = False  # False: run() computes the plain forms; True: run() calls the library

# What a case holds:
#   kind   "norm" (layer norm), "step" (AdamW), "quantise" (to 4 bits, and back to the values they stand for) or "product"
#   norm   N rows, D features; x, y: the rows' and results' types; train: forward and backward; affine: "none", "weight"
#          or "both", held in wtype; add: another gradient of the rows that is added to theirs
#   step   n tensors of about `each` elements, sizes spread by a factor of `spread`; dtype of the parameters ("mixed": a
#          type for each), grad32: gradients in float32; bits of the states; master: float32 copies
#   quantise  N rows, K features of dtype; columns: a feature-major matrix [K, N] whose columns are quantised
#   product   N rows, K features, M columns of a 4-bit matrix; both: the rows are quantised too, within the pass; act;
#             res (with a residual); scores: float32 result


def listed():
    return [
        # One row in front of a layer, in a service's loop.
        dict(name="norm_one", kind="norm", N=1, D=2048, x="bfloat16", y="bfloat16", train=False, affine="both",
             wtype="bfloat16", add=False),
        # Rows of odd width, kept in 32 bits between layers, handed to a 16-bit product.
        dict(name="norm_odd", kind="norm", N=20011, D=1003, x="float32", y="float16", train=False, affine="both",
             wtype="float32", add=False),
        # A training step's share: forward and backward, the gradient around the layer added in the same pass.
        dict(name="norm_train", kind="norm", N=8192, D=4096, x="bfloat16", y="bfloat16", train=True, affine="both",
             wtype="float32", add=True),
        # A small model's step: latency.
        dict(name="step_small", kind="step", n=12, each=2000, spread=50, dtype="float32", grad32=True, bits=32,
             master=False),
        # 16-bit parameters with a float32 copy: what a larger model's step moves.
        dict(name="step_master", kind="step", n=40, each=2500000, spread=200, dtype="bfloat16", grad32=False, bits=32,
             master=True),
        # The states in 8 bits, the parameters' types mixed; what the states stand for comes back with them.
        dict(name="step_8bit", kind="step", n=60, each=1500000, spread=200, dtype="mixed", grad32=False, bits=8,
             master=False),
        # A prompt's rows to 4 bits, in front of a product of 4-bit operands.
        dict(name="quantise_rows", kind="quantise", N=16384, K=2048, dtype="bfloat16", columns=False),
        # A trained codebook of a 75 x 75 map to 4 bits: feature-major, odd both ways.
        dict(name="quantise_map", kind="quantise", N=5625, K=1003, dtype="float32", columns=True),
        # One dense row scored against a 64 x 64 map held in 4 bits.
        dict(name="product_one", kind="product", N=1, K=1024, M=4096, dtype="float16", both=False, act="none",
             res=False, scores=True),
        # Some tens of tokens through a layer held in 4 bits.
        dict(name="product_few", kind="product", N=33, K=2048, M=8192, dtype="bfloat16", both=False, act="gelu",
             res=False, scores=False),
        # A mini-batch of odd width scored against a 75 x 75 map held in 4 bits.
        dict(name="product_75", kind="product", N=2011, K=1003, M=5625, dtype="bfloat16", both=False, act="none",
             res=False, scores=True),
        # A prompt through a layer, its rows quantised on the way.
        dict(name="product_both", kind="product", N=8192, K=2048, M=4096, dtype="bfloat16", both=True, act="silu",
             res=True, scores=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def _width(rng, lo, hi):
    """A width: three in five a multiple of 64, the others any number."""
    v = _log_int(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.6 else v


def draw(rng):
    """One more case: any kind, sizes spread over their ranges on a logarithmic scale."""
    kind = rng.choice(["norm", "step", "quantise", "product", "product"])
    half = rng.choice(["float16", "bfloat16"])
    if kind == "norm":
        x, y = rng.choice([("float32", "float32"), ("float32", half), (half, half)])
        D, train = _width(rng, 16, 16384), rng.random() < 0.6
        return dict(kind=kind, N=_log_int(rng, 1, min(100000, 3e7 / D)), D=D, x=x, y=y, train=train,
                    affine=rng.choice(["none", "weight", "both", "both"]), wtype=rng.choice(["float32", y]),
                    add=train and rng.random() < 0.5)
    if kind == "step":
        n, bits = rng.randint(1, 100), rng.choice([8, 32])
        dtype = rng.choice(["float32", "bfloat16", "float16", "mixed"])
        return dict(kind=kind, n=n, each=_log_int(rng, 100, 8e7 / n), spread=rng.choice([1, 20, 200]), dtype=dtype,
                    grad32=rng.random() < 0.3, bits=bits, master=dtype != "float32" and rng.random() < 0.5)
    if kind == "quantise":
        K = _width(rng, 32, 8192)
        return dict(kind=kind, N=_log_int(rng, 1, min(100000, 3e7 / K)), K=K, dtype=rng.choice(["float32", half]),
                    columns=rng.random() < 0.5)
    K, M = _width(rng, 64, 4096), _width(rng, 64, 8192)
    both, scores = rng.random() < 0.5, rng.random() < 0.4
    return dict(kind=kind, N=_log_int(rng, 1, min(16384, 6e10 / (K * M))), K=K, M=M, dtype=half, both=both,
                act="none" if scores else rng.choice(["none", "relu", "gelu", "silu"]),
                res=not scores and rng.random() < 0.5, scores=scores)


# ------------------------------------------------------------------ inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(shape, device="cuda", generator=g).mul_(scale).to(dtype)


def _hidden(g, N, D, dtype):
    """Rows as layers leave them: features of unequal size, with means, a few much larger than the others."""
    x = torch.randn(N, D, device="cuda", generator=g)
    size = torch.randn(D, device="cuda", generator=g).mul_(0.5).exp_()
    large = torch.rand(D, device="cuda", generator=g) < 0.01
    mean = torch.randn(D, device="cuda", generator=g).mul_(0.5)
    return x.mul_(size * (1 + 15 * large)).add_(mean * (1 + 15 * large)).to(dtype)


def _sizes(case):
    """The tensors' sizes: `each` on average (over their logarithm), spread evenly, the sizes odd as they fall."""
    n, s = case["n"], math.log(case["spread"])
    return [max(1, int(case["each"] * math.exp(s * ((i * 7 % n + 0.5) / n - 0.5)))) for i in range(n)]


def _types(case):
    kinds = [torch.bfloat16, torch.float32, torch.float16]
    return [kinds[i % 3] if case["dtype"] == "mixed" else getattr(torch, case["dtype"]) for i in range(case["n"])]


def _flat(sizes, dtypes, device="cuda"):
    """A buffer for each type, and the tensors in it, each from a multiple of 256 elements on."""
    total = {}
    places = []
    for n, t in zip(sizes, dtypes):
        places.append(total.get(t, 0))
        total[t] = total.get(t, 0) + (n + 255) // 256 * 256
    flat = {t: torch.zeros(m, dtype=t, device=device) for t, m in total.items()}
    return list(flat.values()), [flat[t][p:p + n] for n, t, p in zip(sizes, dtypes, places)]


STEP = dict(step=1000, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, seed=20250)

SHARED = 32  # values of a block of 4-bit ones
BLOCK = 256  # values of a block of 8-bit states


def prepare(case, seed):
    g, s = _generator(seed), {"case": case}
    if case["kind"] == "norm":
        N, D, xt, yt, wt = case["N"], case["D"], *(getattr(torch, case[n]) for n in ("x", "y", "wtype"))
        s["x"] = _hidden(g, N, D, xt)
        s["weight"] = (1 + _normal(g, D, scale=0.2)).to(wt) if case["affine"] != "none" else None
        s["bias"] = _normal(g, D, dtype=wt, scale=0.2) if case["affine"] == "both" else None
        s["y"] = torch.empty(N, D, dtype=yt, device="cuda")
        if case["train"]:
            s["dy"] = _normal(g, N, D, dtype=yt)
            s["add"] = _normal(g, N, D, dtype=xt) if case["add"] else None
            s["stats"] = torch.empty(N, 2, dtype=torch.float64, device="cuda")
            s["grads"] = (torch.empty_like(s["x"]),) + tuple(
                torch.empty(D, dtype=wt, device="cuda") if s[n] is not None else None for n in ("weight", "bias"))
            s["scratch"] = torch.empty(64 * D * (16 + N // 64) + (1 << 24), dtype=torch.uint8, device="cuda")
    elif case["kind"] == "step":
        _prepare_step(s, case, g)
    elif case["kind"] == "quantise":
        N, K, dt = case["N"], case["K"], getattr(torch, case["dtype"])
        blocks = (K + SHARED - 1) // SHARED
        s["x"] = _normal(g, K, N, dtype=dt, scale=K ** -0.5) if case["columns"] else _hidden(g, N, K, dt)
        s["codes"] = torch.empty(N, blocks * 16, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(N, blocks, dtype=torch.uint8, device="cuda")
        s["values"] = torch.empty(*s["x"].shape, dtype=torch.float32 if dt == torch.float32 else torch.bfloat16,
                                  device="cuda")
    else:
        N, K, M, dt = case["N"], case["K"], case["M"], getattr(torch, case["dtype"])
        blocks = (K + SHARED - 1) // SHARED
        s["x"] = _hidden(g, N, K, dt)
        W = _normal(g, M, K, scale=K ** -0.5)
        s["W"] = _codes(W)  # laid out once, as a program that serves keeps it
        s["bias"] = -0.5 * _values(*s["W"], K).square().sum(1) if case["scores"] else _normal(g, M, dtype=dt, scale=0.1)
        s["res"] = _normal(g, N, M, dtype=dt) if case["res"] else None
        s["y"] = torch.empty(N, M, dtype=torch.float32 if case["scores"] else dt, device="cuda")
        s["codes"] = torch.empty(N, blocks * 16, dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(N, blocks, dtype=torch.uint8, device="cuda")
        s["scratch"] = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    return s


def _prepare_step(s, case, g):
    sizes, types = _sizes(case), _types(case)
    gtypes = [torch.float32] * len(sizes) if case["grad32"] else types
    s["flat_p"], s["params"] = _flat(sizes, types)
    _, s["grads"] = _flat(sizes, gtypes)
    f32, u8 = [torch.float32] * len(sizes), [torch.uint8] * len(sizes)
    s["flat_m"], s["m"] = _flat(sizes, f32)  # 8-bit states: the values they stand for come back here
    s["flat_v"], s["v"] = _flat(sizes, f32)
    if case["bits"] == 8:
        blocks = [(n + BLOCK - 1) // BLOCK for n in sizes]
        s["mc"], s["vc"] = _flat(sizes, u8)[1], _flat(sizes, u8)[1]
        s["ms"], s["vs"] = _flat(blocks, u8)[1], _flat(blocks, u8)[1]
    if case["master"]:
        s["flat_w"], s["master"] = _flat(sizes, f32)
    for i, p in enumerate(s["params"]):
        w = torch.randn(p.numel(), device="cuda", generator=g).mul_(0.05)
        p.copy_(w)
        if case["master"]:
            s["master"][i].copy_(w)
        # gradients as training gives them: their size differs from tensor to tensor and from stretch to stretch
        size = torch.randn((p.numel() + 63) // 64, device="cuda", generator=g).mul_(1.0).exp_().mul_(1e-3)
        size = size.repeat_interleave(64)[:p.numel()]
        m = torch.randn(p.numel(), device="cuda", generator=g).mul_(size).mul_(0.3)
        v = torch.rand(p.numel(), device="cuda", generator=g).add_(0.3).mul_(size).mul_(size)
        s["grads"][i].copy_(torch.randn(p.numel(), device="cuda", generator=g).mul_(size))
        if case["bits"] == 8:
            zero = torch.zeros(p.numel(), dtype=torch.int64, device="cuda")
            for x, codes, scales, signed in ((m, s["mc"][i], s["ms"][i], True), (v, s["vc"][i], s["vs"][i], False)):
                c, e = _codes8(x, signed, zero)
                codes.copy_(c)
                scales.copy_(e)
        else:
            s["m"][i].copy_(m)
            s["v"][i].copy_(v)


# ------------------------------------------------------------------ the plain forms


def _plain_norm(s, case):
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    c = x - mean
    c = c - c.mean(1, keepdim=True)
    r = (c.square().mean(1, keepdim=True) + 1e-5).rsqrt()
    h = c * r
    w = s["weight"].float() if s["weight"] is not None else torch.ones_like(h[0])
    y = h * w
    y = (y + s["bias"].float() if s["bias"] is not None else y).to(s["y"].dtype)
    if not case["train"]:
        return y
    dy = s["dy"].float()
    t = dy * w
    dx = r * (t - t.mean(1, keepdim=True) - h * (t * h).mean(1, keepdim=True))
    dx = dx + s["add"].float() if s["add"] is not None else dx
    dw = (dy * h).sum(0).to(s["weight"].dtype) if s["weight"] is not None else None
    db = dy.sum(0).to(s["bias"].dtype) if s["bias"] is not None else None
    return y, dx.to(s["x"].dtype), dw, db


def _power(e):
    """2^e in float32 for whole e from -126 to 127, by its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _scaled_by_power(x, e):
    """x 2^e, e in two halves so that neither leaves the range of float32."""
    half = torch.div(e, 2, rounding_mode="floor")
    return x * _power(half) * _power(e - half)


def _blocks8(x):
    n = x.numel()
    return torch.nn.functional.pad(x, (0, -n % BLOCK)).reshape(-1, BLOCK)


def _codes8(x, signed, random):
    """Codes and blocks' scales of 8-bit states: floating point with 3 bits behind the point and 4 bits of exponent (and
    a sign) or 5, relative to a power of two (the scale, less 127) at which the block's largest value is at most 1.875.
    `random`: 16 bits a value, below which the part that is rounded off is dropped."""
    bits = _blocks8(x).contiguous().view(torch.int32) & 0x7FFFFFFF
    e = ((bits.amax(1, keepdim=True) + 0xFFFFF) >> 23) - 127
    some = e >= -100
    e = torch.where(some, e, 0)
    y = _scaled_by_power(_blocks8(x).abs(), -e) * 2.0 ** (-112 if signed else -96)
    code = (y.view(torch.int32).long() + (_blocks8(random) << 4)) >> 20
    if signed:
        code = code.clamp_max(127) | ((_blocks8(x) < 0).long() << 7)
    else:
        code = torch.where(_blocks8(x) > 0, code.clamp(1, 255), 0)
    code = torch.where(some, code, 0).to(torch.uint8).reshape(-1)[:x.numel()]
    return code, torch.where(some, e + 127, 0).to(torch.uint8).reshape(-1)


def _values8(code, scale, signed):
    """What 8-bit states stand for."""
    c = code.to(torch.int32)
    size = ((c & 127 if signed else c) << 20).view(torch.float32) * 2.0 ** (112 if signed else 96)
    e = scale.to(torch.int32).sub_(127).repeat_interleave(BLOCK)[:c.numel()]
    size = _scaled_by_power(size, e)
    return torch.where(c >= 128, -size, size) if signed else size


def _mix(h):
    """Bits of 32-bit numbers (held in 64) spread over all of them."""
    h = h ^ (h >> 16)
    h = (h * 0xBB67AE85) & 0xFFFFFFFF
    h = h ^ (h >> 15)
    h = (h * 0x6A09E667) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _random(n, tensor):
    """32 bits for each value of a tensor, from the seed, the step and the places of both."""
    first = torch.tensor(STEP["seed"] + STEP["step"] * 0x9E3779B1 + tensor * 0x1F83D9AB, device="cuda") & 0xFFFFFFFF
    i = torch.arange(n, device="cuda")
    return _mix((i * 0x9E3779B1 + (i >> 32) * 0xA54FF53B + _mix(first)) & 0xFFFFFFFF)


def _plain_step(s, case):
    b1, b2, t, lr = STEP["beta1"], STEP["beta2"], STEP["step"], STEP["lr"]
    for i, p in enumerate(s["params"]):
        g = s["grads"][i].float()
        if case["bits"] == 8:
            m = _values8(s["mc"][i], s["ms"][i], True)
            v = _values8(s["vc"][i], s["vs"][i], False)
        else:
            m, v = s["m"][i], s["v"][i]
        m = m * b1 + g * (1 - b1)
        v = v * b2 + (g * g) * (1 - b2)
        w = s["master"][i] if case["master"] else p.float()
        w = w * (1 - lr * STEP["weight_decay"]) - (lr / (1 - b1 ** t)) * (
            m / (v.sqrt() * (1 - b2 ** t) ** -0.5 + STEP["eps"]))
        p.copy_(w)
        if case["master"]:
            s["master"][i].copy_(w)
        if case["bits"] == 8:
            r = _random(p.numel(), i)
            for x, codes, scales, signed, bits in ((m, s["mc"][i], s["ms"][i], True, r & 0xFFFF),
                                                   (v, s["vc"][i], s["vs"][i], False, r >> 16)):
                c, e = _codes8(x, signed, bits)
                codes.copy_(c)
                scales.copy_(e)
            m, v = _values8(s["mc"][i], s["ms"][i], True), _values8(s["vc"][i], s["vs"][i], False)
        s["m"][i].copy_(m)
        s["v"][i].copy_(v)
    return _step_outputs(s, case)


def _step_outputs(s, case):
    return {"p": s["flat_p"], "m": s["flat_m"], "v": s["flat_v"], "w": s["flat_w"] if case["master"] else []}


_FOUR = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what 4 bits stand for, by sign and size


def _codes(x):
    """Rows [n, K] in 4 bits: codes [n, blocks * 16], two to a byte, the first in the low half, and scales [n, blocks]:
    the exponent of the block's largest value, less 2, plus 127. Ties go to the even code, larger values to 6."""
    n, K = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -K % SHARED)).reshape(n, -1, SHARED)
    top = x.abs().amax(2, keepdim=True)
    e = (torch.frexp(top).exponent - 3).clamp_min(-127)
    e = torch.where(top > 0, e, -127)
    y = _scaled_by_power(x.abs(), -e)
    c = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5))
    c = c | (torch.signbit(x).to(torch.uint8) << 3)
    c = c.reshape(n, -1, 2)
    return c[..., 0] | (c[..., 1] << 4), (e + 127).to(torch.uint8).reshape(n, -1)


def _values(codes, scales, K):
    """What 4-bit rows stand for, in float32."""
    n = codes.shape[0]
    table = torch.tensor(_FOUR + tuple(-v for v in _FOUR), device=codes.device)
    v = table[torch.stack((codes & 15, codes >> 4), 2).long()].reshape(n, -1, SHARED)
    return _scaled_by_power(v, scales.to(torch.int32).unsqueeze(2) - 127).reshape(n, -1)[:, :K]


def _plain_quantise(s, case):
    x = s["x"].t() if case["columns"] else s["x"]
    codes, scales = _codes(x)
    s["codes"].copy_(codes)
    s["scales"].copy_(scales)
    v = _values(s["codes"], s["scales"], case["K"])
    return (v.t() if case["columns"] else v).to(s["values"].dtype)


def _act(a, z):
    if a == "relu":
        return z * (z > 0)
    if a == "silu":
        return z / (1 + (-z).exp())
    return z * 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) if a == "gelu" else z


def _plain_product(s, case):
    x = _values(*_codes(s["x"]), case["K"]) if case["both"] else s["x"].float()
    y = _act(case["act"], x @ _values(*s["W"], case["K"]).t() + s["bias"].float())
    return (y + s["res"].float() if case["res"] else y).to(s["y"].dtype)


# ------------------------------------------------------------------ the library's calls


def _own(s, case):
    import paper_2608_24067_amd.dense as dense

    if case["kind"] == "norm":
        if not case["train"]:
            return dense.layer_norm(s["x"], s["weight"], s["bias"], eps=1e-5, out=s["y"])
        y = dense.layer_norm(s["x"], s["weight"], s["bias"], eps=1e-5, out=s["y"], stats=s["stats"])
        return (y,) + dense.layer_norm_bwd(s["x"], s["dy"], s["stats"], s["weight"], add=s["add"], out=s["grads"],
                                           workspace=s["scratch"])
    if case["kind"] == "step":
        n, master = case["n"], s["master"] if case["master"] else [None] * case["n"]
        if case["bits"] == 8:
            states = [dense.AdamwState(*t) for t in zip(s["mc"], s["vc"], s["ms"], s["vs"], master)]
        else:
            states = [dense.AdamwState(*t) for t in zip(s["m"], s["v"], [None] * n, [None] * n, master)]
        dense.adamw(s["params"], s["grads"], states, STEP["step"], lr=STEP["lr"], betas=(STEP["beta1"], STEP["beta2"]),
                    eps=STEP["eps"], weight_decay=STEP["weight_decay"], seed=STEP["seed"])
        if case["bits"] == 8:
            dense.adamw_values(states, out=(s["m"], s["v"]))
        return _step_outputs(s, case)
    if case["kind"] == "quantise":
        q = dense.mx4_quantise(s["x"], columns=case["columns"], out=(s["codes"], s["scales"]))
        return dense.mx4_values(q, columns=case["columns"], out=s["values"])
    x = s["x"]
    if case["both"]:
        x = dense.mx4_quantise(x, out=(s["codes"], s["scales"]))
    return dense.mx4_linear(x, dense.Mx4(*s["W"], case["K"]), s["bias"], residual=s["res"], act=case["act"],
                            out=s["y"], workspace=s["scratch"])


_PLAIN = {"norm": _plain_norm, "step": _plain_step, "quantise": _plain_quantise, "product": _plain_product}


def run(state):
    case = state["case"]
    return _own(state, case) if own else _PLAIN[case["kind"]](state, case)


def _size(name):
    return 4 if name == "float32" else 2


def work(case):
    """What one pass cannot do without: every input read once, every output written once, every product term."""
    if case["kind"] == "norm":
        N, D, x, y = case["N"], case["D"], _size(case["x"]), _size(case["y"])
        weights = {"none": 0, "weight": 1, "both": 2}[case["affine"]] * D * _size(case["wtype"])
        moved = N * D * (x + y) + weights
        if case["train"]:
            moved += N * D * (x + y) + weights + (N * D * x if case["add"] else 0)
        return {"bytes": moved, "flops": N * D * (8 + (14 if case["train"] else 0))}
    if case["kind"] == "step":
        moved = 0
        for n, t in zip(_sizes(case), _types(case)):
            p = 4 if t == torch.float32 else 2
            moved += n * ((8 + p if case["master"] else 2 * p) + (4 if case["grad32"] else p))
            moved += 16 * n if case["bits"] == 32 else 12 * n + 4 * (n / BLOCK)
        return {"bytes": moved, "flops": 15 * sum(_sizes(case))}
    if case["kind"] == "quantise":
        n, x = case["N"] * case["K"], _size(case["dtype"])
        return {"bytes": n * 2 * x + n * 17 / 32, "flops": 4 * n}
    N, K, M, x = case["N"], case["K"], case["M"], 2
    moved = K * M * 17 / 32 + N * K * x + M * (4 if case["scores"] else x) + (N * M * x if case["res"] else 0)
    return {"bytes": moved + N * M * (4 if case["scores"] else x), "flops": 2 * N * K * M}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "step": _exact_step, "quantise": _exact_quantise, "product": _exact_product}[
        case["kind"]](s, case)


def _exact_norm(s, case):
    with torch.enable_grad():
        x = s["x"].double().requires_grad_(case["train"])
        w, b = (s[n].double().requires_grad_(case["train"]) if s[n] is not None else None for n in ("weight", "bias"))
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        y = (x - mean) / torch.sqrt(var + 1e-5)
        y = y if w is None else y * w
        y = y if b is None else y + b
        if not case["train"]:
            return y
        got = torch.autograd.grad(y, [t for t in (x, w, b) if t is not None], s["dy"].double())
    dx = got[0] + (s["add"].double() if s["add"] is not None else 0)
    return (y.detach(), dx, got[1] if w is not None else None, got[-1] if b is not None else None)


def _two(e):
    """2^e in 64 bits, by its bits: a library's power may be off in the last place, and ties are decided there."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _wide8(code, scale, signed):
    """The values of 8-bit states from their fields: sign, exponent, three bits."""
    c, e = code.double(), scale.double().repeat_interleave(BLOCK)[:code.numel()] - 127
    sign = torch.where(c >= 128, -1.0, 1.0) if signed else torch.ones_like(c)
    c = c % 128 if signed else c
    field, last = torch.floor(c / 8), c % 8
    lowest = -14 if signed else -30  # the exponent of the smallest values with a leading one
    size = torch.where(field > 0, (8 + last) * _two(field + lowest - 4), last * 2.0 ** (lowest - 3))
    return sign * size * _two(e)


def _exact_step(s, case):
    """In place, as the step is; 8-bit states have no value but that of their rounding, which is drawn."""
    b1, b2, t = STEP["beta1"], STEP["beta2"], STEP["step"]
    out = {"p": [torch.zeros_like(f, dtype=torch.float64) for f in s["flat_p"]]}
    out["m"], out["v"], out["w"] = ([torch.zeros(s["flat_m"][0].numel(), dtype=torch.float64, device="cuda")] for _ in range(3))
    at, place = {f.dtype: 0 for f in s["flat_p"]}, 0
    which = {f.dtype: o for f, o in zip(s["flat_p"], out["p"])}
    for i, p in enumerate(s["params"]):
        n, g = p.numel(), s["grads"][i].double()
        if case["bits"] == 8:
            m, v = _wide8(s["mc"][i], s["ms"][i], True), _wide8(s["vc"][i], s["vs"][i], False)
        else:
            m, v = s["m"][i].double(), s["v"][i].double()
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        w = s["master"][i].double() if case["master"] else p.double()
        w = w - STEP["lr"] * STEP["weight_decay"] * w
        w = w - STEP["lr"] * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + STEP["eps"])
        which[p.dtype][at[p.dtype]:at[p.dtype] + n] = w
        for name, value in (("m", m), ("v", v), ("w", w)):
            out[name][0][place:place + n] = value
        at[p.dtype] += (n + 255) // 256 * 256
        place += (n + 255) // 256 * 256
    if case["bits"] == 8:
        out["m"] = out["v"] = [None]
    out["w"] = out["w"] if case["master"] else []
    return out


def _exact_four(x):
    """What the rows' 4-bit form stands for: the nearest of the eight sizes, by steps of a half, one and two."""
    n, K = x.shape
    x = torch.nn.functional.pad(x.double(), (0, -K % SHARED)).reshape(n, -1, SHARED)
    top = x.abs().amax(2, keepdim=True)
    unit = _two(torch.where(top > 0, torch.frexp(top).exponent.long() - 3, -127).clamp_min(-127))
    y = x / unit
    a = y.abs()
    r = torch.where(a < 2, torch.round(y * 2) / 2, torch.where(a < 4, torch.round(y), torch.round(y / 2) * 2))
    return (r.clamp(-6, 6) * unit).reshape(n, -1)[:, :K]


def _exact_quantise(s, case):
    return _exact_four(s["x"].t()).t() if case["columns"] else _exact_four(s["x"])


def _exact_product(s, case):
    K, (codes, scales) = case["K"], s["W"]
    four = torch.stack((codes & 15, codes >> 4), 2).reshape(codes.shape[0], -1).double()
    size, half = four % 8, torch.floor(four % 8 / 2)
    size = torch.where(half > 0, (2 + size % 2) * _two(half - 2), (size % 2) / 2)  # two bits of exponent, one behind
    W = torch.where(four >= 8, -size, size) * _two(scales.double() - 127).repeat_interleave(SHARED, 1)
    x = _exact_four(s["x"]) if case["both"] else s["x"].double()
    z = torch.addmm(s["bias"].double(), x, W[:, :K].t())
    if case["act"] == "relu":
        z = torch.relu(z)
    elif case["act"] == "silu":
        z = z * torch.sigmoid(z)
    elif case["act"] == "gelu":
        z = z * torch.special.ndtr(z)
    return z + s["res"].double() if case["res"] else z
