"""Dense rows on a map: ctypes binding of include/som_dense.h. Argument marshalling only.

Products of dense rows with a feature-major matrix (a codebook's scores, a layer), routing of rows to their best
units, the units' experts, clipping of all gradients to a norm; layer norm, AdamW's step, and rows and matrices in 4
bits with their products. As in ``som``, every function checks its tensors
and passes pointers and the current torch stream of the tensors' device to the C entry point of the same name.
Matrices and rows may have any row stride; the elements of a row must be adjacent.

No function takes part in autograd: results carry no graph, also where an argument requires a gradient (the ``_bwd``
functions give the gradients), and what is written in place (``out``, ``pre``, clip's tensors) is written without
autograd's knowledge of it, as if under ``torch.no_grad()`` and without a new version.
"""
from __future__ import annotations

import ctypes
import functools
from array import array
from itertools import chain
from operator import attrgetter
from typing import NamedTuple, Optional

import torch

from .som import SOM_OK, SomError, load  # noqa: F401
from .som import _check as _raise

F32, F16, BF16 = 0, 1, 2
_TYPES = {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}
_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
_SCORES = {"softmax": 0, "sigmoid": 1}


def _check(status, where):
    if status != SOM_OK:
        _raise(status, where)


_current = torch.cuda.current_stream
try:  # the stream's handle without an object around it, where torch offers it
    _handle = torch._C._cuda_getCurrentRawStream
except AttributeError:
    _handle = None


def _stream(t):
    return _handle(t.device.index) if _handle is not None else _current(t.device).cuda_stream


class _RouteConfig(ctypes.Structure):
    _fields_ = [("score", ctypes.c_int32), ("renorm", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("group_top", ctypes.c_int32), ("reserved", ctypes.c_int32 * 4)]


def _named(table, key, what):
    if key not in table:
        raise ValueError(f"{what} must be one of {', '.join(map(str, table))} (got {key})")
    return table[key]


def _type(t, name, halves=True):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in _TYPES or (halves and t.dtype == torch.float32):
        raise TypeError(f"{name} must be {'' if halves else 'float32, '}float16 or bfloat16 (got {t.dtype})")
    return _TYPES[t.dtype]


def _refuse(t, name, shape, dtype, device):
    """Says what is wrong with a tensor that is not what it must be."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.dtype not in (dtype if isinstance(dtype, tuple) else (dtype,)):
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if t.device != device or not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU, with the other tensors")
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must be {shape} (got {tuple(t.shape)})")


def _mat(t, name, shape, dtype, device):
    """Pointer and row stride of a matrix whose rows' elements are adjacent."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device or t.shape != shape or not t.is_cuda:
        _refuse(t, name, shape, dtype, device)
    step, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    if step < shape[1]:
        if shape[0] > 1:
            raise ValueError(f"{name}: rows overlap")
        step = shape[1]
    return t.data_ptr(), step


def _vec(t, name, shape, dtype, device):
    """Pointer of a contiguous tensor of a type, or of one of several."""
    if (not isinstance(t, torch.Tensor) or (t.dtype not in dtype if isinstance(dtype, tuple) else t.dtype != dtype)
            or t.device != device or t.shape != shape or not t.is_cuda):
        _refuse(t, name, shape, dtype, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _work(ws, need, device):
    if ws is None:
        return torch.empty(need, dtype=torch.uint8, device=device) if need else None
    if ws.dtype != torch.uint8 or ws.device != device or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the same device")
    return ws


def _pointer(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel())


def _two(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    return t.shape


# ------------------------------------------------------------------ products

def linear(x, W, bias=None, residual=None, act: str = "none", out=None, out_dtype=None, pre=None):
    """residual + act(x W + bias) for rows x [N, K] and a feature-major W [K, M] (both float16 or both bfloat16).

    bias [M] is float32 or of x's type. The result (``out``, or a new tensor of ``out_dtype``) is of x's type or
    float32. ``pre`` [N, M] takes x W + bias, which linear_bwd of an activation needs. With a codebook W and the bias
    -norms / 2 the result ranks units as their distances do.
    """
    kind, dev = _type(x, "x"), x.device
    (N, K), (K2, M) = _two(x, "x"), _two(W, "W")
    if K2 != K:
        raise ValueError(f"W must have {K} rows (got {K2})")
    if out is None:
        out = torch.empty(N, M, dtype=out_dtype or x.dtype, device=dev)
    xp, ldx = _mat(x, "x", (N, K), x.dtype, dev)
    wp, ldw = _mat(W, "W", (K, M), x.dtype, dev)
    yp, ldy = _mat(out, "out", (N, M), out.dtype if out.dtype in (torch.float32, x.dtype) else x.dtype, dev)
    bp = _vec(bias, "bias", (M,), (torch.float32, x.dtype), dev) if bias is not None else None
    rp, ldr = _mat(residual, "residual", (N, M), x.dtype, dev) if residual is not None else (None, 0)
    pp, ldp = _mat(pre, "pre", (N, M), x.dtype, dev) if pre is not None else (None, 0)
    _check(load().som_linear(kind, xp, ldx, wp, ldw, bp, _TYPES[bias.dtype] if bias is not None else F32,
                             _named(_ACTS, act, "act"), rp, ldr, yp, ldy, _TYPES[out.dtype], pp, ldp, N, K, M,
                             _stream(x)), "som_linear")
    return out


def linear_bwd(x, W, dy, pre=None, act: str = "none", out=None, bias_dtype=None, workspace=None):
    """(dx, dW, dbias) of linear, from dy [N, M] of x's type and the ``pre`` that linear wrote.

    ``out`` may pass the three tensors; one that is None is not computed. dbias is of ``bias_dtype`` (float32 or x's
    type, the default).
    """
    kind, dev = _type(x, "x"), x.device
    (N, K), (K2, M) = _two(x, "x"), _two(W, "W")
    if K2 != K:
        raise ValueError(f"W must have {K} rows (got {K2})")
    a = _named(_ACTS, act, "act")
    if out is None:
        out = (torch.empty(N, K, dtype=x.dtype, device=dev), torch.empty(K, M, dtype=x.dtype, device=dev),
               torch.empty(M, dtype=bias_dtype or x.dtype, device=dev))
    dx, dW, db = out
    lib = load()
    ws = _work(workspace, lib.som_linear_bwd_workspace_bytes(N, K, M, a), dev)
    xp, ldx = _mat(x, "x", (N, K), x.dtype, dev)
    wp, ldw = _mat(W, "W", (K, M), x.dtype, dev)
    gp, ldg = _mat(dy, "dy", (N, M), x.dtype, dev)
    pp, ldp = _mat(pre, "pre", (N, M), x.dtype, dev) if pre is not None else (None, 0)
    dxp, lddx = _mat(dx, "dx", (N, K), x.dtype, dev) if dx is not None else (None, 0)
    dwp, lddw = _mat(dW, "dW", (K, M), x.dtype, dev) if dW is not None else (None, 0)
    dbp = _vec(db, "dbias", (M,), (torch.float32, x.dtype), dev) if db is not None else None
    _check(lib.som_linear_bwd(kind, xp, ldx, wp, ldw, pp, ldp, a, gp, ldg, dxp, lddx, dwp, lddw, dbp,
                              _TYPES[db.dtype] if db is not None else F32, N, K, M, *_pointer(ws), _stream(x)),
           "som_linear_bwd")
    return tuple(out)


# ------------------------------------------------------------------ routing

@functools.lru_cache(maxsize=64)
def _route_config(score, renorm, groups, group_top):
    c = _RouteConfig()
    c.score, c.renorm = _named(_SCORES, score, "score"), 1 if renorm else 0
    c.groups, c.group_top = int(groups), int(group_top)
    return ctypes.byref(c)


def route(logits, k: int, bias=None, score: str = "softmax", renorm: bool = True, groups: int = 1, group_top: int = 0,
          weights_dtype=None, out=None, counts=None):
    """Each row's k best units: (idx int32 [N, k], weights [N, k]), by falling logit + bias, the lowest index first.

    logits [N, E] are float32, float16 or bfloat16; weights (of ``weights_dtype``, the logits' by default) are the
    units' softmax or sigmoid scores without the bias, divided by their sum under ``renorm``. With ``groups`` only
    units of the ``group_top`` best groups are taken. A unit whose logit (or logit + bias) is NaN or -inf is closed;
    missing places hold index -1 and weight 0. ``counts`` int32 [E] takes how many rows took each unit; ``out`` may
    pass (idx, weights).
    """
    kind, dev = _type(logits, "logits", halves=False), logits.device
    N, E = _two(logits, "logits")
    if out is None:
        out = (torch.empty(N, k, dtype=torch.int32, device=dev),
               torch.empty(N, k, dtype=weights_dtype or logits.dtype, device=dev))
    idx, w = out
    lp, ldl = _mat(logits, "logits", (N, E), logits.dtype, dev)
    wt = _type(w, "weights", halves=False)
    _check(load().som_route(kind, lp, ldl, _vec(bias, "bias", (E,), torch.float32, dev) if bias is not None else None,
                            N, E, int(k), _route_config(score, renorm, groups, group_top),
                            _vec(idx, "idx", (N, k), torch.int32, dev), wt, _vec(w, "weights", (N, k), w.dtype, dev),
                            _vec(counts, "counts", (E,), torch.int32, dev) if counts is not None else None,
                            _stream(logits)), "som_route")
    return idx, w


def route_bwd(logits, idx, dweights, bias=None, score: str = "softmax", renorm: bool = True, groups: int = 1,
              group_top: int = 0, out=None):
    """The logits' gradient [N, E] from the weights' [N, k], for the units idx that route took."""
    kind, dev = _type(logits, "logits", halves=False), logits.device
    (N, E), (_, k) = _two(logits, "logits"), _two(idx, "idx")
    if out is None:
        out = torch.empty(N, E, dtype=logits.dtype, device=dev)
    lp, ldl = _mat(logits, "logits", (N, E), logits.dtype, dev)
    dp, lddl = _mat(out, "out", (N, E), logits.dtype, dev)
    wt = _type(dweights, "dweights", halves=False)
    _check(load().som_route_bwd(kind, lp, ldl,
                                _vec(bias, "bias", (E,), torch.float32, dev) if bias is not None else None,
                                _vec(idx, "idx", (N, k), torch.int32, dev), wt,
                                _vec(dweights, "dweights", (N, k), dweights.dtype, dev), N, E, k,
                                _route_config(score, renorm, groups, group_top), dp, lddl, _stream(logits)),
           "som_route_bwd")
    return out


# ------------------------------------------------------------------ experts

def _experts_shapes(x, idx, W1):
    N, D = _two(x, "x")
    n, k = _two(idx, "idx")
    if n != N:
        raise ValueError(f"idx must have {N} rows (got {n})")
    if not isinstance(W1, torch.Tensor) or W1.dim() != 3 or W1.shape[1] != D:
        raise ValueError(f"W1 must be [experts, {D}, inner width]")
    return N, D, k, W1.shape[0], W1.shape[2]


def experts_workspace_bytes(N: int, k: int, E: int, D: int, F: int, keep: bool = False) -> int:
    n = load().som_experts_workspace_bytes(N, k, E, D, F, 1 if keep else 0)
    if n == 0:
        raise ValueError("som_experts_workspace_bytes: invalid sizes")
    return n


def experts(x, idx, w, W1, b1, W2, b2, act: str = "gelu", residual=None, out=None, keep: bool = False,
            workspace=None):
    """residual + the sum over a row's places j of w (act(x W1[e] + b1[e]) W2[e] + b2[e]), e = idx[n, j].

    x [N, D], w [N, k], W1 [E, D, F], b1 [E, F] or None, W2 [E, F, D], b2 [E, D] or None, residual [N, D] or None, all
    float16 or all bfloat16; idx int32 [N, k] (-1: no expert). With ``keep`` the workspace, which must then be passed
    (experts_workspace_bytes), keeps what experts_bwd needs.
    """
    kind, dev, dt = _type(x, "x"), x.device, x.dtype
    N, D, k, E, F = _experts_shapes(x, idx, W1)
    if out is None:
        out = torch.empty(N, D, dtype=dt, device=dev)
    if keep and workspace is None:
        raise ValueError("keep: pass the workspace that experts_bwd is to read")
    ws = _work(workspace, experts_workspace_bytes(N, k, E, D, F, keep) if workspace is None else 0, dev)
    xp, ldx = _mat(x, "x", (N, D), dt, dev)
    op, ldo = _mat(out, "out", (N, D), dt, dev)
    rp, ldr = _mat(residual, "residual", (N, D), dt, dev) if residual is not None else (None, 0)
    _check(load().som_experts(
        kind, xp, ldx, _vec(idx, "idx", (N, k), torch.int32, dev), _vec(w, "w", (N, k), dt, dev),
        _vec(W1, "W1", (E, D, F), dt, dev), _vec(b1, "b1", (E, F), dt, dev) if b1 is not None else None,
        _vec(W2, "W2", (E, F, D), dt, dev), _vec(b2, "b2", (E, D), dt, dev) if b2 is not None else None,
        _named(_ACTS, act, "act"), rp, ldr, op, ldo, N, k, E, D, F, 1 if keep else 0, *_pointer(ws), _stream(x)),
        "som_experts")
    return out


def experts_bwd(x, idx, w, W1, W2, b2, dout, act: str = "gelu", out=None, workspace=None):
    """(dx, dw, dW1, db1, dW2, db2) from dout [N, D] and the workspace that experts(keep=True) left.

    The other arguments are those of experts. ``out`` may pass the six tensors; one that is None is not computed. The
    workspace must not have been passed to another call in between: nothing in it tells.
    """
    kind, dev, dt = _type(x, "x"), x.device, x.dtype
    N, D, k, E, F = _experts_shapes(x, idx, W1)
    if workspace is None:
        raise ValueError("workspace: pass the one that experts(keep=True) left")
    if out is None:
        out = tuple(torch.empty(s, dtype=dt, device=dev)
                    for s in ((N, D), (N, k), (E, D, F), (E, F), (E, F, D), (E, D)))
    dx, dw, dW1, db1, dW2, db2 = out
    xp, ldx = _mat(x, "x", (N, D), dt, dev)
    gp, ldg = _mat(dout, "dout", (N, D), dt, dev)
    dxp, lddx = _mat(dx, "dx", (N, D), dt, dev) if dx is not None else (None, 0)

    def given(t, name, shape):
        return _vec(t, name, shape, dt, dev) if t is not None else None

    _check(load().som_experts_bwd(
        kind, xp, ldx, _vec(idx, "idx", (N, k), torch.int32, dev), _vec(w, "w", (N, k), dt, dev),
        _vec(W1, "W1", (E, D, F), dt, dev), _vec(W2, "W2", (E, F, D), dt, dev), given(b2, "b2", (E, D)),
        _named(_ACTS, act, "act"), gp, ldg, dxp, lddx, given(dw, "dw", (N, k)), given(dW1, "dW1", (E, D, F)),
        given(db1, "db1", (E, F)), given(dW2, "dW2", (E, F, D)), given(db2, "db2", (E, D)), N, k, E, D, F,
        *_pointer(_work(workspace, 0, dev)), _stream(x)), "som_experts_bwd")
    return tuple(out)


# ------------------------------------------------------------------ clipping

def clip(tensors, max_norm: float, out=None, norm=None, workspace=None):
    """Scales the tensors together to a norm of at most max_norm; returns (outs, norm before scaling, float32 [1]).

    The tensors are contiguous, each float32, float16 or bfloat16, on one device. ``out`` passes the tensors that are
    written (the same ones to scale in place, which is the default). An infinite or NaN norm scales nothing.
    """
    tensors = list(tensors)
    outs = tensors if out is None else list(out)
    if len(outs) != len(tensors):
        raise ValueError(f"out must hold {len(tensors)} tensors")
    if norm is None:
        if not tensors:
            raise ValueError("no tensors: pass norm")
        norm = torch.empty(1, dtype=torch.float32, device=tensors[0].device)
    n, dev = len(tensors), norm.device
    if not norm.is_cuda:
        raise ValueError("norm must be on the GPU")
    at, types, lengths = dev.index, [], []
    for t in tensors:
        kind = _TYPES.get(t.dtype) if isinstance(t, torch.Tensor) else None
        if kind is None:
            _type(t, "tensors", halves=False)
        if t.get_device() != at or not t.is_contiguous():
            raise ValueError("tensors must be contiguous and on one GPU")
        types.append(kind)
        lengths.append(t.numel())
    if out is not None:
        for o, t, m in zip(outs, tensors, lengths):
            if (not isinstance(o, torch.Tensor) or o.dtype is not t.dtype or o.numel() != m or o.get_device() != at
                    or not o.is_contiguous()):
                raise ValueError("out must hold contiguous tensors of the same sizes and types")
    pointers = ctypes.c_void_p * n
    ins = pointers(*[t.data_ptr() for t in tensors])
    tos = ins if out is None else pointers(*[o.data_ptr() for o in outs])
    sizes, types = (ctypes.c_int64 * n)(*lengths), (ctypes.c_int32 * n)(*types)
    lib = load()
    ws = _work(workspace, lib.som_clip_workspace_bytes(sizes, n), dev)
    _check(lib.som_clip(ins, tos, sizes, types, n, float(max_norm), _vec(norm, "norm", (1,), torch.float32, dev),
                        *_pointer(ws), _stream(norm)), "som_clip")
    return outs, norm


# ------------------------------------------------------------------ layer norm

try:  # the current device's number, without the wait for its initialisation that torch's own function checks for
    _device = torch._C._cuda_getDevice
except AttributeError:
    _device = torch.cuda.current_device


def _on(device, call, *args):
    """A call with `device` as the current one, which a launch on one of its streams needs."""
    if device.index == _device():
        return call(*args)
    with torch.cuda.device(device):
        return call(*args)


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out=None, out_dtype=None, stats=None):
    """(x - mean) / sqrt(var + eps) * weight + bias over each row of x [N, D].

    x is float32, float16 or bfloat16; the result (``out``, or a new tensor of ``out_dtype``) is of x's type, or of any
    of the three for float32 rows. weight and bias [D], or None, are both float32 or both of the result's type.
    ``stats`` float64 [N, 2] takes each row's mean and 1 / sqrt(var + eps), which layer_norm_bwd needs. ``out`` may be x.
    """
    kind, dev = _type(x, "x", halves=False), x.device
    N, D = _two(x, "x")
    if out is None:
        out = torch.empty(N, D, dtype=out_dtype or x.dtype, device=dev)
    to = _type(out, "out", halves=False)
    xp, ldx = _mat(x, "x", (N, D), x.dtype, dev)
    yp, ldy = _mat(out, "out", (N, D), out.dtype, dev)
    some = weight if weight is not None else bias
    wdt = some.dtype if isinstance(some, torch.Tensor) and some.dtype == out.dtype else torch.float32
    wp = _vec(weight, "weight", (D,), wdt, dev) if weight is not None else None
    bp = _vec(bias, "bias", (D,), wdt, dev) if bias is not None else None
    sp = _vec(stats, "stats", (N, 2), torch.float64, dev) if stats is not None else None
    _check(_on(dev, load().som_layer_norm, kind, xp, ldx, wp, bp, _TYPES[wdt], float(eps), yp, ldy, to, sp, N, D,
               _stream(x)), "som_layer_norm")
    return out


def layer_norm_bwd(x, dy, stats, weight=None, add=None, out=None, weight_dtype=None, workspace=None):
    """(dx, dweight, dbias) of layer_norm, from dy [N, D] of its result's type and the ``stats`` it wrote.

    ``add`` [N, D] of x's type is added to dx: the gradient that reaches x by another way, as round a layer. ``out``
    may pass the three tensors; one that is None is not computed. dweight and dbias are of the weight's type
    (``weight_dtype`` where there is none: float32, the default, or dy's type). ``out``'s dx may be ``add`` or dy.
    """
    kind, dev = _type(x, "x", halves=False), x.device
    N, D = _two(x, "x")
    g = _type(dy, "dy", halves=False)
    wdt = weight.dtype if isinstance(weight, torch.Tensor) else weight_dtype
    if out is None:
        wdt = wdt or torch.float32
        out = (torch.empty(N, D, dtype=x.dtype, device=dev), torch.empty(D, dtype=wdt, device=dev),
               torch.empty(D, dtype=wdt, device=dev))
    dx, dw, db = out
    wdt = wdt or next((t.dtype for t in (dw, db) if isinstance(t, torch.Tensor)), torch.float32)
    if wdt not in (torch.float32, dy.dtype):
        raise TypeError(f"weight, dweight and dbias must be float32 or {dy.dtype} (got {wdt})")
    lib = load()
    ws = _work(workspace, lib.som_layer_norm_bwd_workspace_bytes(N, D) if workspace is None else 0, dev)
    xp, ldx = _mat(x, "x", (N, D), x.dtype, dev)
    gp, ldg = _mat(dy, "dy", (N, D), dy.dtype, dev)
    ap, lda = _mat(add, "add", (N, D), x.dtype, dev) if add is not None else (None, 0)
    dxp, lddx = _mat(dx, "dx", (N, D), x.dtype, dev) if dx is not None else (None, 0)
    wp = _vec(weight, "weight", (D,), wdt, dev) if weight is not None else None
    dwp = _vec(dw, "dweight", (D,), wdt, dev) if dw is not None else None
    dbp = _vec(db, "dbias", (D,), wdt, dev) if db is not None else None
    _check(_on(dev, lib.som_layer_norm_bwd, kind, xp, ldx, wp, _TYPES[wdt], gp, ldg, g,
               _vec(stats, "stats", (N, 2), torch.float64, dev), ap, lda, dxp, lddx, dwp, dbp, N, D, *_pointer(ws),
               _stream(x)), "som_layer_norm_bwd")
    return tuple(out)


# ------------------------------------------------------------------ AdamW

class AdamwState(NamedTuple):
    """A tensor's running means: float32 like the tensor, or, with scales, in 8 bits (uint8 codes and blocks' scales);
    and its float32 copy, or None."""
    m: torch.Tensor
    v: torch.Tensor
    m_scales: Optional[torch.Tensor] = None
    v_scales: Optional[torch.Tensor] = None
    master: Optional[torch.Tensor] = None


# A tensor of a step as the C structure holds it: nine words of 64 bits, seven pointers, the size and the two types.
_ADAMW_WORDS = 9


class _AdamwConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay", "grad_scale")] + [
        ("step", ctypes.c_int64), ("bits", ctypes.c_int32), ("seed", ctypes.c_uint32), ("lr_at", ctypes.c_void_p),
        ("step_at", ctypes.c_void_p), ("norm", ctypes.c_void_p), ("reserved", ctypes.c_int64 * 4)]


STATE_BLOCK = 256  # values of a block of 8-bit states


def adamw_state(param, bits: int = 32, master: bool = False) -> AdamwState:
    """The state of a parameter before its first step: zeros, in 32 bits or 8, and with ``master`` a float32 copy."""
    _type(param, "param", halves=False)
    copy = param.detach().float().clone().contiguous() if master else None
    if bits == 32:
        m, v = (torch.zeros(param.shape, dtype=torch.float32, device=param.device) for _ in range(2))
        return AdamwState(m, v, None, None, copy)
    if bits != 8:
        raise ValueError(f"bits must be 32 or 8 (got {bits})")
    blocks = (param.numel() + STATE_BLOCK - 1) // STATE_BLOCK
    m, v = (torch.zeros(param.shape, dtype=torch.uint8, device=param.device) for _ in range(2))
    ms, vs = (torch.zeros(blocks, dtype=torch.uint8, device=param.device) for _ in range(2))
    return AdamwState(m, v, ms, vs, copy)


def _refuse_held(t, name, n, dtype):
    raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on the parameters' GPU"
                     + (f" (got {t.dtype}, {t.numel()} elements on {t.device})" if isinstance(t, torch.Tensor) else ""))


def _held(t, name, n, dtype, at):
    """The pointer of a contiguous tensor of n elements on device number `at`."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.numel() != n or t.get_device() != at or not t.is_contiguous():
        _refuse_held(t, name, n, dtype)
    return t.data_ptr()


# What a list of tensors is asked, one question at a time: faster than tensor by tensor.
_numel, _number, _dtype = torch.Tensor.numel, torch.Tensor.get_device, attrgetter("dtype")
_dense, _address = torch.Tensor.is_contiguous, torch.Tensor.data_ptr


def _held_all(ts, name, dtype, sizes, at):
    """The pointers of such tensors; dtype None: of any type."""
    try:
        if (list(map(_numel, ts)) == sizes and set(map(_number, ts)) == {at}
                and (dtype is None or set(map(_dtype, ts)) == {dtype}) and all(map(_dense, ts))):
            return list(map(_address, ts))
    except (AttributeError, TypeError):  # something that is no tensor
        pass
    return [_held(t, name, n, t.dtype if dtype is None else dtype, at) for t, n in zip(ts, sizes)]


def _state_pointers(states, sizes, eight, at):
    """Checks the states and returns their pointers, in the C structure's order: m, v, their scales, the masters."""
    ms, vs, m_scales, v_scales, masters = zip(*states)
    none, kind = [0] * len(sizes), torch.uint8 if eight else torch.float32
    if any([(x is not None) != eight for x in m_scales]) or any([(x is not None) != eight for x in v_scales]):
        raise ValueError("the states must all be in 32 bits, or all in 8")
    scales = (none, none)
    if eight:
        blocks = [(n + STATE_BLOCK - 1) // STATE_BLOCK for n in sizes]
        scales = (_held_all(m_scales, "m_scales", kind, blocks, at), _held_all(v_scales, "v_scales", kind, blocks, at))
    copies, missing = none, sum([t is None for t in masters])  # not masters.count(None): a tensor compares slowly
    if missing == 0:
        copies = _held_all(masters, "master", torch.float32, sizes, at)
    elif missing < len(sizes):
        copies = [0 if t is None else _held(t, "master", n, torch.float32, at) for t, n in zip(masters, sizes)]
    return (_held_all(ms, "m", kind, sizes, at), _held_all(vs, "v", kind, sizes, at), *scales, copies)


def _table(*columns):
    """The C structures, one after the other, and their address."""
    words = array("q", list(chain.from_iterable(zip(*columns))))
    return words, words.buffer_info()[0]


def _scalar_at(t, name, dtype, dev):
    return _vec(t, name, (1,), dtype, dev)


def adamw(params, grads, states, step, lr=1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
          grad_scale: float = 1.0, seed: int = 0, norm=None):
    """One step of AdamW over all parameters, in place.

    The parameters and their gradients are contiguous, each float32, float16 or bfloat16, on one device; states are
    AdamwState (adamw_state), all in 32 bits or all in 8. A state's master, where it has one, is what the step reads and
    updates; the parameter takes its rounded value. ``step`` is this step's number from 1 on, ``lr`` the rate; either
    may be a tensor [1] on the device (int32, float32), so that a captured step goes on when replayed.
    Gradients are multiplied by ``grad_scale``. ``norm``, float32 [1], as clip returns it: where it is infinite or NaN
    the step is left out. ``seed`` (0 ... 2^32 - 1) decides the rounding of 8-bit states, together with the step.
    No tensor may hold elements of another.
    """
    params, grads, states = list(params), list(grads), list(states)
    n = len(params)
    if len(grads) != n or len(states) != n:
        raise ValueError(f"grads and states must hold {n} entries each")
    if not n:
        return
    if not isinstance(params[0], torch.Tensor) or not params[0].is_cuda:
        raise ValueError("the parameters must be on the GPU")
    dev = params[0].device
    at, eight = dev.index, states[0][2] is not None
    try:
        kinds, grad_kinds = ([_TYPES[t] for t in map(_dtype, ts)] for ts in (params, grads))
    except (AttributeError, KeyError):
        for t in params + grads:
            _type(t, "params and grads", halves=False)
        raise
    sizes = list(map(_numel, params))
    pointers = _held_all(params, "params", None, sizes, at)
    table, address = _table(pointers, _held_all(grads, "grads", None, sizes, at), *_state_pointers(states, sizes, eight, at),
                            sizes, [k | g << 32 for k, g in zip(kinds, grad_kinds)])
    if len(set(pointers)) < n and len({p for p, m in zip(pointers, sizes) if m}) < sum([m > 0 for m in sizes]):
        raise ValueError("params holds a tensor twice")
    c = _AdamwConfig()
    if isinstance(lr, torch.Tensor):
        c.lr_at, lr = _scalar_at(lr, "lr", torch.float32, dev), 0.0
    if isinstance(step, torch.Tensor):
        c.step_at, step = _scalar_at(step, "step", torch.int32, dev), 1
    if not 0 <= int(seed) < 1 << 32:
        raise ValueError("seed must be 0 ... 2^32 - 1")
    c.lr, c.beta1, c.beta2, c.eps, c.weight_decay = float(lr), float(betas[0]), float(betas[1]), float(eps), float(weight_decay)
    c.grad_scale, c.step, c.bits, c.seed = float(grad_scale), int(step), 8 if eight else 32, int(seed)
    if norm is not None:
        c.norm = _scalar_at(norm, "norm", torch.float32, dev)
    _check(_on(dev, load().som_adamw, address, n, ctypes.byref(c), _stream(params[0])), "som_adamw")


def adamw_values(states, out=None):
    """(m, v) of 8-bit states as lists of float32 tensors; ``out`` may pass both lists."""
    states = list(states)
    n = len(states)
    if out is None:
        out = tuple([torch.empty(s[0].shape, dtype=torch.float32, device=s[0].device) for s in states] for _ in range(2))
    if len(out[0]) != n or len(out[1]) != n:
        raise ValueError(f"out must hold two lists of {n} tensors")
    if not n:
        return out
    if not isinstance(states[0][0], torch.Tensor) or not states[0][0].is_cuda:
        raise ValueError("the states must be on the GPU")
    dev = states[0][0].device
    sizes, none = list(map(_numel, [s[0] for s in states])), [0] * n
    held = _state_pointers([(*s[:4], None) for s in states], sizes, True, dev.index)
    table, address = _table(none, none, *held, sizes, none)  # read during the call
    tos = [array("q", _held_all(ts, name, torch.float32, sizes, dev.index)) for ts, name in zip(out, ("m", "v"))]
    _check(_on(dev, load().som_adamw_values, address, n, tos[0].buffer_info()[0], tos[1].buffer_info()[0], _stream(states[0][0])), "som_adamw_values")
    return out


# ------------------------------------------------------------------ 4 bits

class Mx4(NamedTuple):
    """Rows (or a matrix's columns) in 4 bits: codes uint8 [n, 16 ceil(width / 32)], scales uint8 [n, ceil(width / 32)]
    (som_dense.h says what they stand for), and how many features they hold."""
    codes: torch.Tensor
    scales: torch.Tensor
    width: int


def _four(q, name, width, dev):
    """Pointers and the number of rows of an Mx4."""
    codes, scales, K = q
    if K != width or width < 1:
        raise ValueError(f"{name} must hold {width} features (got {K})")
    blocks = (width + 31) // 32
    n = codes.shape[0] if isinstance(codes, torch.Tensor) and codes.dim() == 2 else -1
    return _vec(codes, name + ".codes", (n, 16 * blocks), torch.uint8, dev), _vec(scales, name + ".scales", (n, blocks),
                                                                                  torch.uint8, dev), n


def mx4_quantise(x, columns: bool = False, out=None) -> Mx4:
    """x in 4 bits: its rows [n, K], or with ``columns`` those of a feature-major matrix [K, n], as linear's W.

    x is float32, float16 or bfloat16. Blocks of 32 features share a power of two, the exponent of the largest less 2;
    values are rounded to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times it, ties to the even code. A block with an
    infinity or a NaN stands for NaN. ``out`` may pass (codes, scales).
    """
    kind, dev = _type(x, "x", halves=False), x.device
    rows, width = _two(x, "x")
    xp, ldx = _mat(x, "x", (rows, width), x.dtype, dev)
    n, K = (width, rows) if columns else (rows, width)
    blocks = (K + 31) // 32
    if out is None:
        out = (torch.empty(n, 16 * blocks, dtype=torch.uint8, device=dev), torch.empty(n, blocks, dtype=torch.uint8, device=dev))
    q = Mx4(out[0], out[1], K)
    cp = _vec(q.codes, "codes", (n, 16 * blocks), torch.uint8, dev)
    sp = _vec(q.scales, "scales", (n, blocks), torch.uint8, dev)
    _check(_on(dev, load().som_mx4_quantise, kind, xp, ldx, 1 if columns else 0, cp, sp, n, K, _stream(x)), "som_mx4_quantise")
    return q


def mx4_values(q: Mx4, columns: bool = False, dtype=None, out=None):
    """What q stands for, rounded to ``dtype`` (float32, float16 or bfloat16, the default, which holds it exactly but for
    the smallest scales): rows [n, width], or with ``columns`` a feature-major matrix [width, n]."""
    dev = q[0].device
    cp, sp, n = _four(q, "q", q[2], dev)
    shape = (q[2], n) if columns else (n, q[2])
    if out is None:
        out = torch.empty(shape, dtype=dtype or torch.bfloat16, device=dev)
    kind = _type(out, "out", halves=False)
    yp, ldy = _mat(out, "out", shape, out.dtype, dev)
    _check(_on(dev, load().som_mx4_values, kind, cp, sp, 1 if columns else 0, yp, ldy, n, q[2], _stream(out)), "som_mx4_values")
    return out


def mx4_linear(x, W: Mx4, bias=None, residual=None, act: str = "none", out=None, out_dtype=None, dtype=None,
               workspace=None):
    """residual + act(x W + bias), as linear, with W in 4 bits (mx4_quantise(W, columns=True)).

    x is rows [N, K] in float16 or bfloat16, or in 4 bits (an Mx4; the result's type is then ``dtype``, that of out,
    residual or a 16-bit bias, a 16-bit ``out_dtype``, or bfloat16). bias, residual and the result are as in linear.
    """
    packed = isinstance(x, tuple)
    if packed:
        dev, K = x[0].device, x[2]
        xp, xs, N = _four(x, "x", K, dev)
        ldx, at = 0, x[0]
        if dtype is None:
            dtype = next((t.dtype for t in (out, residual, bias) if isinstance(t, torch.Tensor) and t.dtype != torch.float32),
                         out_dtype if out_dtype not in (None, torch.float32) else torch.bfloat16)
    else:
        _type(x, "x")
        dev, at, dtype, xs = x.device, x, x.dtype, None
        N, K = _two(x, "x")
        xp, ldx = _mat(x, "x", (N, K), dtype, dev)
    if dtype not in (torch.float16, torch.bfloat16):
        raise TypeError(f"dtype must be float16 or bfloat16 (got {dtype})")
    wp, ws, M = _four(W, "W", K, dev)
    if out is None:
        out = torch.empty(N, M, dtype=out_dtype or dtype, device=dev)
    yp, ldy = _mat(out, "out", (N, M), out.dtype if out.dtype in (torch.float32, dtype) else dtype, dev)
    bp = _vec(bias, "bias", (M,), (torch.float32, dtype), dev) if bias is not None else None
    rp, ldr = _mat(residual, "residual", (N, M), dtype, dev) if residual is not None else (None, 0)
    lib = load()
    work = _work(workspace, lib.som_mx4_linear_workspace_bytes(N, K, M, 1 if packed else 0) if workspace is None else 0, dev)
    _check(_on(dev, lib.som_mx4_linear, _TYPES[dtype], xp, ldx, xs, wp, ws, bp,
               _TYPES[bias.dtype] if bias is not None else F32, _named(_ACTS, act, "act"), rp, ldr, yp, ldy,
               _TYPES[out.dtype], N, K, M, *_pointer(work), _stream(at)), "som_mx4_linear")
    return out
