"""Dense rows on a map: ctypes binding of include/som_dense.h. Argument marshalling only.

Products of dense rows with a feature-major matrix (a codebook's scores, a layer), routing of rows to their best
units, the units' experts, and clipping of all gradients to a norm. As in ``som``, every function checks its tensors
and passes pointers and the current torch stream of the tensors' device to the C entry point of the same name.
Matrices and rows may have any row stride; the elements of a row must be adjacent.

No function takes part in autograd: results carry no graph, also where an argument requires a gradient (the ``_bwd``
functions give the gradients), and what is written in place (``out``, ``pre``, clip's tensors) is written without
autograd's knowledge of it, as if under ``torch.no_grad()`` and without a new version.
"""
from __future__ import annotations

import ctypes
import functools

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
