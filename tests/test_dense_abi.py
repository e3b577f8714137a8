"""CPU tests of the dense entry points (include/som_dense.h): workspace queries, constants, and every argument check
that returns before anything reaches the GPU, through the C ABI and through the binding."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

import paper_2608_24067_amd.dense as dense
import paper_2608_24067_amd.som as som

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2608_24067_amd")
FAKE = ctypes.c_void_p(1 << 20)  # never followed: every call here is refused or has no rows
ODD = ctypes.c_void_p((1 << 20) + 1)
BIG = 1 << 40
INVALID, WORKSPACE = som.SOM_ERR_INVALID_ARG, som.SOM_ERR_WORKSPACE


def linear(**k):
    a = dict(type=2, X=FAKE, ldx=64, W=FAKE, ldw=32, bias=FAKE, bias_type=0, act=0, res=FAKE, ldr=32, Y=FAKE, ldy=32,
             y_type=2, pre=FAKE, ldp=32, N=10, K=64, M=32, stream=None)
    a.update(k)
    return som.load().som_linear(*a.values())


def linear_bwd(**k):
    a = dict(type=1, X=FAKE, ldx=64, W=FAKE, ldw=32, pre=FAKE, ldp=32, act=2, dY=FAKE, lddy=32, dX=FAKE, lddx=64,
             dW=FAKE, lddw=32, db=FAKE, bias_type=1, N=10, K=64, M=32, ws=FAKE, bytes=BIG, stream=None)
    a.update(k)
    return som.load().som_linear_bwd(*a.values())


def test_linear_refusals():
    for bad in (dict(type=0), dict(type=3), dict(X=None), dict(W=None), dict(Y=None), dict(ldx=63), dict(ldw=31),
                dict(ldr=31), dict(ldy=31), dict(ldp=31), dict(act=4), dict(act=-1), dict(y_type=1), dict(bias_type=1),
                dict(N=-1), dict(K=0), dict(M=0), dict(K=1 << 30), dict(M=1 << 30), dict(N=1 << 30), dict(X=ODD),
                dict(W=ODD), dict(Y=ODD), dict(bias=ctypes.c_void_p((1 << 20) + 2)), dict(res=ODD), dict(pre=ODD)):
        assert linear(**bad) == INVALID, bad
        assert som.last_error().startswith("som_linear"), som.last_error()
    assert linear(N=0, X=None, W=None, Y=None) == som.SOM_OK
    assert linear(N=0, K=0) == INVALID


def test_linear_bwd_refusals():
    lib = som.load()
    for bad in (dict(type=0), dict(X=None), dict(W=None), dict(dY=None), dict(pre=None), dict(ldx=63), dict(ldw=31),
                dict(lddy=31), dict(ldp=31), dict(lddx=63), dict(lddw=31), dict(act=9), dict(bias_type=2), dict(N=-1),
                dict(K=0), dict(M=1 << 30), dict(dY=ODD), dict(dX=ODD), dict(dW=ODD), dict(db=ODD)):
        assert linear_bwd(**bad) == INVALID, bad
    need = lib.som_linear_bwd_workspace_bytes(10, 64, 32, 2)
    assert need >= 10 * 32 * 2 and need % 256 == 0
    assert linear_bwd(bytes=need - 1) == WORKSPACE
    assert linear_bwd(ws=None) == WORKSPACE
    assert linear_bwd(ws=ctypes.c_void_p((1 << 20) + 128)) == WORKSPACE
    assert lib.som_linear_bwd_workspace_bytes(10, 64, 32, 0) == 0  # neither dz nor parts
    # many rows of a small dW are added up in parts
    assert lib.som_linear_bwd_workspace_bytes(100_000, 64, 32, 0) >= 2 * 64 * 32 * 4
    for bad in ((-1, 64, 32, 2), (10, 0, 32, 2), (10, 64, 0, 2), (10, 64, 32, 7), (10, 1 << 30, 32, 2)):
        assert lib.som_linear_bwd_workspace_bytes(*bad) == 0


def config(**k):
    c = dense._RouteConfig()
    for name, v in k.items():
        if name == "reserved":
            c.reserved[2] = v
        else:
            setattr(c, name, v)
    return ctypes.byref(c)


def route(cfg=None, bwd=False, **k):
    a = dict(type=0, logits=FAKE, ldl=24, bias=FAKE, N=10, E=24, k=4)
    if bwd:
        a = dict(type=0, logits=FAKE, ldl=24, bias=FAKE, idx=FAKE, wt=2, dw=FAKE, N=10, E=24, k=4, cfg=cfg, dl=FAKE,
                 lddl=24, stream=None)
    else:
        a.update(cfg=cfg, idx=FAKE, wt=2, w=FAKE, counts=FAKE, stream=None)
    a.update(k)
    return getattr(som.load(), "som_route_bwd" if bwd else "som_route")(*a.values())


@pytest.mark.parametrize("bwd", [False, True])
def test_route_refusals(bwd):
    for bad in (dict(type=3), dict(wt=-1), dict(logits=None), dict(idx=None), dict(ldl=23), dict(N=-1), dict(N=1 << 30),
                dict(E=0), dict(E=4097, ldl=5000), dict(k=0), dict(k=25), dict(k=33, E=64, ldl=64),
                dict(logits=ctypes.c_void_p((1 << 20) + 2)), dict(idx=ODD), dict(bias=ODD)):
        assert route(bwd=bwd, **bad) == INVALID, bad
    for bad in (dict(score=2), dict(renorm=2), dict(groups=5), dict(groups=-1), dict(groups=4, group_top=5),
                dict(groups=4, group_top=-1), dict(reserved=1)):
        assert route(cfg=config(**bad), bwd=bwd) == INVALID, bad
    assert route(cfg=config(groups=65), bwd=bwd, E=130, ldl=130) == INVALID
    if bwd:
        assert route(bwd=True, dw=None) == INVALID and route(bwd=True, dl=None) == INVALID
        assert route(bwd=True, lddl=23) == INVALID and route(bwd=True, dl=ODD) == INVALID
        assert route(bwd=True, N=0, logits=None, idx=None, dw=None, dl=None) == som.SOM_OK
    else:
        assert route(w=None) == INVALID and route(counts=ODD) == INVALID
        assert route(N=0, logits=None, idx=None, w=None, counts=None) == som.SOM_OK


def experts(bwd=False, **k):
    size = dict(N=10, k=2, E=8, D=64, F=96)
    size.update({n: k.pop(n) for n in list(k) if n in size})
    a = dict(type=2, X=FAKE, ldx=64, idx=FAKE, w=FAKE, W1=FAKE)
    if bwd:
        a.update(W2=FAKE, b2=FAKE, act=2, dout=FAKE, lddo=64, dX=FAKE, lddx=64, dw=FAKE, dW1=FAKE, db1=FAKE, dW2=FAKE,
                 db2=FAKE, **size, ws=FAKE, bytes=BIG, stream=None)
    else:
        a.update(b1=FAKE, W2=FAKE, b2=FAKE, act=2, res=FAKE, ldr=64, out=FAKE, ldo=64, **size, keep=0, ws=FAKE,
                 bytes=BIG, stream=None)
    a.update(k)
    return getattr(som.load(), "som_experts_bwd" if bwd else "som_experts")(*a.values())


SIZES = (dict(N=-1), dict(k=0), dict(k=33), dict(E=0), dict(E=1025), dict(D=0), dict(F=0), dict(F=1 << 24),
         dict(D=1 << 24), dict(N=1 << 29, k=2), dict(N=1 << 30, k=1))


@pytest.mark.parametrize("bwd", [False, True])
def test_experts_refusals(bwd):
    lib = som.load()
    for bad in SIZES + (dict(type=0), dict(act=4), dict(X=None), dict(idx=None), dict(w=None), dict(W1=None),
                        dict(W2=None), dict(ldx=63), dict(X=ODD), dict(idx=ODD), dict(W1=ODD), dict(b2=ODD)):
        assert experts(bwd, **bad) == INVALID, bad
    need = lib.som_experts_workspace_bytes(10, 2, 8, 64, 96, 1 if bwd else 0)
    assert experts(bwd, bytes=need - 1) == WORKSPACE and experts(bwd, ws=None) == WORKSPACE
    if bwd:
        assert experts(True, dout=None) == INVALID and experts(True, lddo=63) == INVALID
        assert experts(True, lddx=63) == INVALID and experts(True, dW2=ODD) == INVALID
    else:
        assert experts(out=None) == INVALID and experts(ldo=63) == INVALID and experts(ldr=63) == INVALID
        assert experts(keep=2) == INVALID
        assert experts(N=0, X=None, idx=None, w=None, W1=None, W2=None, out=None, ws=None, bytes=0) == som.SOM_OK


def test_experts_workspace():
    lib = som.load()
    n = lib.som_experts_workspace_bytes(1000, 2, 8, 64, 96, 0)
    assert n % 256 == 0 and n >= 2000 * (96 * 2 + 64 * 4 + 12)
    assert lib.som_experts_workspace_bytes(1000, 2, 8, 64, 96, 1) >= n + 2000 * 96 * 4
    assert lib.som_experts_workspace_bytes(2000, 2, 8, 64, 96, 0) > n
    assert lib.som_experts_workspace_bytes(0, 1, 1, 1, 1, 0) > 0
    for bad in SIZES:
        a = dict(N=10, k=2, E=8, D=64, F=96)
        a.update(bad)
        assert lib.som_experts_workspace_bytes(*a.values(), 0) == 0, bad
    assert lib.som_experts_workspace_bytes(10, 2, 8, 64, 96, 2) == 0


def test_clip_refusals():
    lib = som.load()
    n = 3
    ptr, sizes, types = (ctypes.c_void_p * n)(1 << 20, 1 << 20, 1 << 20), (ctypes.c_int64 * n)(5, 0, 70000), (ctypes.c_int32 * n)(0, 1, 2)
    need = lib.som_clip_workspace_bytes(sizes, n)
    assert need % 256 == 0 and need > 0

    def clip(**k):
        a = dict(ins=ptr, outs=ptr, sizes=sizes, types=types, n=n, max_norm=1.0, norm=FAKE, ws=FAKE, bytes=BIG, stream=None)
        a.update(k)
        return lib.som_clip(*a.values())

    for bad in (dict(ins=None), dict(outs=None), dict(sizes=None), dict(types=None), dict(n=-1), dict(max_norm=0.0),
                dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(max_norm=float("inf")), dict(norm=None),
                dict(norm=ODD), dict(sizes=(ctypes.c_int64 * n)(5, -1, 7)), dict(types=(ctypes.c_int32 * n)(0, 1, 3)),
                dict(ins=(ctypes.c_void_p * n)(1 << 20, 1 << 20, None)),
                dict(outs=(ctypes.c_void_p * n)(1 << 20, 1 << 20, (1 << 20) + 1))):
        assert clip(**bad) == INVALID, bad
    assert clip(bytes=need - 1) == WORKSPACE and clip(ws=None) == WORKSPACE
    assert lib.som_clip_workspace_bytes((ctypes.c_int64 * 1)(-5), 1) == 0


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "som_dense.h")).read()
    for name, value in (("SOM_F32", dense.F32), ("SOM_F16", dense.F16), ("SOM_BF16", dense.BF16),
                        ("SOM_ACT_NONE", dense._ACTS["none"]), ("SOM_ACT_RELU", dense._ACTS["relu"]),
                        ("SOM_ACT_GELU", dense._ACTS["gelu"]), ("SOM_ACT_SILU", dense._ACTS["silu"]),
                        ("SOM_SCORE_SOFTMAX", dense._SCORES["softmax"]),
                        ("SOM_SCORE_SIGMOID", dense._SCORES["sigmoid"])):
        assert re.search(rf"\b{name} = {value}\b", text), name


def test_binding_refuses_what_is_not_on_the_gpu_or_of_another_kind():
    x, W = torch.zeros(4, 8, dtype=torch.float16), torch.zeros(8, 6, dtype=torch.float16)
    for call in (lambda: dense.linear(x, W, out=torch.zeros(4, 6, dtype=torch.float16)),
                 lambda: dense.route(torch.zeros(4, 8), 2, out=(torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))),
                 lambda: dense.clip([x], 1.0)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        dense.linear(x.float(), W.float())  # fp32 rows
    with pytest.raises(TypeError):
        dense.linear([1.0], W)
    with pytest.raises(ValueError):
        dense.linear(x, torch.zeros(7, 6, dtype=torch.float16))
    with pytest.raises(TypeError):
        dense.route(torch.zeros(4, 8, dtype=torch.float64), 2)
    with pytest.raises(ValueError):
        dense.experts(x, torch.zeros(4, 2, dtype=torch.int32), x[:, :2], torch.zeros(3, 9, 5), None, None, None)
    with pytest.raises(ValueError):
        dense.clip([], 1.0)
    with pytest.raises(ValueError):
        dense.experts_workspace_bytes(4, 2, 0, 8, 8)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_header_compiles_as_c11_and_links(tmp_path):
    src = tmp_path / "use_dense.c"
    src.write_text(r"""
#include "som_dense.h"
#include <string.h>
int main(void)
{
    som_route_config cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.score = SOM_SCORE_SIGMOID;
    cfg.groups = 3;
    if (som_route(SOM_F32, NULL, 8, NULL, 4, 8, 2, &cfg, NULL, SOM_BF16, NULL, NULL, NULL) != SOM_ERR_INVALID_ARG) return 1;
    if (strstr(som_last_error(), "groups") == NULL) return 2;
    if (som_experts_workspace_bytes(10, 2, 8, 64, 96, 1) == 0) return 3;
    const int64_t sizes[2] = {3, 70000};
    if (som_clip_workspace_bytes(sizes, 2) < 256 + 3 * sizeof(double)) return 4;
    if (som_linear(SOM_F16, NULL, 1, NULL, 1, NULL, SOM_F32, SOM_ACT_GELU, NULL, 0, NULL, 1, SOM_F32, NULL, 0, 0, 1, 1,
                   NULL) != SOM_OK) return 5;
    return 0;
}
""")
    exe = str(tmp_path / "use_dense")
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", f"-I{ROOT}/include", str(src),
                        "-o", exe, f"-L{PKG}", "-lsom", f"-Wl,-rpath,{PKG}"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([exe], timeout=120).returncode == 0
