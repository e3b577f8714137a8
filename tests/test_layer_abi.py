"""CPU tests of layer norm, AdamW and the 4-bit operators (include/som_dense.h): workspace queries and every argument
check that returns before anything reaches the GPU, through the C ABI and through the binding; and the plain forms that
the GPU tests compare with, against themselves."""
import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import layer_ref as ref
import paper_2608_24067_amd.dense as dense
import paper_2608_24067_amd.som as som

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2608_24067_amd")
FAKE = ctypes.c_void_p(1 << 20)  # never followed: every call here is refused or has nothing to do
ODD = ctypes.c_void_p((1 << 20) + 1)
BIG = 1 << 40
INVALID, WORKSPACE = som.SOM_ERR_INVALID_ARG, som.SOM_ERR_WORKSPACE


def norm(**k):
    a = dict(type=2, X=FAKE, ldx=64, w=FAKE, b=FAKE, wt=0, eps=1e-5, Y=FAKE, ldy=64, yt=2, stats=FAKE, N=10, D=64, stream=None)
    a.update(k)
    return som.load().som_layer_norm(*a.values())


def norm_bwd(**k):
    a = dict(type=2, X=FAKE, ldx=64, w=FAKE, wt=0, dY=FAKE, lddy=64, yt=2, stats=FAKE, add=FAKE, lda=64, dX=FAKE, lddx=64,
             dw=FAKE, db=FAKE, N=10, D=64, ws=FAKE, bytes=BIG, stream=None)
    a.update(k)
    return som.load().som_layer_norm_bwd(*a.values())


def test_layer_norm_refusals():
    for bad in (dict(type=3), dict(yt=1), dict(yt=0), dict(yt=5), dict(wt=1), dict(X=None), dict(Y=None), dict(ldx=63),
                dict(ldy=63), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf), dict(eps=math.nan), dict(eps=1e-39),
                dict(N=-1), dict(N=1 << 30), dict(D=0), dict(D=1 << 20, ldx=1 << 21, ldy=1 << 21), dict(X=ODD), dict(Y=ODD),
                dict(w=ctypes.c_void_p((1 << 20) + 2)), dict(b=ODD), dict(stats=ctypes.c_void_p((1 << 20) + 4))):
        assert norm(**bad) == INVALID, bad
        assert som.last_error().startswith("som_layer_norm"), som.last_error()
    assert norm(N=0, X=None, Y=None) == som.SOM_OK
    lib = som.load()
    for bad in (dict(type=3), dict(yt=1), dict(wt=1), dict(X=None), dict(dY=None), dict(stats=None), dict(ldx=63),
                dict(lddy=63), dict(lda=63), dict(lddx=63), dict(N=-1), dict(D=0), dict(dX=ODD), dict(add=ODD), dict(dY=ODD),
                dict(dw=ODD), dict(db=ODD)):
        assert norm_bwd(**bad) == INVALID, bad
    need = lib.som_layer_norm_bwd_workspace_bytes(10, 64)
    assert need % 256 == 0 and need >= 2 * 64 * 4
    assert norm_bwd(bytes=need - 1) == WORKSPACE and norm_bwd(ws=None) == WORKSPACE
    assert norm_bwd(ws=ctypes.c_void_p((1 << 20) + 128)) == WORKSPACE
    assert lib.som_layer_norm_bwd_workspace_bytes(1 << 20, 64) > lib.som_layer_norm_bwd_workspace_bytes(1000, 64)
    for bad in ((-1, 64), (10, 0), (1 << 30, 64), (10, 1 << 20)):
        assert lib.som_layer_norm_bwd_workspace_bytes(*bad) == 0


class Tensor(ctypes.Structure):
    """som_adamw_tensor"""
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scales", "v_scales", "master")] + [
        ("size", ctypes.c_int64), ("type", ctypes.c_int32), ("grad_type", ctypes.c_int32)]


def adamw(tensor=None, count=1, **k):
    t = Tensor()
    for n in ("param", "grad", "m", "v", "m_scales", "v_scales", "master"):
        setattr(t, n, 1 << 20)
    t.size, t.type, t.grad_type = 1000, 2, 0
    for n, v in (tensor or {}).items():
        setattr(t, n, v)
    c = dense._AdamwConfig(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0, step=1, bits=32)
    for n, v in k.items():
        if n == "reserved":
            c.reserved[3] = v
        else:
            setattr(c, n, v)
    return som.load().som_adamw((Tensor * 1)(t), count, ctypes.byref(c), None)


def test_adamw_refusals():
    for bad in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(weight_decay=-0.1), dict(weight_decay=math.inf),
                dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-39),
                dict(eps=1e39), dict(grad_scale=math.nan), dict(grad_scale=math.inf), dict(step=0), dict(step=-1),
                dict(step=1 << 31), dict(bits=16), dict(bits=0), dict(reserved=1), dict(norm=(1 << 20) + 2),
                dict(lr_at=(1 << 20) + 1), dict(step_at=(1 << 20) + 1), dict(count=-1)):
        assert adamw(**bad) == INVALID, bad
        assert som.last_error().startswith("som_adamw"), som.last_error()
    for bad in (dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(type=3), dict(grad_type=-1), dict(size=-1),
                dict(size=(1 << 38) + 1), dict(param=(1 << 20) + 1), dict(grad=(1 << 20) + 2), dict(m=(1 << 20) + 2),
                dict(master=(1 << 20) + 2)):
        assert adamw(bad) == INVALID, bad
    for bad in (dict(m_scales=None), dict(v_scales=None)):
        assert adamw(bad, bits=8) == INVALID, bad
    lib = som.load()
    assert lib.som_adamw(None, 1, None, None) == INVALID
    assert adamw(count=0) == som.SOM_OK
    assert adamw(dict(size=0, param=None, grad=None, m=None, v=None)) == som.SOM_OK
    t = Tensor(m=1 << 20, v=1 << 20, m_scales=1 << 20, v_scales=1 << 20, size=10)
    one, none, off = ((ctypes.c_void_p * 1)(p) for p in (1 << 20, None, (1 << 20) + 2))
    table = (Tensor * 1)(t)
    for m, v in ((none, one), (one, none), (off, one), (None, one), (one, None)):
        assert lib.som_adamw_values(table, 1, m, v, None) == INVALID
    assert lib.som_adamw_values(None, 0, None, None, None) == som.SOM_OK


def quantise(values=False, **k):
    a = dict(type=0, X=FAKE, ldx=100, columns=0, codes=FAKE, scales=FAKE, n=10, K=100, stream=None)
    a.update(k)
    lib = som.load()
    if not values:
        return lib.som_mx4_quantise(*a.values())
    return lib.som_mx4_values(a["type"], a["codes"], a["scales"], a["columns"], a["X"], a["ldx"], a["n"], a["K"], None)


@pytest.mark.parametrize("values", [False, True])
def test_mx4_refusals(values):
    for bad in (dict(type=3), dict(X=None), dict(codes=None), dict(scales=None), dict(ldx=99), dict(columns=2),
                dict(columns=1, n=101), dict(n=-1), dict(n=1 << 30), dict(K=0), dict(K=1 << 30, ldx=1 << 31), dict(X=ODD),
                dict(codes=ctypes.c_void_p((1 << 20) + 8))):
        assert quantise(values, **bad) == INVALID, bad
        assert som.last_error().startswith("som_mx4_values" if values else "som_mx4_quantise")
    assert quantise(values, n=0, X=None, codes=None, scales=None) == som.SOM_OK


def mx4_linear(**k):
    a = dict(type=2, X=FAKE, ldx=64, xs=None, w=FAKE, ws=FAKE, bias=FAKE, bias_type=0, act=0, res=FAKE, ldr=32, Y=FAKE, ldy=32,
             y_type=2, N=10, K=64, M=32, work=FAKE, bytes=BIG, stream=None)
    a.update(k)
    return som.load().som_mx4_linear(*a.values())


def test_mx4_linear_refusals():
    for bad in (dict(type=0), dict(type=3), dict(X=None), dict(w=None), dict(ws=None), dict(Y=None), dict(ldx=63), dict(ldr=31),
                dict(ldy=31), dict(act=4), dict(y_type=1), dict(bias_type=1), dict(N=-1), dict(N=1 << 30), dict(K=0), dict(M=0),
                dict(K=1 << 30), dict(M=1 << 30), dict(X=ODD), dict(Y=ODD), dict(res=ODD), dict(bias=ODD),
                dict(w=ctypes.c_void_p((1 << 20) + 8)), dict(xs=FAKE, X=ctypes.c_void_p((1 << 20) + 8))):
        assert mx4_linear(**bad) == INVALID, bad
        assert som.last_error().startswith("som_mx4_linear"), som.last_error()
    assert mx4_linear(N=0, X=None, w=None, ws=None, Y=None) == som.SOM_OK
    lib = som.load()
    for N, K, M, packed in ((1, 64, 64, 0), (33, 4096, 8192, 1), (8192, 2048, 4096, 0)):
        need = lib.som_mx4_linear_workspace_bytes(N, K, M, packed)
        assert need % 256 == 0
        if need:
            xs = FAKE if packed else None
            assert mx4_linear(N=N, K=K, M=M, ldx=K, ldr=M, ldy=M, xs=xs, bytes=need - 1) == WORKSPACE
    for bad in ((-1, 64, 64, 0), (1, 0, 64, 0), (1, 64, 0, 1), (1, 64, 64, 2)):
        assert lib.som_mx4_linear_workspace_bytes(*bad) == 0


def test_binding_refuses_what_is_not_on_the_gpu_or_of_another_kind():
    x, half = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        dense.layer_norm(x)
    with pytest.raises(TypeError):
        dense.layer_norm(x.double())
    with pytest.raises(ValueError):
        dense.layer_norm(torch.zeros(4))
    with pytest.raises(TypeError):
        dense.layer_norm_bwd(x, half, torch.zeros(4, 2, dtype=torch.float64), torch.zeros(64, dtype=torch.bfloat16))
    state = dense.adamw_state(x)
    for call in (lambda: dense.adamw([x], [x], [state], 1), lambda: dense.adamw([x], [], [state], 1),
                 lambda: dense.adamw_values([dense.adamw_state(x, 8)]), lambda: dense.adamw_state(x, 16),
                 lambda: dense.mx4_quantise(x), lambda: dense.mx4_values(dense.Mx4(torch.zeros(4, 32, dtype=torch.uint8),
                                                                               torch.zeros(4, 2, dtype=torch.uint8), 64)),
                 lambda: dense.mx4_linear(half, dense.Mx4(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 64)),
                 lambda: dense.mx4_linear(half, dense.Mx4(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8), 63))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        dense.mx4_linear(x, None)  # fp32 rows
    with pytest.raises(TypeError):
        dense.adamw_state(x.double())


def test_states_start_as_zeros():
    p = torch.randn(7, 100).to(torch.bfloat16)
    s = dense.adamw_state(p, 8, master=True)
    assert s.m.dtype == torch.uint8 and s.m.shape == p.shape and s.m_scales.shape == (3,)
    assert torch.equal(s.master, p.float()) and s.master.data_ptr() != p.data_ptr()
    assert not s.m.any() and not s.v_scales.any()
    s = dense.adamw_state(p.float(), master=True)
    assert s.master.data_ptr() != p.data_ptr() and s.m_scales is None


def test_plain_codes_of_states_keep_their_mean_and_their_largest():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=1 << 16) * np.exp(rng.normal(size=1 << 16))).astype(np.float32)
    for signed, y in ((True, x), (False, x * x)):
        total = np.zeros(y.size)
        for step in range(64):
            r = ref.random_bits(y.size, 3, 7, step).astype(np.int64)
            total += ref.values8(*ref.codes8(y, signed, r & 0xFFFF if signed else r >> 16), signed)
        one = ref.values8(*ref.codes8(y, signed, r & 0xFFFF if signed else r >> 16), signed)
        top = np.abs(y).reshape(-1, 256).max(1).repeat(256)
        assert (np.abs(one - y) <= np.abs(y) / 8 + top * 2.0 ** (-16 if signed else -32)).all()
        # 64 x 65,536 draws, each within an eighth: 8 standard deviations of their weighted mean
        off = (total / 64 - y).sum()
        assert abs(off) <= 8 * np.sqrt((y.astype(np.float64) ** 2).sum()) / 16 / 8 + np.abs(y).sum() * 2.0 ** -16


def test_plain_four_bit_codes():
    x = np.array([[0.0, 0.25, 0.26, 0.75, -0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, 6.0, 7.9, -0.2] + [0.0] * 18])
    codes, scales = ref.codes4(x)
    assert scales[0, 0] == 127
    want = [0, 0, 0.5, 1, -1, 1, 2, 2, 4, 4, 6, 6, 6, 0] + [0] * 18
    assert ref.values4(codes, scales, 32)[0].tolist() == want


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_header_compiles_as_c11_and_links(tmp_path):
    src = tmp_path / "use_layers.c"
    src.write_text(r"""
#include "som_dense.h"
#include <string.h>
int main(void)
{
    som_adamw_tensor t;
    som_adamw_config c;
    memset(&t, 0, sizeof t);
    memset(&c, 0, sizeof c);
    c.eps = 1e-8, c.beta1 = 0.9, c.beta2 = 0.999, c.grad_scale = 1, c.step = 1, c.bits = 8;
    if (som_adamw(&t, 1, &c, NULL) != SOM_OK) return 1;
    t.size = 5;
    if (som_adamw(&t, 1, &c, NULL) != SOM_ERR_INVALID_ARG) return 2;
    if (strstr(som_last_error(), "null") == NULL) return 3;
    if (som_layer_norm_bwd_workspace_bytes(100, 50) < 2 * 50 * sizeof(float)) return 4;
    if (som_mx4_quantise(SOM_F32, NULL, 8, 0, NULL, NULL, 0, 8, NULL) != SOM_OK) return 5;
    return sizeof(som_adamw_tensor) == 72 && sizeof(som_adamw_config) == 120 ? 0 : 6;
}
""")
    exe = str(tmp_path / "use_layers")
    r = subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", f"-I{ROOT}/include", str(src),
                        "-o", exe, f"-L{PKG}", "-lsom", f"-Wl,-rpath,{PKG}"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([exe], timeout=120).returncode == 0
    assert ctypes.sizeof(Tensor) == 72 == 8 * dense._ADAMW_WORDS and ctypes.sizeof(dense._AdamwConfig) == 120
