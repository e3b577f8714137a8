"""som_experts and its gradients against an expert-by-expert form in 64 bits, on the GPU."""
import pytest
import torch

import paper_2608_24067_amd.dense as dense
from dense_ref import LIP, U, act, check, curve, slope, sums, wide

pytestmark = pytest.mark.gpu


def case(seed, N, k, E, D, F, dtype, dev, empty=0.1, lonely=False, ones=False):
    g = torch.Generator().manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g) * scale).to(dtype).to(dev)

    s = dict(x=normal(N, D), W1=normal(E, D, F, scale=D ** -0.5), b1=normal(E, F, scale=0.2),
             W2=normal(E, F, D, scale=F ** -0.5), b2=normal(E, D, scale=0.2))
    idx = torch.randint(0, E, (N, k), generator=g, dtype=torch.int32)  # an expert may stand twice in a row
    if lonely:
        idx[:] = E - 1  # one expert takes all
    idx[torch.rand(N, k, generator=g) < empty] = -1
    if N > 2:
        idx[N // 2] = -1  # a row that no expert takes
        idx[0, 0] = E + 3  # an index that is none
    s["idx"] = idx.to(dev)
    s["w"] = (torch.rand(N, k, generator=g) + 0.1).to(dtype).to(dev)
    s["w"][N - 1] = 0
    return s, g


def forms(s, a, res):
    """out and the bound of what is rounded or summed before it."""
    x, w, idx = wide(s["x"]), wide(s["w"]), s["idx"].cpu()
    E, u = s["W1"].shape[0], U[s["x"].dtype]
    D, F = s["W1"].shape[1:]
    out = wide(res).clone() if res is not None else torch.zeros_like(x)
    bound = 2.0 ** -20 * (out.abs() + 1)
    for e in range(E):
        n, j = (idx == e).nonzero(as_tuple=True)
        if not n.numel():
            continue
        W1, W2 = wide(s["W1"][e]), wide(s["W2"][e])
        b1 = wide(s["b1"][e]) if s["b1"] is not None else torch.zeros(F, dtype=torch.float64)
        b2 = wide(s["b2"][e]) if s["b2"] is not None else torch.zeros(D, dtype=torch.float64)
        z = x[n] @ W1 + b1
        dz = sums(D + 1, x[n].abs() @ W1.abs() + b1.abs())
        we = w[n, j][:, None]
        h = we * act(a, z)
        dh = u * h.abs() + we * (LIP * dz + 2.0 ** -20 * z.abs().clamp_min(1))
        out.index_add_(0, n, h @ W2 + we * b2)
        bound.index_add_(0, n, dh @ W2.abs() + sums(F + 2, (h.abs() + dh) @ W2.abs() + we * b2.abs()))
    return out, bound


SHAPES = [
    (1, 1, 1, 8, 8), (1, 2, 4, 64, 128), (1, 2, 64, 256, 512), (3, 2, 5, 31, 33), (4, 4, 3, 24, 40),
    (17, 3, 7, 65, 130), (33, 4, 32, 128, 96), (100, 2, 8, 72, 200), (700, 2, 3, 136, 264), (2000, 1, 4, 100, 50),
    (600, 32, 2, 64, 72), (40, 2, 1024, 16, 24),
]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,k,E,D,F", SHAPES)
def test_experts(dev, dtype, N, k, E, D, F):
    for a, lonely in (("gelu", False), ("none", True)):
        s, g = case(31, N, k, E, D, F, dtype, dev, lonely=lonely)
        out = dense.experts(**s, act=a, residual=s["x"])
        ref, bound = forms(s, a, s["x"])
        check(out, ref, bound, f"out, {a}")


def test_tiles_of_every_size(dev):
    # enough rows and columns for tiles of 128 and 256, aligned or not
    for N, k, E, D, F, off in ((1500, 2, 5, 1024, 1160, 0), (5000, 2, 4, 2048, 2056, 0), (5000, 2, 4, 2048, 2056, 1)):
        s, g = case(32, N, k, E, D, F, torch.bfloat16, dev, empty=0.3)
        if off:  # the rows start at any element
            buf = torch.empty(N * (D + off), dtype=torch.bfloat16, device=dev).view(N, D + off)[:, off:]
            buf.copy_(s["x"])
            s["x"] = buf
        out = dense.experts(**s, act="silu")
        ref, bound = forms(s, "silu", None)
        check(out, ref, bound, f"out {N}")


def test_without_biases_in_place_and_strided(dev):
    s, g = case(33, 50, 2, 6, 64, 80, torch.float16, dev)
    s["b1"] = s["b2"] = None
    buf = torch.full((50, 96), float("nan"), dtype=torch.float16, device=dev)
    res = buf[:, 8:72]
    res.copy_(torch.randn(50, 64, generator=g).half())
    ref, bound = forms(s, "relu", res)
    dense.experts(**s, act="relu", residual=res, out=res)
    check(res, ref, bound, "in place")
    assert torch.isnan(buf[:, :8]).all() and torch.isnan(buf[:, 72:]).all()


def gradients(s, a, dout, pre):
    """By the formulas, with the slopes at the z that is held in the rows' type; and their bounds."""
    x, w, idx, g = wide(s["x"]), wide(s["w"]), s["idx"].cpu(), wide(dout)
    E, u = s["W1"].shape[0], U[s["x"].dtype]
    D, F = s["W1"].shape[1:]
    ref = {n: torch.zeros(s[n].shape, dtype=torch.float64) for n in ("x", "w", "W1", "b1", "W2", "b2")}
    off = {n: torch.zeros_like(t) for n, t in ref.items()}
    for e in range(E):
        n, j = (idx == e).nonzero(as_tuple=True)
        if not n.numel():
            continue
        W1, W2, b1, b2 = (wide(s[q][e]) for q in ("W1", "W2", "b1", "b2"))
        we, ge, xe = w[n, j][:, None], g[n], x[n]
        z = xe @ W1 + b1
        ez = u * z.abs() + sums(D + 1, xe.abs() @ W1.abs() + b1.abs())  # z as held
        h, sl = act(a, z), slope(a, z)
        eh = LIP * ez + 2.0 ** -20 * z.abs().clamp_min(1)
        es = curve(a) * ez + 2.0 ** -20 * z.abs().clamp_min(1)
        if a == "relu":
            es = es + (z.abs() <= ez).double()  # the kink may lie between z and its rounding
        q = ge @ W2.T
        eq = sums(D, ge.abs() @ W2.abs().T)
        dz = we * q * sl
        edz = we * (eq * (sl.abs() + es) + q.abs() * es)
        edz = edz + u * (dz.abs() + edz)
        nj = (n, j)
        ref["w"][nj] = (h * q).sum(1) + ge @ b2
        t = (h.abs() + eh) * (q.abs() + eq)
        off["w"][nj] = (eh * q.abs() + h.abs() * eq + eh * eq).sum(1) + sums(D + F, t.sum(1) + ge.abs() @ b2.abs())
        ref["x"].index_add_(0, n, dz @ W1.T)
        off["x"].index_add_(0, n, edz @ W1.abs().T + sums(F + 34, (dz.abs() + edz) @ W1.abs().T))
        ref["W1"][e], ref["b1"][e] = xe.T @ dz, dz.sum(0)
        c = len(n)
        off["W1"][e] = xe.abs().T @ edz + sums(c, xe.abs().T @ (dz.abs() + edz))
        off["b1"][e] = edz.sum(0) + sums(c, (dz.abs() + edz).sum(0))
        hw = we * h
        ehw = we * (eh + u * h.abs())
        ref["W2"][e], ref["b2"][e] = hw.T @ ge, (we * ge).sum(0)
        off["W2"][e] = ehw.T @ ge.abs() + sums(c, (hw.abs() + ehw).T @ ge.abs())
        off["b2"][e] = sums(c, (we * ge.abs()).sum(0))
    return ref, off


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,k,E,D,F", SHAPES + [(3000, 2, 2, 1032, 520), (5000, 2, 4, 2048, 1160)])
def test_experts_gradients(dev, dtype, N, k, E, D, F):
    a = ["gelu", "silu", "relu", "none"][(N + E) % 4]
    s, g = case(34, N, k, E, D, F, dtype, dev)
    dout = torch.randn(N, D, generator=g).to(dtype).to(dev)
    ws = torch.empty(dense.experts_workspace_bytes(N, k, E, D, F, keep=True), dtype=torch.uint8, device=dev)
    dense.experts(**s, act=a, keep=True, workspace=ws)
    got = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], dout, act=a, workspace=ws)
    ref, off = gradients(s, a, dout, None)
    for name, t in zip(("x", "w", "W1", "b1", "W2", "b2"), got):
        check(t, ref[name], off[name], f"d{name}, {a}")
    # the workspace serves again, for a part of the gradients, with the same bits
    for i in range(6):
        out = [None] * 6
        out[i] = torch.full_like(got[i], float("nan"))
        part = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], dout, act=a, out=out, workspace=ws)
        assert torch.equal(part[i], got[i])


@pytest.mark.parametrize("a", ["gelu", "silu", "none"])
def test_experts_gradients_against_differences(dev, a):
    s, g = case(35, 9, 2, 3, 16, 24, torch.float16, dev, empty=0.0)
    dout = torch.randn(9, 16, generator=g).half().to(dev)
    ws = torch.empty(dense.experts_workspace_bytes(9, 2, 3, 16, 24, keep=True), dtype=torch.uint8, device=dev)
    dense.experts(**s, act=a, keep=True, workspace=ws)
    got = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], dout, act=a, workspace=ws)
    names = ("x", "w", "W1", "b1", "W2", "b2")
    args = {n: wide(s[n]) for n in names}
    idx = s["idx"].cpu().long()

    def f(t):
        total = 0.0
        for n in range(9):
            for j in range(2):
                e = int(idx[n, j])
                if 0 <= e < 3:
                    y = act(a, t["x"][n] @ t["W1"][e] + t["b1"][e]) @ t["W2"][e] + t["b2"][e]
                    total = total + t["w"][n, j] * (y * wide(dout)[n]).sum()
        return float(total)

    h = 1e-6
    _, off = gradients(s, a, dout, None)
    for name, grad in zip(names, got):
        v = torch.randn(args[name].shape, generator=g, dtype=torch.float64)
        diff = (f({**args, name: args[name] + h * v}) - f({**args, name: args[name] - h * v})) / (2 * h)
        room = ((off[name] + U[torch.float16] * (wide(grad).abs() + off[name])) * v.abs()).sum()
        assert abs(diff - float((wide(grad) * v).sum())) <= float(room) + 1e-6


def test_bad_values_stay_in_their_rows(dev):
    s, g = case(36, 300, 2, 4, 64, 96, torch.bfloat16, dev)
    clean = dense.experts(**s)
    s["x"][150 - 1] = float("nan")
    s["x"][7] = float("inf")
    got = dense.experts(**s)
    keep = torch.ones(300, dtype=torch.bool, device=dev)
    keep[149] = keep[7] = False
    assert torch.equal(got[keep], clean[keep])


def test_no_rows_and_no_expert(dev):
    s, g = case(37, 4, 2, 3, 32, 40, torch.float16, dev)
    s["idx"].fill_(-1)
    assert torch.equal(dense.experts(**s, residual=s["x"]), s["x"])
    ws = torch.empty(dense.experts_workspace_bytes(4, 2, 3, 32, 40, keep=True), dtype=torch.uint8, device=dev)
    dense.experts(**s, keep=True, workspace=ws)
    grads = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], s["x"], workspace=ws)
    assert not any(bool(t.any()) for t in grads)
    none = {n: (t[:0] if n in ("x", "idx", "w") else t) for n, t in s.items()}
    assert dense.experts(**none).shape == (0, 32)
    ws = torch.empty(dense.experts_workspace_bytes(0, 2, 3, 32, 40, keep=True), dtype=torch.uint8, device=dev)
    out = [torch.full_like(s[n], float("nan")) for n in ("W1", "b1", "W2", "b2")]
    dense.experts_bwd(none["x"], none["idx"], none["w"], s["W1"], s["W2"], s["b2"], none["x"], workspace=ws,
                      out=[None, None] + out)
    assert not any(bool(t.any()) for t in out)


def test_same_bits_on_another_stream(dev):
    s, g = case(38, 900, 2, 8, 128, 256, torch.bfloat16, dev)
    first = dense.experts(**s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = dense.experts(**s)
    torch.cuda.synchronize()
    assert torch.equal(first, again)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,k,E,D,F", [
    (1, 2, 4, 700, 900), (2, 3, 8, 1030, 515), (5, 3, 16, 2048, 300), (1, 1, 3, 1000, 3), (4, 4, 2, 5, 600),
    (16, 1, 5, 777, 1025),
])
def test_few_pairs_whose_reductions_are_split(dev, dtype, N, k, E, D, F):
    for a in ("silu", "gelu"):
        s, g = case(39, N, k, E, D, F, dtype, dev, empty=0.0 if N == 1 else 0.1)
        if N == 1:
            s["w"].fill_(0.75)
        out = dense.experts(**s, act=a, residual=s["x"])
        ref, bound = forms(s, a, s["x"])
        check(out, ref, bound, f"out, {a}")


@pytest.mark.parametrize("N,k,E", [(3000, 1, 1024), (2049, 1, 17), (1100, 2, 300), (70000, 1, 5)])
def test_orders_of_many_pairs(dev, N, k, E):
    # the identity as experts: every row comes back as often as its weights say
    g = torch.Generator().manual_seed(40)
    x = torch.randn(N, 8, generator=g).half().to(dev)
    idx = torch.randint(-1, E, (N, k), generator=g, dtype=torch.int32).to(dev)
    w = torch.ones(N, k, dtype=torch.float16, device=dev)
    eye = torch.eye(8, dtype=torch.float16, device=dev).expand(E, 8, 8).contiguous()
    scale = (1 + torch.arange(E, device=dev) % 7).half()
    out = dense.experts(x, idx, w, eye * scale[:, None, None], None, eye, None, act="none")
    times = (scale[idx.clamp_min(0).long()].float() * (idx >= 0)).sum(1, keepdim=True)
    # powers and small multiples of 11-bit values: each product is rounded to fp16 once, and so is the sum
    assert bool(((out.float() - x.float() * times).abs() <= 2.0 ** -10 * (k + 1) * x.float().abs() * times + 1e-6).all())


def test_weights_past_32_bit_offsets(dev):
    # 2.5 billion weights a matrix; only the experts that are met are filled
    N, k, E, D, F = 6, 2, 600, 1024, 4096
    g = torch.Generator().manual_seed(41)
    met = [0, 299, 511, 599]
    W1, W2 = (torch.empty(E, *d, dtype=torch.bfloat16, device=dev) for d in ((D, F), (F, D)))
    for e in met:
        W1[e] = (torch.randn(D, F, generator=g) * D ** -0.5).bfloat16()
        W2[e] = (torch.randn(F, D, generator=g) * F ** -0.5).bfloat16()
    x = torch.randn(N, D, generator=g).bfloat16().to(dev)
    for rows in (N, 400):  # few pairs, and tiles
        idx = torch.tensor(met, dtype=torch.int32)[torch.randint(0, 4, (rows, k), generator=g)].to(dev)
        xs = x[torch.arange(rows) % N].contiguous()
        w = torch.full((rows, k), 0.5, dtype=torch.bfloat16, device=dev)
        out = dense.experts(xs, idx, w, W1, None, W2, None, act="relu")
        ref = torch.zeros(rows, D, device=dev)
        size = torch.zeros(rows, D, device=dev)
        for e in met:
            hit = (idx == e).float().sum(1, keepdim=True) * 0.5
            h = torch.relu(xs.float() @ W1[e].float())
            ref += hit * (h @ W2[e].float())
            size += hit * (h @ W2[e].float().abs())
        # the inner rows are rounded once (2^-8 of them at most), the results once
        assert bool(((out.float() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-4).all())
        del ref, size
    del W1, W2
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,k,E,D,F", [
    (12, 2, 64, 1024, 136),  # 24 pairs, each by itself, both reductions split
    (32, 2, 64, 72, 520),    # 64 of them
    (33, 2, 70, 65, 131),    # 66: ordered
    (16, 4, 60, 40, 48),     # more than experts: ordered
    (20, 4, 64, 520, 72),    # a tile a CU: the tiles of 32 rows
    (21, 4, 64, 515, 75),    # which odd rows do not take
])
def test_few_rows_an_expert(dev, dtype, N, k, E, D, F):
    s, g = case(41, N, k, E, D, F, dtype, dev)
    out = dense.experts(**s, act="silu", residual=s["x"])
    ref, bound = forms(s, "silu", s["x"])
    check(out, ref, bound, "out")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("N,k,E,D,F", [
    (127, 1, 16, 1024, 520), (128, 2, 32, 512, 512), (116, 1, 13, 515, 777), (70, 2, 24, 264, 1032),
    (40, 1, 12, 136, 1100), (1300, 2, 9, 128, 264), (2600, 2, 5, 1024, 2056),
])
def test_gradients_where_one_expert_takes_most_rows(dev, dtype, N, k, E, D, F):
    # few rows an expert on average (the first five), tiles of 32, 128 and 256; a workspace that holds no number
    s, g = case(44, N, k, E, D, F, dtype, dev, empty=0.0)
    loads = torch.full((N * k,), E // 2, dtype=torch.int32)
    loads[:E - 1] = torch.tensor([e for e in range(E) if e != E // 2], dtype=torch.int32)
    s["idx"] = loads[torch.randperm(N * k, generator=g)].view(N, k).to(dev)
    dout = torch.randn(N, D, generator=g).to(dtype).to(dev)
    ws = torch.full((dense.experts_workspace_bytes(N, k, E, D, F, keep=True),), 255, dtype=torch.uint8, device=dev)
    dense.experts(**s, act="silu", keep=True, workspace=ws)
    got = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], dout, act="silu", workspace=ws)
    ref, off = gradients(s, "silu", dout, None)
    for name, t in zip(("x", "w", "W1", "b1", "W2", "b2"), got):
        check(t, ref[name], off[name], f"d{name}")


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("D,F", [(3, 12), (5, 64), (7, 100), (12, 5), (64, 3), (100, 7), (7, 8), (300, 5), (6, 700)])
@pytest.mark.parametrize("N", [2, 40])  # few pairs, and ordered ones
def test_fewer_than_eight_features(dev, dtype, N, D, F):
    s, g = case(45, N, 2, 9, D, F, dtype, dev, empty=0.0)
    out = dense.experts(**s, act="gelu", residual=s["x"])
    ref, bound = forms(s, "gelu", s["x"])
    check(out, ref, bound, "out")


def test_weights_gradient_of_more_rows_than_a_grid_holds_along_x(dev):
    # 64 threads a row; whole numbers throughout, so that every value is exact
    N, D = (1 << 26) + 3, 8
    x = torch.randint(-2, 3, (N, D), dtype=torch.int8, device=dev).half()
    dout = torch.randint(-2, 3, (N, D), dtype=torch.int8, device=dev).half()
    idx = torch.randint(0, 2, (N, 1), dtype=torch.int32, device=dev)
    w = torch.ones(N, 1, dtype=torch.float16, device=dev)
    eye = torch.eye(D, dtype=torch.float16, device=dev).expand(2, D, D).contiguous()
    W1 = eye * torch.tensor([1.0, 2.0], device=dev).half()[:, None, None]
    ws = torch.empty(dense.experts_workspace_bytes(N, 1, 2, D, D, keep=True), dtype=torch.uint8, device=dev)
    out = dense.experts(x, idx, w, W1, None, eye, None, act="none", keep=True, workspace=ws)
    times = (1 + idx).half()
    assert torch.equal(out, x * times)
    got = [torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))] + [None] * 4
    dense.experts_bwd(x, idx, w, W1, eye, None, dout, act="none", out=got, workspace=ws)
    assert torch.equal(got[0], dout * times)
    assert torch.equal(got[1], (out * dout).sum(1, keepdim=True))
    del x, dout, idx, w, ws, out, times, got
    torch.cuda.empty_cache()


def test_gradients_of_more_tiles_than_a_grid_holds_along_x(dev):
    # 1,024 experts of 2^14 tiles each, two of them met
    N, E, D, F = 4, 1024, 1, 1 << 21
    g = torch.Generator().manual_seed(46)
    W1, W2 = torch.zeros(E, D, F, dtype=torch.float16, device=dev), torch.zeros(E, F, D, dtype=torch.float16, device=dev)
    for e in (5, E - 1):
        W1[e, 0] = torch.randint(-2, 3, (F,), generator=g).half()
        W2[e, :, 0] = torch.randint(-1, 2, (F,), generator=g).half() * 2.0 ** -10
    idx = torch.tensor([[5], [E - 1], [E - 1], [-1]], dtype=torch.int32, device=dev)
    x = torch.tensor([[1.0], [2.0], [-1.0], [1.0]], device=dev).half()
    dout = torch.tensor([[2.0], [-1.0], [1.0], [3.0]], device=dev).half()
    w = torch.ones(N, 1, dtype=torch.float16, device=dev)
    ws = torch.empty(dense.experts_workspace_bytes(N, 1, E, D, F, keep=True), dtype=torch.uint8, device=dev)
    dense.experts(x, idx, w, W1, None, W2, None, act="none", keep=True, workspace=ws)
    grads = [None, None, torch.full_like(W1, float("nan")), None, torch.full_like(W2, float("nan")), None]
    dense.experts_bwd(x, idx, w, W1, W2, None, dout, act="none", out=grads, workspace=ws)
    # by hand: dW1 = x (dout W2), dW2 = (x W1) dout, all exact
    dW1, dW2 = grads[2], grads[4]
    assert torch.equal(dW1[5, 0], 2 * W2[5, :, 0]) and torch.equal(dW2[5, :, 0], 2 * W1[5, 0])
    assert torch.equal(dW1[E - 1, 0], -3 * W2[E - 1, :, 0]) and torch.equal(dW2[E - 1, :, 0], -3 * W1[E - 1, 0])
    for t in (dW1, dW2):
        t[5], t[E - 1] = 0, 0
        assert not t.any()
    del W1, W2, dW1, dW2, grads, ws
    torch.cuda.empty_cache()


@pytest.mark.parametrize("size", [1e-3, 1e-4, 1e-5, 100.0])
@pytest.mark.parametrize("N,k,E,D,F", [(2, 2, 4, 264, 520), (30, 2, 64, 200, 136), (33, 2, 20, 128, 96),
                                       (900, 2, 5, 72, 200), (3000, 2, 2, 1032, 520)])
def test_weights_of_other_sizes_than_one(dev, size, N, k, E, D, F):
    # fp16: w act(z) would be subnormal, or beyond the type, where act(z) and the results are neither
    dtype = torch.float16
    s, g = case(47, N, k, E, D, F, dtype, dev, empty=0.0)
    s["x"] = s["x"] * (64 if size > 1 else 1)
    s["W2"] = (s["W2"].float() * (2.0 ** -9 if size > 1 else 64 if size < 2e-4 else 8)).to(dtype)
    s["w"] = ((torch.rand(N, k, generator=g) + 0.5) * size * (10 if size > 1 else 1)).to(dtype).to(dev)
    out = dense.experts(**s, act="relu")
    ref, bound = forms(s, "relu", None)
    bound = bound - 2.0 ** -20 + 2.0 ** -40  # no residual: nothing of size one is rounded
    check(out, ref, bound, "out")
    dout = torch.randn(N, D, generator=g).to(dtype).to(dev)
    ws = torch.empty(dense.experts_workspace_bytes(N, k, E, D, F, keep=True), dtype=torch.uint8, device=dev)
    check(dense.experts(**s, act="relu", keep=True, workspace=ws), ref, bound, "out, kept")
    dx, dw, dW1, db1, dW2, db2 = dense.experts_bwd(s["x"], s["idx"], s["w"], s["W1"], s["W2"], s["b2"], dout, act="relu",
                                                   workspace=ws)
    ref, off = gradients(s, "relu", dout, None)
    check(dw, ref["w"], off["w"], "dw")
    if size < 1:  # (sums of large weights lie beyond fp16)
        check(db2, ref["b2"], off["b2"], "db2")
        # w act(z) is held in fp16 for dW2: half its smallest subnormal may be lost of each
        grain = torch.zeros(E, D, dtype=torch.float64)
        grain.index_add_(0, s["idx"].cpu().reshape(-1).clamp(0, E - 1).long(),
                         wide(dout).abs().repeat_interleave(k, 0) * 2.0 ** -25)
        check(dW2, ref["W2"], off["W2"] + grain[:, None, :], "dW2")
