"""som_layer_norm and its backward pass against 64 bits, on the GPU."""
import math

import pytest
import torch

import layer_ref as ref
import paper_2608_24067_amd.dense as dense
from dense_ref import check, wide

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
PAIRS = [(F32, F32), (F32, F16), (F32, BF16), (F16, F16), (BF16, BF16)]
EPS = 1e-5


def strided(t, extra, offset, dev):
    """t on the device, its rows `extra` elements longer than needed and starting `offset` elements into the buffer."""
    N, D = t.shape
    flat = torch.full((N * (D + extra) + offset,), float("nan"), dtype=t.dtype, device=dev)
    out = flat[offset:].reshape(N, D + extra)[:, :D]
    return out.copy_(t)


def inputs(seed, N, D, x, y, wt, dev, extra=0, offset=0, mean=0.5, size=1.0):
    g = torch.Generator().manual_seed(seed)
    rows = (torch.randn(N, D, generator=g) * size + mean).to(x)
    w, b = (1 + 0.3 * torch.randn(D, generator=g)).to(wt), (0.3 * torch.randn(D, generator=g)).to(wt)
    dy, add = torch.randn(N, D, generator=g).to(y), torch.randn(N, D, generator=g).to(x)
    return (strided(rows, extra, offset, dev), w.to(dev), b.to(dev), strided(dy, extra, offset, dev),
            strided(add, extra, offset, dev))


def run(x, w, b, dy, add, y_type, eps=EPS):
    N, D = x.shape
    out = torch.full((N, D), float("nan"), dtype=y_type, device=x.device)
    stats = torch.full((N, 2), float("nan"), dtype=torch.float64, device=x.device)
    y = dense.layer_norm(x, w, b, eps=eps, out=out, stats=stats)
    grads = dense.layer_norm_bwd(x, dy, stats, w, add=add, weight_dtype=None if w is not None else torch.float32)
    return y, stats, grads


def verify(x, w, b, dy, add, y, stats, grads, eps=EPS):
    want, bound, mean, inv = ref.norm(x, w, b, eps)
    check(y, want, bound, "y")
    # fp64 sums of distances from the row's first value: some hundred roundings of 2^-53 of at most twice the span
    span = wide(x).abs().amax(1, keepdim=True)
    assert ((wide(stats)[:, :1] - mean).abs() <= 2.0 ** -45 * span + 1e-300).all()
    assert ((wide(stats)[:, 1:] / inv - 1).abs() <= 2.0 ** -43 * (1 + (span * inv).square())).all()
    for got, (value, off), name in zip(grads, ref.norm_grad(x, w, dy, eps, add), ("dx", "dweight", "dbias")):
        check(got, value, off, name)


@pytest.mark.parametrize("x,y", PAIRS)
@pytest.mark.parametrize("N,D", [(1, 1), (3, 7), (5, 64), (70, 65), (9, 130), (37, 256), (33, 515), (18, 1003),
                                 (7, 2048), (6, 2057), (5, 4096), (4, 4101), (3, 8192), (3, 8200), (2, 16384), (2, 16390)])
def test_layer_norm(dev, x, y, N, D):
    args = inputs(N * 1000 + D, N, D, x, y, F32, dev)
    y_, stats, grads = run(*args, y)
    verify(*args, y_, stats, grads)


@pytest.mark.parametrize("x,y", [(F32, BF16), (F16, F16)])
@pytest.mark.parametrize("D", [33000, 70001])
def test_long_rows(dev, x, y, D):
    args = inputs(D, 3, D, x, y, y, dev)
    y_, stats, grads = run(*args, y)
    verify(*args, y_, stats, grads)


@pytest.mark.parametrize("x,y", PAIRS)
@pytest.mark.parametrize("extra,offset", [(1, 1), (8, 3), (24, 0)])
@pytest.mark.parametrize("D", [96, 1000, 3001])
def test_strides_and_alignment(dev, x, y, extra, offset, D):
    args = inputs(7, 21, D, x, y, y, dev, extra, offset)
    y_, stats, grads = run(*args, y)
    verify(*args, y_, stats, grads)


@pytest.mark.parametrize("N,D", [(70000, 16), (5000, 300), (1201, 2048)])
def test_many_rows(dev, N, D):
    args = inputs(N, N, D, BF16, BF16, F32, dev)
    y_, stats, grads = run(*args, BF16)
    verify(*args, y_, stats, grads)


@pytest.mark.parametrize("weight,bias,add", [(False, False, False), (True, False, True), (False, True, False)])
def test_without_weight_bias_or_add(dev, weight, bias, add):
    x, w, b, dy, more = inputs(11, 40, 200, BF16, BF16, BF16, dev)
    args = (x, w if weight else None, b if bias else None, dy, more if add else None)
    y_, stats, grads = run(*args, BF16)
    verify(*args, y_, stats, grads)


@pytest.mark.parametrize("mean,size", [(1e4, 1.0), (0.0, 1e-20), (1.0, 1e-6), (0.0, 1e30), (3e37, 1e30), (0.0, 1e-42)])
def test_means_and_sizes_at_the_ends(dev, mean, size):
    # a large mean, a tiny spread and squares beyond fp32's range cost no precision
    x, w, b, dy, add = inputs(13, 12, 500, F32, F32, F32, dev, mean=mean, size=size)
    eps = 1e-37
    y_, stats, grads = run(x, w, b, dy, None, F32, eps)
    want, bound, *_ = ref.norm(x, w, b, eps)
    check(y_, want, bound, "y")
    (dx, off), *_ = ref.norm_grad(x, w, dy, eps)
    # 1 / std rounds to fp32's subnormals for the largest
    check(grads[0], dx, off + 2.0 ** -148 * wide(dy).abs().amax(), "dx")


def test_opposite_ends_of_the_range(dev):
    x = torch.tensor([[3.4e38, -3.4e38, 1e38, 0.0] * 5], device=dev)
    y = dense.layer_norm(x)
    want, bound, *_ = ref.norm(x, None, None, 1e-5)
    check(y, want, bound, "y")


def test_constant_rows(dev):
    x = torch.full((4, 300), 7.25, device=dev)
    b = torch.randn(300, device=dev)
    stats = torch.empty(4, 2, dtype=torch.float64, device=dev)
    y = dense.layer_norm(x, None, b, stats=stats)
    assert torch.equal(y, b.expand(4, 300)) and torch.allclose(stats[:, 1], torch.tensor(1e-5, dtype=torch.float64, device=dev) ** -0.5)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("at", [0, 5])
def test_a_row_with_no_number_spoils_itself_alone(dev, bad, at):
    x, w, b, dy, add = inputs(17, 10, 260, BF16, BF16, F32, dev)
    y0, stats0, (dx0, *_) = run(x, w, b, dy, add, BF16)
    x[3, at] = bad
    y1, _, (dx1, *_) = run(x, w, b, dy, add, BF16)
    keep = torch.arange(10, device=dev) != 3
    assert torch.equal(y0[keep], y1[keep]) and torch.equal(dx0[keep], dx1[keep])
    assert y1[3].isnan().all() and dx1[3].isnan().all()


def test_in_place_and_nothing_past_the_rows(dev):
    x, w, b, dy, add = inputs(19, 30, 777, BF16, BF16, F32, dev, extra=5)
    y, stats, (dx, dw, db) = run(x, w, b, dy, add, BF16)
    x2 = strided(x.cpu(), 5, 0, dev)
    dense.layer_norm(x2, w, b, out=x2)
    assert torch.equal(x2, y)
    assert x2.as_strided((29, 5), (782, 1), 777).isnan().all()  # what lies between the rows
    for name in ("add", "dy"):
        a2, g2 = strided(add.cpu(), 5, 0, dev), strided(dy.cpu(), 5, 0, dev)
        to = a2 if name == "add" else g2
        dense.layer_norm_bwd(x, g2, stats, w, add=a2, out=(to, None, None))
        assert torch.equal(to, dx)
        assert to.as_strided((29, 5), (782, 1), 777).isnan().all()


def test_parts_of_the_gradient_alone(dev):
    x, w, b, dy, add = inputs(23, 300, 200, F32, BF16, F32, dev)
    _, stats, (dx, dw, db) = run(x, w, b, dy, add, BF16)
    assert torch.equal(dense.layer_norm_bwd(x, dy, stats, w, add=add, out=(torch.empty_like(dx), None, None))[0], dx)
    assert torch.equal(dense.layer_norm_bwd(x, dy, stats, w, out=(None, torch.empty_like(dw), None))[1], dw)
    assert torch.equal(dense.layer_norm_bwd(x, dy, stats, w, out=(None, None, torch.empty_like(db)))[2], db)


def test_no_rows(dev):
    x = torch.empty(0, 50, device=dev)
    stats = torch.empty(0, 2, dtype=torch.float64, device=dev)
    assert dense.layer_norm(x, stats=stats).shape == (0, 50)
    dx, dw, db = dense.layer_norm_bwd(x, x, stats, torch.ones(50, device=dev),
                                      out=(torch.empty(0, 50, device=dev),) + tuple(torch.full((50,), 9.0, device=dev) for _ in range(2)))
    assert not dw.any() and not db.any()


def test_same_bits_on_repeats_and_on_another_stream(dev):
    args = inputs(29, 3000, 515, BF16, BF16, F32, dev)
    first = run(*args, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(*args, BF16)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip((first[0], first[1], *first[2]), (again[0], again[1], *again[2])):
        assert torch.equal(a, b)


def test_gradient_against_differences(dev):
    # L = sum(y dy) along a direction, by the kernels' own forward pass; the difference quotient's truncation is known
    # from 64 bits, and each y is off by at most its bound
    x, w, b, dy, _ = inputs(31, 6, 40, F32, F32, F32, dev)
    d = torch.randn(6, 40, generator=torch.Generator().manual_seed(5)).to(dev)
    t = 2.0 ** -6
    _, _, (dx, dw, db) = run(x, w, b, dy, None, F32)

    def loss(rows, exact):
        y, bound, *_ = ref.norm(rows, w, b, EPS)
        if not exact:
            y, bound = wide(dense.layer_norm(rows, w, b, eps=EPS)), bound + ref.E * y.abs()
        return float((y * wide(dy)).sum()), float((bound * wide(dy).abs()).sum())

    up, down = x + t * d, x - t * d  # rounded once: both sides take the rows as they are
    step = (wide(up) - wide(down))
    (l1, e1), (l0, e0) = loss(up, False), loss(down, False)
    (x1, _), (x0, _) = loss(up, True), loss(down, True)
    (want, off), *_ = ref.norm_grad(x, w, dy, EPS)
    truncation = abs((x1 - x0) - float((want * step).sum()))
    assert abs((l1 - l0) - float((wide(dx) * step).sum())) <= e1 + e0 + truncation + float(
        ((off + ref.E * want.abs()) * step.abs()).sum())


def test_captured_forward_and_backward_replayed(dev):
    args = inputs(37, 200, 384, BF16, BF16, F32, dev)
    x, w, b, dy, add = args
    y = torch.empty(200, 384, dtype=BF16, device=dev)
    stats = torch.empty(200, 2, dtype=torch.float64, device=dev)
    out = (torch.empty_like(y), torch.empty_like(w), torch.empty_like(b))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=dev)

    def step():
        dense.layer_norm(x, w, b, out=y, stats=stats)
        dense.layer_norm_bwd(x, dy, stats, w, add=add, out=out, workspace=ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        x.copy_(torch.randn(200, 384, generator=torch.Generator().manual_seed(k)).to(BF16))
        want = run(x, w, b, dy, add, BF16)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, c in zip((y, stats, *out), (want[0], want[1], *want[2])):
            assert torch.equal(a, c)


@pytest.mark.parametrize("x,y", [(F32, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("D", [66000, 70001, 1000003])
def test_the_largest_value_far_from_a_long_rows_mean(dev, x, y, D):
    # its distance from the mean passes fp32's range, while the spread of so many features does not come near it
    top = torch.finfo(x).max
    rows = torch.full((3, D), -top / 100)
    rows[:, ::3] *= 1.01
    rows[0, 17] = rows[1, D - 1] = rows[2, 0] = top
    rows[2] *= -1
    g = torch.Generator().manual_seed(D)
    rows, dy = rows.to(x).to(dev), torch.randn(3, D, generator=g).to(y).to(dev)
    w, b = (1 + 0.3 * torch.randn(D, generator=g)).to(dev), (0.3 * torch.randn(D, generator=g)).to(dev)
    y_, stats, (dx, dw, db) = run(rows, w, b, dy, None, y)
    want, bound, *_ = ref.norm(rows, w, b, EPS)
    check(y_, want, bound, "y")
    (vx, off), (vw, off_w), (vb, off_b) = ref.norm_grad(rows, w, dy, EPS)
    check(dx, vx, off + 2.0 ** -146, "dx")  # near fp32's smallest values: a few roundings of 2^-149
    check(dw, vw, off_w, "dweight")
    check(db, vb, off_b, "dbias")
