"""Layer norm's gradient and the products with 4-bit matrices where their sums are exact (layer_exact), compared for equality,
and with bounds by the depth of the sums, on the GPU."""
import pytest
import torch

import layer_exact as exact
import layer_ref as ref
import paper_2608_24067_amd.dense as dense
from dense_ref import check, sums, wide

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def verify_gradient(x, dy, stats):
    dw, db = exact.gradient_sums(x, dy)
    _, gw, gb = dense.layer_norm_bwd(x, dy, stats)
    assert torch.equal(gw.double(), dw.double()) and torch.equal(gb.double(), db.double())
    # without dx, and each sum alone
    _, gw, _ = dense.layer_norm_bwd(x, dy, stats, out=(None, torch.empty_like(gw), None))
    _, _, gb = dense.layer_norm_bwd(x, dy, stats, out=(None, None, torch.empty_like(gb)))
    assert torch.equal(gw.double(), dw.double()) and torch.equal(gb.double(), db.double())


@pytest.mark.parametrize("N,D,x,y", exact.GRADIENTS)
def test_gradients(dev, N, D, x, y):
    verify_gradient(*exact.gradient(N, D, getattr(torch, x), getattr(torch, y), 1, dev))


def test_gradients_of_rows_past_32_bits(dev):
    verify_gradient(*exact.gradient(1050001, 2048, BF16, BF16, 2, dev))  # 2^31 elements at row 1,048,576
    torch.cuda.empty_cache()


@pytest.mark.parametrize("N,D", [(70000, 16), (5000, 300), (1201, 2048)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_many_rows(dev, N, D, dtype):
    g = torch.Generator().manual_seed(N)
    x, dy = torch.randn(N, D, generator=g).to(dtype).to(dev), torch.randn(N, D, generator=g).to(dtype).to(dev)
    stats = torch.empty(N, 2, dtype=torch.float64, device=dev)
    dense.layer_norm(x, stats=stats)
    _, dw, db = dense.layer_norm_bwd(x, dy, stats)
    _, _, mean, inv = ref.norm(x, None, None, 1e-5)
    h, t = (wide(x) - mean) * inv, wide(dy)
    # h itself is off by 6 E of it
    check(dw, (t * h).sum(0), exact.gradient_bound(N, (t * h).abs().sum(0)) + 6 * ref.E * (t * h).abs().sum(0), "dweight")
    check(db, t.sum(0), exact.gradient_bound(N, t.abs().sum(0)), "dbias")


def verify_product(dev, dtype, N, K, M, packed, extra=0):
    (x, xv), (codes, scales, wv) = exact.factors(N, K, M, packed)
    want, *_ = exact.multiply(xv, wv)
    W = dense.Mx4(codes.to(dev), scales.to(dev), K)
    if packed:
        rows = dense.Mx4(x[0].to(dev), x[1].to(dev), K)
    else:
        rows = torch.full((N, K + extra), float("nan"), dtype=dtype, device=dev)[:, :K].copy_(x)
    y = dense.mx4_linear(rows, W, out_dtype=F32, dtype=dtype if packed else None)
    assert torch.equal(wide(y), want)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", exact.PRODUCTS)
def test_products(dev, dtype, packed, N, K, M):
    verify_product(dev, dtype, N, K, M, packed)
    if not packed:
        verify_product(dev, dtype, N, K, M, packed, extra=3)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", exact.LONG)
def test_products_of_long_rows(dev, dtype, packed, N, K, M):
    verify_product(dev, dtype, N, K, M, packed)
    if not packed:
        verify_product(dev, dtype, N, K, M, packed, extra=3)


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("N,K,M", [(1, 1024, 4096), (17, 1003, 70), (33, 2048, 300), (300, 320, 2000), (2011, 1003, 1125), (3300, 513, 1700)])
def test_products_of_any_numbers(dev, dtype, packed, N, K, M):
    g = torch.Generator().manual_seed(N + K)
    x = torch.randn(N, K, generator=g).to(dtype).to(dev)
    W = dense.mx4_quantise((torch.randn(K, M, generator=g) * torch.exp(torch.randn(1, M, generator=g))).to(dev), columns=True)
    b = torch.randn(M, generator=g)
    rows = dense.mx4_quantise(x) if packed else x
    xv, wv = ref.values4(rows.codes, rows.scales, K) if packed else wide(x), ref.values4(W.codes, W.scales, K)
    y = dense.mx4_linear(rows, W, b.to(dev), out_dtype=F32, dtype=dtype if packed else None)
    check(y, xv @ wv.t() + wide(b), sums(K + 2, xv.abs() @ wv.abs().t() + wide(b).abs()), "y")
