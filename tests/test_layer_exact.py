"""CPU tests of the inputs whose sums are exact (layer_exact): the sums are, and a result that leaves out a row, a unit of
features or a part of the sum differs."""
import pytest
import torch

import layer_exact as exact
import layer_ref as ref
from dense_ref import check, sums


@pytest.mark.parametrize("N,D,x,y", [c for c in exact.GRADIENTS if c[0] * c[1] <= 1 << 22])
def test_gradients(N, D, x, y):
    rows, dy, _ = exact.gradient(N, D, getattr(torch, x), getattr(torch, y), 1)
    dw, db = exact.gradient_sums(rows, dy)
    assert 6 * N < 1 << 24
    # every row counts in every sum, so none can be left out, or taken twice
    assert ((rows.float() * dy.float()).min() >= 1) and dy.float().min() >= 1
    assert torch.equal(dw.double(), (rows.double() * dy.double()).sum(0)) and torch.equal(db.double(), dy.double().sum(0))


def test_the_largest_gradient_stays_exact():
    assert all(6 * N < 1 << 24 for N in [1050001] + [c[0] for c in exact.GRADIENTS])


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("N,K,M", exact.PRODUCTS + exact.LONG)
def test_products(N, K, M, packed):
    N, M = min(N, 40), min(M, 60)  # rows and columns are alike
    (_, xv), (_, _, wv) = exact.factors(N, K, M, packed)
    want, size, unit = exact.multiply(xv, wv)
    assert float(size.max()) < unit * (1 << 24)
    # the part of each unit of features, and that of the last feature alone, is not zero in every result
    whole = K // exact.UNIT * exact.UNIT
    for u in range(0, whole, 1 << 20):
        a, b = (t[:, u:min(u + (1 << 20), whole)].reshape(t.shape[0], -1, exact.UNIT).transpose(0, 1) for t in (xv[:2], wv[:5]))
        assert bool((a @ b.transpose(1, 2)).ne(0).flatten(1).any(1).all())
    assert bool((xv[:, -1:] @ wv[:, -1:].t()).ne(0).all())
    if K > whole:
        assert K == 1 or bool((xv[:, whole:] @ wv[:, whole:].t()).ne(0).any())
    assert bool(want.ne(0).any())


def test_the_bound_by_depth_rejects_a_lost_part():
    # what test_gradients_of_many_rows allows is less than one part of 512, or the last 100 rows, make
    N, D = 70000, 16
    g = torch.Generator().manual_seed(N)
    h, dy = torch.randn(N, D, generator=g).double(), torch.randn(N, D, generator=g).double()
    terms = h * dy
    want, bound = terms.sum(0), exact.gradient_bound(N, terms.abs().sum(0))
    check(want.float(), want, bound, "dweight")
    for lost in (terms[:136].sum(0), terms[-100:].sum(0), want):
        with pytest.raises(AssertionError):
            check((want - lost).float(), want, bound, "dweight")


def test_the_bound_of_a_product_rejects_a_lost_block():
    N, K, M = 40, 1003, 60
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn(N, K, generator=g).double(), torch.randn(M, K, generator=g).double()
    want, size = x @ w.t(), x.abs() @ w.abs().t()
    check(want.float(), want, sums(K + 2, size), "y")
    for part in (slice(0, 32), slice(K - 11, K), slice(0, K)):
        with pytest.raises(AssertionError):
            check((want - x[:, part] @ w[:, part].t()).float(), want, sums(K + 2, size), "y")
