"""som_route and its gradient against row-by-row forms in 64 bits, on the GPU."""
import math

import pytest
import torch

import paper_2608_24067_amd.dense as dense
from dense_ref import TINY, U, check, route, route_grad, wide

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]


def logits(seed, N, E, dtype, dev, pad=0, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    t = torch.full((N, E + pad), float("nan"), dtype=dtype, device=dev)[:, :E]
    t.copy_((torch.randn(N, E, generator=g) * scale).to(dtype))
    return t, g


def close(got, ref, what):
    """A weight is a quotient of a few exponentials and an fp32 sum over at most 4,096 of them, 2^-18 of it."""
    check(got, ref, 2.0 ** -18 * ref.abs() + 2.0 ** -120, what)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,E,k,pad,groups,top", [
    (1, 1, 1, 0, 1, 1),
    (1, 64, 2, 0, 1, 1),
    (5, 3, 3, 1, 1, 1),
    (19, 65, 8, 0, 1, 1),
    (33, 256, 16, 3, 8, 3),
    (7, 63, 5, 0, 9, 2),
    (9, 128, 32, 0, 64, 20),
    (18, 1000, 4, 0, 1, 1),
    (6, 1024, 32, 0, 4, 1),
    (3, 1025, 7, 0, 5, 2),
    (2, 4096, 20, 5, 64, 64),
])
@pytest.mark.parametrize("score,renorm,biased", [("softmax", True, False), ("softmax", False, True),
                                                  ("sigmoid", True, True), ("sigmoid", False, False)])
def test_route(dev, dtype, N, E, k, pad, groups, top, score, renorm, biased):
    l, g = logits(21, N, E, dtype, dev, pad)
    bias = torch.randn(E, generator=g).to(dev) if biased else None
    counts = torch.full((E,), -9, dtype=torch.int32, device=dev)
    how = dict(score=score, renorm=renorm, groups=groups, group_top=top)
    idx, w = dense.route(l, k, bias=bias, counts=counts, **how)
    ri, rw = route(l, k, bias, **how)
    assert torch.equal(idx.cpu(), ri)
    close(w, rw, "weights")
    assert torch.equal(counts.cpu().long(), torch.bincount(ri[ri >= 0].long(), minlength=E))
    dw = torch.randn(N, k, generator=g).to(dtype).to(dev)
    dl = dense.route_bwd(l, idx, dw, bias=bias, **how)
    # sums of k terms dw w (|w| <= 1), their differences rounded in fp32, scaled by scores of at most 1
    ref = route_grad(l, idx, dw, bias, score, renorm)
    over = 1.0
    if score == "sigmoid" and renorm:  # divided by the sum of the scores
        some = ri >= 0
        s = torch.sigmoid(wide(l).gather(1, ri.clamp_min(0).long())) * some
        over = 1.0 / s.sum(1, keepdim=True).clamp_min(1e-30)
    check(dl, ref, 2.0 ** -17 * wide(dw).abs().sum(1, keepdim=True) * over.clamp_min(1) if torch.is_tensor(over)
          else 2.0 ** -17 * wide(dw).abs().sum(1, keepdim=True).expand_as(ref), "dlogits")


@pytest.mark.parametrize("E,groups", [(24, 1), (24, 4), (300, 1), (300, 10), (2000, 8)])
@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_closed_units(dev, E, groups, score, renorm):
    inf, big = math.inf, torch.finfo(torch.float32).max
    l, g = logits(22, 12, E, torch.float32, dev)
    l[0] = -inf                                # every unit closed
    l[1] = math.nan
    l[2, :-1] = -inf                           # one unit open
    l[3] = -big                                # the type's lowest value is a value
    l[4, ::2] = -big
    l[5, 3] = inf                              # one infinity, then two
    l[6, 1] = l[6, E - 1] = inf
    l[7] = 0.0                                 # ties: the lowest indexes
    l[7, ::2] = -0.0
    l[8, ::3] = math.nan
    l[9] = big
    l[10] = -200.0                             # scores that underflow
    how = dict(score=score, renorm=renorm, groups=groups, group_top=max(1, groups // 2))
    k = 6
    bias = torch.zeros(E, device=dev)
    for b in (None, bias):
        idx, w = dense.route(l, k, bias=b, **how)
        ri, rw = route(l, k, b, **how)
        assert torch.equal(idx.cpu(), ri)
        close(w, rw, "weights")
        assert not w[idx < 0].any() and bool((idx[:2] == -1).all())
        dw = torch.randn(12, k, generator=g).to(dev)
        dl = dense.route_bwd(l, idx, dw, bias=b, **how)
        assert bool(torch.isfinite(dl).all())
        assert not dl[(l == -inf) | torch.isnan(l)].any()
        rows = [2, 3, 4, 5, 6, 7, 8, 9, 11]
        ref = route_grad(l, idx, dw, b, score, renorm)
        check(dl[rows], ref[rows], 2.0 ** -15 * wide(dw).abs().sum(1, keepdim=True)[rows].expand(-1, E), "dlogits")
    bias[5] = -inf                             # a unit closed to every row by the bias
    bias[7] = math.nan
    idx, w = dense.route(l, k, bias=bias, **how)
    ri, rw = route(l, k, bias, **how)
    assert torch.equal(idx.cpu(), ri) and not bool(((idx == 5) | (idx == 7)).any())
    close(w, rw, "weights")


def test_lowest_value_of_short_types(dev):
    for dt in (torch.float16, torch.bfloat16):
        l = torch.full((3, 40), torch.finfo(dt).min, dtype=dt, device=dev)
        l[1, 20] = 0
        l[2, 1:] = -math.inf
        idx, w = dense.route(l, 3, renorm=False)
        ri, rw = route(l, 3, renorm=False)
        assert torch.equal(idx.cpu(), ri)
        close(w, rw, "weights")


def test_weights_of_another_type_and_gradient_against_differences(dev):
    l, g = logits(23, 6, 37, torch.float32, dev)
    for score, renorm in (("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)):
        idx, w = dense.route(l, 4, score=score, renorm=renorm, weights_dtype=torch.bfloat16)
        ri, rw = route(l, 4, None, score, renorm)
        assert w.dtype == torch.bfloat16 and torch.equal(idx.cpu(), ri)
        close(w, rw, "weights")
        dw = torch.randn(6, 4, generator=g).bfloat16().to(dev)
        dl = dense.route_bwd(l, idx, dw, score=score, renorm=renorm)
        v = torch.randn(6, 37, generator=g, dtype=torch.float64)
        h = 1e-6

        def f(x):  # the weights of the units taken, as a function of the logits, in 64 bits
            p = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, 1)
            t = p.gather(1, ri.long())
            t = t / t.sum(1, keepdim=True) if renorm else t
            return float((wide(dw) * t).sum())

        diff = (f(wide(l) + h * v) - f(wide(l) - h * v)) / (2 * h)
        assert abs(diff - float((wide(dl) * v).sum())) <= 1e-5 * (1 + float(wide(dw).abs().sum()))


def test_foreign_indexes_are_skipped(dev):
    l, g = logits(24, 4, 50, torch.float32, dev)
    idx = torch.tensor([[3, -1], [50, 7], [-5, 2 ** 30], [1, 0]], dtype=torch.int32, device=dev)
    dw = torch.randn(4, 2, generator=g).to(dev)
    dl = dense.route_bwd(l, idx, dw, renorm=False)
    check(dl, route_grad(l, idx, dw, None, "softmax", False), 2.0 ** -17 * wide(dw).abs().sum(1, keepdim=True).expand(4, 50),
          "dlogits")
    assert not dl[2].any()


def test_many_rows_and_no_rows(dev):
    l, _ = logits(25, 20011, 48, torch.bfloat16, dev)
    counts = torch.empty(48, dtype=torch.int32, device=dev)
    idx, w = dense.route(l, 3, counts=counts)
    key = l.float().cpu()
    ref = key.sort(dim=1, descending=True, stable=True).indices[:, :3].int()
    assert torch.equal(idx.cpu(), ref)
    assert torch.equal(counts.cpu().long(), torch.bincount(ref.reshape(-1).long(), minlength=48))
    counts.fill_(7)
    idx, w = dense.route(l[:0], 3, counts=counts)
    assert idx.shape == (0, 3) and not counts.any()
    assert dense.route_bwd(l[:0], idx, w).shape == (0, 48)
    assert U[torch.float16] and TINY[torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("E,groups", [(24, 1), (24, 4), (300, 1), (300, 10), (2000, 8)])
def test_zeros_of_both_signs_are_equal(dev, dtype, E, groups):
    l = torch.zeros(4, E, dtype=dtype, device=dev)
    l[:, ::2] = -0.0
    l[3] = -0.0
    bias = torch.full((E,), -0.0, device=dev)
    bias[E // 2] = 0.0
    how = dict(groups=groups, group_top=max(1, groups // 2))
    for b in (bias, None):
        idx, w = dense.route(l, 5, bias=b, **how)
        ri, rw = route(l, 5, b, **how)
        assert torch.equal(idx.cpu(), ri)
        close(w, rw, "weights")


@pytest.mark.parametrize("N,E", [((1 << 26) + 5, 65), ((1 << 28) + 3, 4)])
def test_more_threads_than_a_grid_holds_along_x(dev, N, E):
    # 64 threads a row, or 16: 2^32 of them. One logit of every row stands out
    best = torch.arange(N, dtype=torch.int32, device=dev).bitwise_xor_(N >> 3).remainder_(E)
    l = torch.zeros(N, E, dtype=torch.float16, device=dev)
    l.scatter_(1, best[:, None].long(), 3.0)
    counts = torch.empty(E, dtype=torch.int32, device=dev)
    idx, w = dense.route(l, 1, renorm=False, counts=counts)
    assert torch.equal(idx[:, 0], best)
    p = math.exp(3) / (math.exp(3) + E - 1)
    assert float((w - p).abs().max()) <= 2.0 ** -11 * p + 2.0 ** -17
    assert torch.equal(counts, torch.bincount(best, minlength=E).int())
    dw = torch.ones(N, 1, dtype=torch.float16, device=dev)
    dl = dense.route_bwd(l, idx, dw, renorm=False, out=torch.full_like(l, float("nan")))
    q = p / math.exp(3)  # the others' share: their gradient is -p q, the best one's p (1 - p)
    top = torch.zeros(N, dtype=torch.float16, device=dev)
    for a in range(0, N, 1 << 25):
        b = slice(a, a + (1 << 25))
        at = best[b, None].long()
        top[b] = dl[b].gather(1, at)[:, 0]
        assert float((dl[b].scatter(1, at, -p * q) + p * q).abs().max()) <= 2.0 ** -10 * p * q + 2.0 ** -17
    assert float((top - p * (1 - p)).abs().max()) <= 2.0 ** -10 * p * (1 - p) + 2.0 ** -17
    del l, dl, idx, w, best, dw, top
    torch.cuda.empty_cache()


@pytest.mark.parametrize("E,groups", [(24, 1), (24, 4), (300, 10), (2000, 1)])
def test_infinity_ranks_above_every_number_and_weighs_as_the_largest(dev, E, groups):
    big, inf = torch.finfo(torch.float32).max, math.inf
    l, g = logits(26, 4, E, torch.float32, dev)
    l[0, 3], l[0, 5] = big, inf
    l[1, E - 1] = inf
    l[2, 2], l[2, 4] = inf, inf
    bias = torch.zeros(E, device=dev)
    bias[E - 1], bias[1] = -1e38, inf  # an infinity stays one; a bias makes one of a number
    how = dict(groups=groups, group_top=max(1, groups // 2))
    for b in (None, bias):
        for score, renorm in (("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)):
            idx, w = dense.route(l, 4, bias=b, score=score, renorm=renorm, **how)
            ri, rw = route(l, 4, b, score, renorm, **how)
            assert torch.equal(idx.cpu(), ri)
            close(w, rw, "weights")
            if b is None:
                assert idx[0, :2].tolist() == [5, 3] or groups > 1
