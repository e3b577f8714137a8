"""Layer norm, AdamW and the 4-bit operators run together: the example's normalised experts (examples/map_experts.py), a
captured training step, and rows that are normalised, quantised and multiplied."""
import importlib.util
import os

import pytest
import torch

import layer_ref as ref
import paper_2608_24067_amd.dense as dense
from dense_ref import check, sums, wide

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("map_experts", os.path.join(ROOT, "examples", "map_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients_of_normed_experts(dev, example):
    prototypes = torch.randn(48, 16, generator=torch.Generator().manual_seed(2))
    model = example.NormedExperts(prototypes, 72, seed=3)
    g = torch.Generator().manual_seed(7)
    model.weight.copy_(1 + 0.2 * torch.randn(48, generator=g))
    model.bias.copy_(0.2 * torch.randn(48, generator=g))
    x, _ = example.rows(200, prototypes, seed=4)
    out, kept = model.forward(x)
    _, _, (scores, idx, w) = kept
    dout = torch.randn(200, 48, generator=g).bfloat16().to(dev)
    grads, dx = model.gradients(x, kept, dout)
    assert len(grads) == len(model.params) == 7

    p = [t.cpu().double().requires_grad_(True) for t in model.params]
    xs, at = x.cpu().double().requires_grad_(True), idx.cpu().long()
    weight, bias, W, W1, b1, W2, b2 = p
    mean = xs.mean(1, keepdim=True)
    h = (xs - mean) / torch.sqrt((xs - mean).square().mean(1, keepdim=True) + 1e-5) * weight + bias
    check(kept[0], h.detach(), 2.0 ** -18 * (h.detach().abs() + 1), "h")
    # The values that follow are those of the rounded h: a score moves by sum_i h_i W_i d_i, |d_i| <= 2^-9, some
    # |h| |W| 2^-9 / sqrt(3) = 7 x 7 x 0.0011 = 0.05 here, and the softmax makes that 5% of a weight (26 roundings).
    h = h + (wide(kept[0]) - h).detach()
    s = h @ W - 0.5 * W.square().sum(0)
    wt = torch.softmax(s.gather(1, at), 1)
    y = xs
    for j in range(2):
        e = at[:, j]
        z = (h.unsqueeze(2) * W1[e]).sum(1) + b1[e]
        inner = z * 0.5 * torch.erfc(-z * 0.5 ** 0.5)
        y = y + wt[:, j:j + 1] * ((inner.unsqueeze(2) * W2[e]).sum(1) + b2[e])
    wanted = torch.autograd.grad((y * dout.cpu().double()).sum(), p + [xs])

    # bf16 rounds to 2^-9 of a value: some ten such roundings lie between (the normalised rows, the weights, the inner
    # rows, dz, dw, dscores, the two gradients of the normalised rows, their sum, and the result)
    def near(got, want, what):
        off = float((got.cpu().double() - want.detach()).norm() / want.detach().norm())
        assert off <= 10 * 2.0 ** -9, f"{what}: {off / 2 ** -9:.2f} roundings"

    near(out, y, "out")
    for name, a, b in zip(("weight", "bias", "gate", "W1", "b1", "W2", "b2", "dx"), grads + [dx], wanted):
        near(a, b, name)


@pytest.mark.parametrize("bits", [32, 8])
def test_the_example_runs(dev, example, bits):
    losses = example.main(["--steps", "3", "--rows", "700", "--width", "96", "--edge", "4", "--adamw", str(bits)])
    assert len(losses) == 3 and all(0 < loss < float("inf") for loss in losses)


@pytest.mark.parametrize("both", [True, False])
def test_answers_in_4_bits(dev, example, both):
    # the units are those of scores from what the codes stand for, and the rows go through their experts
    prototypes = torch.randn(96, 25, generator=torch.Generator().manual_seed(2))
    model = example.NormedExperts(prototypes, 64, bits=8, seed=3)
    for s in range(2):
        model.step(*example.rows(300, prototypes, seed=s))
    x, _ = example.rows(333, prototypes, seed=9)
    out, idx = model.answer(x, both)
    h = dense.layer_norm(x, model.weight, model.bias)
    W, W1, b1, W2, b2 = model.experts.params
    four, bias = model.four
    rows = dense.mx4_quantise(h)
    hv = ref.values4(rows.codes, rows.scales, 96) if both else wide(h)
    wv = ref.values4(four.codes, four.scales, 96)
    scores = hv @ wv.t() + wide(bias)
    off = sums(2 * 96 + 4, hv.abs() @ wv.abs().t() + wide(bias).abs())
    # routing takes the two highest of score + balance: none that is left out is higher by more than the bounds
    key, bound = scores + wide(model.experts.balance), off + 2.0 ** -22 * (scores.abs() + 1)
    at = idx.cpu().long()
    lowest = (key - bound).gather(1, at).min(1, keepdim=True).values
    left = (key - bound).scatter(1, at, float("-inf")).max(1, keepdim=True).values
    least = (key + bound).gather(1, at).min(1, keepdim=True).values
    assert bool((left <= least).all()) and bool(lowest.isfinite().all())
    w = torch.softmax(scores.gather(1, at), 1).to(BF16).to(dev)
    again = dense.experts(h, idx, w, W1, b1, W2, b2, residual=x)
    # the weights may differ by a rounding of bf16
    assert float((out.double() - again.double()).norm()) <= 4 * 2.0 ** -9 * float(again.double().norm())


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_training_step(dev, bits):
    """Normalise, multiply, their gradients, the clipped norm and AdamW in one graph: replays go on as eager steps do."""
    N, D, M = 260, 96, 80

    def state():
        g = torch.Generator().manual_seed(5)
        s = {"x": torch.empty(N, D, dtype=BF16, device=dev), "dz": torch.empty(N, M, dtype=BF16, device=dev)}
        s["params"] = [torch.ones(D, device=dev), torch.zeros(D, device=dev),
                       (torch.randn(D, M, generator=g) * 0.1).bfloat16().to(dev), torch.zeros(M, dtype=BF16, device=dev)]
        s["states"] = [dense.adamw_state(p, bits, master=p.dtype == BF16) for p in s["params"]]
        s["h"], s["z"], s["dh"], s["dx"] = (torch.empty(N, k, dtype=BF16, device=dev) for k in (D, M, D, D))
        s["stats"] = torch.empty(N, 2, dtype=torch.float64, device=dev)
        s["grads"] = [torch.empty_like(p) for p in s["params"]]
        s["clipped"] = [torch.empty_like(p) for p in s["params"]]
        s["norm"], s["lr"] = torch.empty(1, device=dev), torch.full((1,), 1e-2, device=dev)
        s["number"] = torch.zeros(1, dtype=torch.int32, device=dev)
        s["ws"] = torch.empty(1 << 22, dtype=torch.uint8, device=dev)
        return s

    def step(s):
        weight, bias, W, b = s["params"]
        dweight, dbias, dW, db = s["grads"]
        s["number"].add_(1)
        dense.layer_norm(s["x"], weight, bias, out=s["h"], stats=s["stats"])
        dense.linear(s["h"], W, b, out=s["z"])
        dense.linear_bwd(s["h"], W, s["dz"], out=(s["dh"], dW, db), workspace=s["ws"])
        dense.layer_norm_bwd(s["x"], s["dh"], s["stats"], weight, out=(s["dx"], dweight, dbias), workspace=s["ws"])
        dense.clip(s["grads"], 1.0, out=s["clipped"], norm=s["norm"], workspace=s["ws"])
        dense.adamw(s["params"], s["clipped"], s["states"], s["number"], lr=s["lr"], norm=s["norm"])

    def fill(s, k):
        g = torch.Generator().manual_seed(100 + k)
        s["x"].copy_(torch.randn(N, D, generator=g).bfloat16())
        s["dz"].copy_(torch.randn(N, M, generator=g).bfloat16())
        s["lr"].fill_(1e-2 / (k + 1))

    def held(s):
        return [*s["params"], *(t for state in s["states"] for t in state if t is not None), s["z"], s["dx"], s["norm"]]

    a, b = state(), state()
    fill(a, 0), fill(b, 0)
    step(a), step(b)  # once outside, as before any capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(b)
    for k in range(1, 5):
        fill(a, k), fill(b, k)
        step(a)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held(a), held(b))), k
    assert int(b["number"]) == 5


def test_a_step_without_a_number_changes_nothing(dev, example):
    prototypes = torch.randn(48, 16, generator=torch.Generator().manual_seed(2))
    model = example.NormedExperts(prototypes, 72, bits=8, seed=3)
    x, target = example.rows(100, prototypes, seed=4)
    model.step(x, target)
    before = [t.clone() for t in model.params]
    target[3, 5] = float("inf")
    _, norm = model.step(x, target)
    assert not bool(norm.isfinite())
    assert all(torch.equal(a, b) for a, b in zip(before, model.params))


def test_normalised_rows_in_4_bits(dev):
    # layer norm of rows in 32 bits to bf16, their codes, the product, and back to the rows' width
    N, D, M = 77, 200, 150
    g = torch.Generator().manual_seed(1)
    x = torch.randn(N, D, generator=g).to(dev)
    W = dense.mx4_quantise((torch.randn(D, M, generator=g) * D ** -0.5).to(dev), columns=True)
    h = dense.layer_norm(x, out=torch.empty(N, D, dtype=BF16, device=dev))
    rows = dense.mx4_quantise(h)
    codes, scales = ref.codes4(wide(h))
    assert (rows.codes.cpu().numpy() == codes).all() and (rows.scales.cpu().numpy() == scales).all()
    y = dense.mx4_linear(rows, W, out_dtype=F32)
    hv, wv = ref.values4(rows.codes, rows.scales, D), ref.values4(W.codes, W.scales, D)
    check(y, hv @ wv.t(), sums(D, hv.abs() @ wv.abs().t()), "y")
    check(dense.mx4_linear(h, W, out_dtype=F32), wide(h) @ wv.t(), sums(D, wide(h).abs() @ wv.abs().t()), "y, rows in 16 bits")


def test_a_step_that_is_left_out_leaves_no_trace(dev, example):
    # parameters, running means, the gate's balance, the step's number, and the steps after it: as if it had not been
    prototypes = torch.randn(48, 16, generator=torch.Generator().manual_seed(2))

    def held(model):
        return [t.clone() for t in (*model.params, *(t for s in model.states for t in s if t is not None),
                                    model.experts.balance, model.taken)]

    for first in (False, True):
        one, two = (example.NormedExperts(prototypes, 72, bits=8, seed=3) for _ in range(2))
        if not first:
            assert all(bool(m.step(*example.rows(100, prototypes, seed=4))[1].isfinite()) for m in (one, two))
        before = held(one)
        x, target = example.rows(100, prototypes, seed=5)
        target[3, 5] = float("inf")
        _, norm = one.step(x, target)
        assert not bool(norm.isfinite())
        assert all(torch.equal(a, b) for a, b in zip(before, held(one)))
        for s in (6, 7):
            for m in (one, two):
                m.step(*example.rows(100, prototypes, seed=s))
            assert all(torch.equal(a, b) for a, b in zip(held(one), held(two)))
        assert int(one.taken) == (2 if first else 3)


def test_rows_much_larger_than_the_experts_part(dev, example):
    # the sum with the rows is rounded once: a bf16 result is off by half its step, and by the experts' own part's error,
    # which the same call without the residual shows the size of
    prototypes = torch.randn(48, 16, generator=torch.Generator().manual_seed(2))
    model = example.NormedExperts(prototypes, 72, seed=3)
    x, _ = example.rows(200, prototypes, seed=4)
    x = x + 37.0
    out, (h, _, (_, idx, w)) = model.forward(x)
    _, W1, b1, W2, b2 = model.experts.params
    assert torch.equal(out, dense.experts(h, idx, w, W1, b1, W2, b2, residual=x))
    part = dense.experts(h, idx, w, W1, b1, W2, b2)
    want = wide(x) + wide(part)
    check(out, want, 2.0 ** -8 * wide(part).abs(), "out")
