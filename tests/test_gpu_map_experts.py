"""The dense operators run together (examples/map_experts.py): a training step against autograd in 64 bits, steps that
learn, and a captured step replayed against the eager one."""
import importlib.util
import os

import pytest
import torch

import paper_2608_24067_amd.dense as dense
from dense_ref import act

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("map_experts", os.path.join(ROOT, "examples", "map_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_a_step_against_autograd(dev, example):
    prototypes = torch.randn(48, 16, generator=torch.Generator().manual_seed(2))
    model = example.MapExperts(prototypes, inner=72, seed=3)
    x, target = example.rows(200, prototypes, seed=4)
    out, kept = model.forward(x)
    scores, idx, w = kept
    dout = torch.randn(200, 48, generator=torch.Generator().manual_seed(6)).bfloat16().to(dev)
    grads = model.backward(x, kept, dout)

    p = [t.cpu().double().requires_grad_(True) for t in model.params]
    xs, at = x.cpu().double(), idx.cpu().long()
    s = xs @ p[0] + model.gate_bias.cpu().double()
    wt = torch.softmax(s.gather(1, at), 1)  # the softmax over all units, divided by the taken ones' sum
    y = xs.clone()
    for j in range(2):
        e = at[:, j]
        z = torch.bmm(xs.unsqueeze(1), p[1][e]).squeeze(1) + p[2][e]
        h = z * 0.5 * torch.erfc(-z * 0.5 ** 0.5)
        y = y + wt[:, j:j + 1] * (torch.bmm(h.unsqueeze(1), p[3][e]).squeeze(1) + p[4][e])
    # bf16 rounds to 2^-9 of a value; a handful of such roundings lie between (weights, inner rows, dz, dw and
    # dscores, and the result), each spread over the sums that follow
    def near(got, ref, roundings, what):
        off = float((got.cpu().double() - ref.detach()).norm() / ref.detach().norm())
        assert off <= roundings * 2.0 ** -9, f"{what}: {off / 2 ** -9:.2f} roundings"

    near(out, y, 4, "out")
    ref = torch.autograd.grad((y * dout.cpu().double()).sum(), p)
    for name, a, b in zip(("gate", "W1", "b1", "W2", "b2"), grads, ref):
        near(a, b, 8, name)
    # the best-matching unit is the first that routing takes
    d = (xs.unsqueeze(2) - p[0].detach().unsqueeze(0)).square().sum(1)
    best = d.min(1).values
    assert bool((d.gather(1, at[:, :1]).squeeze(1) - best <= 1e-3 * best).all())


def test_it_learns_and_balances(dev, example):
    losses = example.main(["--steps", "30", "--rows", "1500", "--width", "96", "--edge", "4"])
    assert losses[-1] < 0.6 * losses[0]


def test_captured_step_replays(dev):
    """Scores, routing, experts and their gradients in a graph: every replay gives the eager call's bits."""
    g = torch.Generator().manual_seed(8)

    def normal(*shape, scale=1.0):
        return (torch.randn(shape, generator=g) * scale).bfloat16().to(dev)

    N, D, F, E, k = 300, 64, 96, 12, 2
    x, gate, dout = normal(N, D), normal(D, E), normal(N, D)
    W1, b1, W2, b2 = normal(E, D, F, scale=0.1), normal(E, F), normal(E, F, D, scale=0.1), normal(E, D)
    ws = torch.empty(dense.experts_workspace_bytes(N, k, E, D, F, keep=True), dtype=torch.uint8, device=dev)
    scores, idx = torch.empty(N, E, device=dev), torch.empty(N, k, dtype=torch.int32, device=dev)
    w, counts, out = normal(N, k), torch.empty(E, dtype=torch.int32, device=dev), torch.empty_like(x)
    grads = tuple(torch.empty_like(t) for t in (x, w, W1, b1, W2, b2))
    clipped, norm = [torch.empty_like(t) for t in grads], torch.empty(1, device=dev)
    clip_ws = torch.empty(1 << 20, dtype=torch.uint8, device=dev)

    def run():
        dense.linear(x, gate, out=scores)
        dense.route(scores, k, out=(idx, w), counts=counts)
        dense.experts(x, idx, w, W1, b1, W2, b2, residual=x, out=out, keep=True, workspace=ws)
        dense.experts_bwd(x, idx, w, W1, W2, b2, dout, out=grads, workspace=ws)
        dense.clip(grads, 1.0, out=clipped, norm=norm, workspace=clip_ws)

    def results():
        return [t.clone() for t in (scores, idx, w, counts, out, *grads, *clipped, norm)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        x.copy_(normal(N, D))  # other rows each time, and other work between the replays
        run()
        eager = results()
        for t in (scores, out, norm, *grads, *clipped):
            t.fill_(float("nan"))
        counts.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, results())), i


def test_the_gate_follows_its_prototypes(dev, example):
    """Where the prototypes have changed, too, the best score is the best-matching unit's, and their gradient is that
    of scores whose bias is -|w|^2 / 2."""
    prototypes = 0.3 * torch.randn(48, 16, generator=torch.Generator().manual_seed(2))  # near: every share counts
    model = example.MapExperts(prototypes, inner=72, seed=3)
    for s in range(3):
        model.step(*example.rows(200, prototypes, seed=50 + s))
    with torch.no_grad():  # and further in place, each by another factor
        model.W.mul_(torch.linspace(0.7, 1.4, 16, device=dev).bfloat16())
    model.balance.zero_()
    x, _ = example.rows(200, prototypes, seed=4)
    out, kept = model.forward(x)
    scores, idx, w = kept
    xs, at = x.cpu().double(), idx.cpu().long()
    p = model.params[0].cpu().double().requires_grad_(True)
    d = (xs.unsqueeze(2) - p.detach().unsqueeze(0)).square().sum(1)
    best = d.min(1).values
    assert bool((d.gather(1, at[:, :1]).squeeze(1) - best <= 1e-3 * best).all())
    dout = torch.randn(200, 48, generator=torch.Generator().manual_seed(6)).bfloat16().to(dev)
    grads = model.gradients(x, kept, dout)
    assert len(grads) == len(model.params)
    s = xs @ p - 0.5 * p.square().sum(0)
    W1, b1, W2, b2 = (t.cpu().double() for t in model.params[1:])
    y = torch.stack([torch.bmm(act("gelu", torch.bmm(xs.unsqueeze(1), W1[at[:, j]]) + b1[at[:, j]].unsqueeze(1)),
                               W2[at[:, j]]).squeeze(1) + b2[at[:, j]] for j in range(2)], 1)
    wt = torch.softmax(s.gather(1, at), 1)
    (ref,) = torch.autograd.grad((wt.unsqueeze(2) * y * dout.cpu().double().unsqueeze(1)).sum(), p)
    # as in a step: some eight roundings of bf16, each spread over the sums that follow
    assert float((grads[0].cpu().double() - ref).norm()) <= 8 * 2.0 ** -9 * float(ref.norm())
