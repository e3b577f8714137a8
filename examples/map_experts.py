"""Local experts on a map: dense rows are scored against a map's units, routed to their best two, and each unit's
expert (a two-layer network) learns what holds in its region of the map.

    python examples/map_experts.py [--steps N] [--adamw 32|8]

One step is what a training program does with the dense operators: scores (``dense.linear`` with the codebook and
-|w|^2 / 2 as its bias, so that the highest score is the best-matching unit), routing with a bias that balances the
units' loads, the experts with the rows as residual, their gradients, the gate's gradient through the routing weights,
and all gradients clipped together. The rows and the function to learn are synthetic.

With ``--adamw`` the rows are normalised first (``dense.layer_norm``), AdamW takes the step, its running means in 32 or 8
bits, and the trained map answers with its prototypes and rows in 4 bits (``dense.mx4_linear``).
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2608_24067_amd.dense as dense  # noqa: E402
import paper_2608_24067_amd.som as som  # noqa: E402


class MapExperts:
    """A map of `units` prototypes over `width` features, an expert of inner width `inner` at each."""

    def __init__(self, prototypes, inner, taken=2, seed=0, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)
        width, units = prototypes.shape  # feature-major, as codebooks are
        dt = torch.bfloat16

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g) * scale).to(dt).to(device)

        self.taken, self.units = taken, units
        self.W = prototypes.to(dt).to(device)
        self.gate_bias = None  # of the last forward pass
        self.balance = torch.zeros(units, device=device)
        self.params = [self.W, normal(units, width, inner, scale=width ** -0.5), normal(units, inner, scale=0.02),
                       normal(units, inner, width, scale=inner ** -0.5 * 0.1), normal(units, width, scale=0.02)]
        self.counts = torch.empty(units, dtype=torch.int32, device=device)
        self.workspace = None

    def forward(self, x, keep=True, residual=None):
        """(out, what the backward pass needs) of rows x [N, width]; out is the experts' part and ``residual`` (x)."""
        W, W1, b1, W2, b2 = self.params
        # the norms of the prototypes as they are held now: the search's own pass over the widened codebook
        self.gate_bias = (-0.5 * som.codebook_norms(W.float(), W.shape[0], W.shape[1])).float()
        scores = dense.linear(x, W, self.gate_bias, out_dtype=torch.float32)
        idx, w = dense.route(scores, self.taken, bias=self.balance, weights_dtype=x.dtype, counts=self.counts)
        need = dense.experts_workspace_bytes(x.shape[0], self.taken, self.units, W1.shape[1], W1.shape[2], keep)
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        out = dense.experts(x, idx, w, W1, b1, W2, b2, residual=x if residual is None else residual, keep=keep,
                            workspace=self.workspace)
        return out, (scores, idx, w)

    def backward(self, x, kept, dout, dx=None):
        """The gradients of the parameters, in their order, with the gate's bias held, and that of this bias. ``dx``
        may pass two tensors [N, width] for the rows' gradients through the experts and through the scores."""
        W, W1, b1, W2, b2 = self.params
        scores, idx, w = kept
        through, into = dx if dx is not None else (None, None)
        grads = [torch.empty_like(t) for t in (w, W1, b1, W2, b2)]
        _, dw, *expert_grads = dense.experts_bwd(x, idx, w, W1, W2, b2, dout, out=(through, *grads), workspace=self.workspace)
        dscores = dense.route_bwd(scores, idx, dw, bias=self.balance).to(x.dtype)
        dbias = torch.empty_like(self.gate_bias)
        _, dW, _ = dense.linear_bwd(x, W, dscores, out=(into, torch.empty_like(W), dbias))
        return [dW] + expert_grads + [dbias]

    def gradients(self, x, kept, dout):
        """The parameters' gradients: the bias is -|w|^2 / 2, whose share is -w times the bias's gradient."""
        dW, *expert_grads, dbias = self.backward(x, kept, dout)
        return [(dW.float() - self.W.float() * dbias).to(dW.dtype)] + expert_grads

    def step(self, x, target, rate=0.5, max_norm=1.0):
        """One step of gradient descent on the mean squared distance to target; returns (loss, gradients' norm)."""
        out, kept = self.forward(x)
        miss = out.float() - target.float()
        grads = self.gradients(x, kept, (miss * (2.0 / miss.shape[0])).to(x.dtype))
        grads, norm = dense.clip(grads, max_norm)
        for p, g in zip(self.params, grads):
            p.sub_((rate * g.float()).to(p.dtype))
        self.rebalance(x.shape[0])
        return miss.square().sum(1).mean(), norm

    def rebalance(self, n, counts=True):
        """Units that take more than their share become less attractive, without a gradient; nothing changes where
        ``counts``, a truth value on the host or the GPU, is false."""
        share = self.counts.float() / max(1.0, float(n * self.taken)) * self.units
        self.balance += 0.05 * (1.0 - share) * counts


class NormedExperts:
    """The experts of a map behind a layer norm: out = x + the experts' part for norm(x), trained by AdamW, whose
    running means are held in `bits`, with float32 copies of the parameters, and served with a map in 4 bits."""

    def __init__(self, prototypes, inner, bits=32, **settings):
        self.experts = MapExperts(prototypes, inner, **settings)
        dev, width = self.experts.W.device, prototypes.shape[0]
        self.weight, self.bias = torch.ones(width, device=dev), torch.zeros(width, device=dev)
        self.params = [self.weight, self.bias] + self.experts.params
        self.states = [dense.adamw_state(p, bits, master=p.dtype != torch.float32) for p in self.params]
        self.taken = torch.zeros(1, dtype=torch.int32, device=dev)  # steps that were not left out
        self.four = None  # the prototypes in 4 bits, since the last step

    def forward(self, x):
        stats = torch.empty(x.shape[0], 2, dtype=torch.float64, device=x.device)
        h = dense.layer_norm(x, self.weight, self.bias, stats=stats)
        out, kept = self.experts.forward(h, residual=x)
        return out, (h, stats, kept)

    def gradients(self, x, kept, dout):
        """The parameters' gradients, in their order, and the rows', which go round the layer too."""
        h, stats, inner = kept
        through, into = torch.empty_like(h), torch.empty_like(h)
        dW, *grads, dbias = self.experts.backward(h, inner, dout, dx=(through, into))
        dW = (dW.float() - self.experts.W.float() * dbias).to(dW.dtype)
        dx, dweight, dnorm = dense.layer_norm_bwd(x, through.add_(into), stats, self.weight, add=dout)
        return [dweight, dnorm, dW] + grads, dx

    def step(self, x, target, rate=3e-3, max_norm=1.0):
        """One step on the mean squared distance to target; returns (loss, gradients' norm). Gradients that hold no
        number leave it out: nothing changes, and it does not count."""
        out, kept = self.forward(x)
        miss = out.float() - target.float()
        grads, _ = self.gradients(x, kept, (miss * (2.0 / miss.shape[0])).to(x.dtype))
        grads, norm = dense.clip(grads, max_norm)
        counts = norm.isfinite()  # asked and answered on the GPU
        self.taken += counts
        dense.adamw(self.params, grads, self.states, self.taken, lr=rate, norm=norm)
        self.four = None
        self.experts.rebalance(x.shape[0], counts)
        return miss.square().sum(1).mean(), norm

    def answer(self, x, both=True):
        """The rows' outputs with the scores from prototypes in 4 bits (and the rows too, or in 16): (out, idx)."""
        m = self.experts
        W, W1, b1, W2, b2 = m.params
        if self.four is None:
            bias = (-0.5 * som.codebook_norms(W.float(), W.shape[0], W.shape[1])).float()
            self.four = dense.mx4_quantise(W, columns=True), bias
        h = dense.layer_norm(x, self.weight, self.bias)
        scores = dense.mx4_linear(dense.mx4_quantise(h) if both else h, *self.four, out_dtype=torch.float32, dtype=h.dtype)
        idx, w = dense.route(scores, m.taken, bias=m.balance, weights_dtype=x.dtype)
        return dense.experts(h, idx, w, W1, b1, W2, b2, residual=x), idx


def rows(n, prototypes, seed, device="cuda"):
    """Rows around the prototypes, and a target that differs from region to region."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    width, units = prototypes.shape
    near = torch.randint(0, units, (n,), generator=g)
    x = prototypes.t()[near] + 0.3 * torch.randn(n, width, generator=g)
    turn = torch.randn(units, width, generator=torch.Generator().manual_seed(5)) * 0.5
    return x.bfloat16().to(device), (x + torch.tanh(x * turn[near])).bfloat16().to(device)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--rows", type=int, default=4096)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--edge", type=int, default=8, help="the map is edge x edge units")
    ap.add_argument("--adamw", type=int, choices=(32, 8), help="normalise the rows and take steps of AdamW, its states in so many bits")
    a = ap.parse_args(argv)
    prototypes = torch.randn(a.width, a.edge ** 2, generator=torch.Generator().manual_seed(1))
    normed = NormedExperts(prototypes, 2 * a.width, bits=a.adamw) if a.adamw else None
    model = normed.experts if normed else MapExperts(prototypes, inner=2 * a.width)
    losses = []
    for s in range(a.steps):
        x, target = rows(a.rows, prototypes, seed=100 + s)
        loss, norm = (normed or model).step(x, target)
        losses.append(float(loss))
        if s % 10 == 0 or s == a.steps - 1:
            print(f"step {s}: loss {losses[-1]:.4f}, gradient norm {float(norm):.3f}, fullest unit "
                  f"{int(model.counts.max())} of {a.rows * model.taken} places", flush=True)
    if normed:
        x, target = rows(a.rows, prototypes, seed=100 + a.steps)
        out, (_, _, (_, idx, _)) = normed.forward(x)
        four, at = normed.answer(x)
        away = [float((t.float() - target.float()).square().sum(1).mean()) for t in (out, four)]
        print(f"{float((at[:, 0] == idx[:, 0]).float().mean()):.1%} of the rows have the same first unit with the map in "
              f"4 bits; loss {away[0]:.4f}, in 4 bits {away[1]:.4f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
