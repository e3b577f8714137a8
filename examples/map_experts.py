"""Local experts on a map: dense rows are scored against a map's units, routed to their best two, and each unit's
expert (a two-layer network) learns what holds in its region of the map.

    python examples/map_experts.py [--steps N]

One step is what a training program does with the dense operators: scores (``dense.linear`` with the codebook and
-|w|^2 / 2 as its bias, so that the highest score is the best-matching unit), routing with a bias that balances the
units' loads, the experts with the rows as residual, their gradients, the gate's gradient through the routing weights,
and all gradients clipped together. The rows and the function to learn are synthetic.
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

    def forward(self, x, keep=True):
        """(out, what the backward pass needs) of rows x [N, width]."""
        W, W1, b1, W2, b2 = self.params
        # the norms of the prototypes as they are held now: the search's own pass over the widened codebook
        self.gate_bias = (-0.5 * som.codebook_norms(W.float(), W.shape[0], W.shape[1])).float()
        scores = dense.linear(x, W, self.gate_bias, out_dtype=torch.float32)
        idx, w = dense.route(scores, self.taken, bias=self.balance, weights_dtype=x.dtype, counts=self.counts)
        need = dense.experts_workspace_bytes(x.shape[0], self.taken, self.units, W1.shape[1], W1.shape[2], keep)
        if self.workspace is None or self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        out = dense.experts(x, idx, w, W1, b1, W2, b2, residual=x, keep=keep, workspace=self.workspace)
        return out, (scores, idx, w)

    def backward(self, x, kept, dout):
        """The gradients of the parameters, in their order, with the gate's bias held, and that of this bias."""
        W, W1, b1, W2, b2 = self.params
        scores, idx, w = kept
        _, dw, *expert_grads = dense.experts_bwd(x, idx, w, W1, W2, b2, dout, workspace=self.workspace)
        dscores = dense.route_bwd(scores, idx, dw, bias=self.balance).to(x.dtype)
        dbias = torch.empty_like(self.gate_bias)
        _, dW, _ = dense.linear_bwd(x, W, dscores, out=(None, torch.empty_like(W), dbias))
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
        # units that take more than their share become less attractive, without a gradient
        share = self.counts.float() / max(1.0, float(x.shape[0] * self.taken)) * self.units
        self.balance += 0.05 * (1.0 - share)
        return miss.square().sum(1).mean(), norm


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
    a = ap.parse_args(argv)
    prototypes = torch.randn(a.width, a.edge ** 2, generator=torch.Generator().manual_seed(1))
    model = MapExperts(prototypes, inner=2 * a.width)
    losses = []
    for s in range(a.steps):
        x, target = rows(a.rows, prototypes, seed=100 + s)
        loss, norm = model.step(x, target)
        losses.append(float(loss))
        if s % 10 == 0 or s == a.steps - 1:
            print(f"step {s}: loss {losses[-1]:.4f}, gradient norm {float(norm):.3f}, fullest unit "
                  f"{int(model.counts.max())} of {a.rows * model.taken} places", flush=True)
    return losses


if __name__ == "__main__":
    main()
