"""Trains a small mixture of experts' feed-forward layer in BFP: each token goes
through two of the experts, an expert is an up-projection, a ReLU and a
down-projection, and the weights take orthogonalised updates.

Every product runs on BFP operands: the weights in both their groupings, the
activations and gradients converted in the experts' order on the way.  The
router is a plain linear layer with softmax over the chosen experts' scores.

    python examples/expert_ffn.py --steps 30
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_15456_amd as fb  # noqa: E402


class Experts:
    """The weights of one projection of all experts: [experts, d_out, d_in] in FP32,
    their momentum, and their two BFP groupings."""

    def __init__(self, experts, d_out, d_in, m, gen):
        self.w = torch.randn((experts, d_out, d_in), generator=gen, device="cuda") / d_in ** 0.5
        self.momentum = torch.zeros_like(self.w)
        self.work = torch.empty(fb.orthogonalize_ws_size(self.w), dtype=torch.uint8, device="cuda")
        self.m = m
        self._convert()

    def _convert(self):
        self.along_in = fb.quantize(self.w, m=self.m)                  # of the forward product
        self.along_out = fb.quantize(self.w, group_axis=1, m=self.m)   # of the gradient to the input

    def forward(self, x, plan):
        return fb.gemm_experts(x, self.along_in, plan)

    def backward(self, dy, dyt, xt, plan):
        """(gradient to the input, gradient of the weights)"""
        return fb.gemm_experts(dy, self.along_out, plan), fb.gemm_experts_grad(dyt, xt, plan)

    def update(self, dw, lr):
        step, _ = fb.orthogonal_update(dw, self.momentum, momentum_out=self.momentum, workspace=self.work)
        # (scaled as the shape asks for: the update's entries are about 1 / sqrt(larger side))
        self.w.add_(step, alpha=-lr * max(1.0, self.w.shape[1] / self.w.shape[2]) ** 0.5)
        self._convert()


def train(steps=30, tokens=2048, d=256, hidden=512, experts=8, top=2, m=4, lr=0.05, seed=0, log=print):
    """Trains on the outputs of a fixed random layer; returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    up, down = Experts(experts, hidden, d, m, gen), Experts(experts, d, hidden, m, gen)
    router = torch.randn((experts, d), generator=gen, device="cuda") / d ** 0.5
    teacher = [torch.randn(s, generator=gen, device="cuda") / s[1] ** 0.5 for s in ((hidden, d), (d, hidden))]
    losses = []
    for step in range(steps):
        x = torch.randn((tokens, d), generator=gen, device="cuda")
        target = torch.relu(x @ teacher[0].t()) @ teacher[1].t()
        # the router's choice, and the plan that all of the layer's calls share
        scores, ids = torch.topk(x @ router.t(), top, dim=1)
        gates = torch.softmax(scores, dim=1)
        plan = fb.expert_plan(ids, experts)
        # forward: both groupings of each activation from one read
        xr, xt = fb.quantize_experts(x, plan, gather=True, m=m)
        h = up.forward(xr, plan)
        ar, at = fb.quantize_experts(torch.relu(h), plan, m=m)
        y = down.forward(ar, plan)
        out = fb.combine_experts(y, plan, gates)
        diff = out - target
        losses.append(float(diff.square().mean()))
        # backward, gradients rounded stochastically
        dy, dgates = fb.combine_experts_grad(diff * (2.0 / tokens), y, plan, gates)
        sr = dict(m=m, rounding="stochastic", seed_rows=4 * step, seed_cols=4 * step + 1)
        dyr, dyt = fb.quantize_experts(dy, plan, **sr)
        da, dw_down = down.backward(dyr, dyt, at, plan)
        dhr, dht = fb.quantize_experts(torch.where(h > 0, da, torch.zeros_like(da)), plan,
                                       **dict(sr, seed_rows=4 * step + 2, seed_cols=4 * step + 3))
        dx, dw_up = up.backward(dhr, dht, xt, plan)
        dx = fb.combine_experts(dx, plan)  # (the sum over a token's experts)
        dscores = gates * (dgates - (gates * dgates).sum(dim=1, keepdim=True))
        drouter = torch.zeros_like(router).index_add_(0, ids.reshape(-1),
                                                      (dscores[:, :, None] * x[:, None, :]).reshape(-1, d))
        assert dx.shape == x.shape  # (for the layer below)
        rate = lr * (1.0 - step / steps)
        up.update(dw_up, rate)
        down.update(dw_down, rate)
        router.add_(drouter, alpha=-0.1)
        if step % 5 == 0 or step + 1 == steps:
            log("step %3d  loss %.4f" % (step, losses[-1]))
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--m", type=int, default=4, help="magnitude bits of every BFP operand")
    a = ap.parse_args()
    train(steps=a.steps, tokens=a.tokens, m=a.m)
