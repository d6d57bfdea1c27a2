"""Local models on a trained map: documents in clusters, each cluster with its own
relation between a document and its target, learned by a mixture of experts
whose gate starts as the map.

    python examples/local_models.py

Trains a map on the documents, makes one expert per unit with the map as the
gate (the best-scored expert is the document's best-matching unit), trains gate
and experts together in bf16 with fp32 masters and 8-bit optimizer states, and
answers single documents.  Prints the mean squared error as it falls, beside that
of one linear model for all documents (least squares).
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_1905_09598_amd as som
import workloads
from paper_1905_09598_amd import local


def make_task(n, d, out, clusters, seed=0):
    """Documents of a Gaussian mixture (n, d) and targets (n, out), a linear map of
    the document that depends on its cluster."""
    x = torch.from_numpy(workloads.gaussian_mixture(n, d, clusters, 0.2, seed=seed)).cuda()
    g = torch.Generator().manual_seed(seed)
    centres = x[torch.randperm(n, generator=g)[:clusters].cuda()]
    which = torch.cdist(x, centres).argmin(1)
    maps = torch.randn(clusters, out, d, generator=g).cuda() / d ** 0.5
    target = torch.empty(n, out, device="cuda")
    for c in range(clusters):
        rows = which == c
        target[rows] = x[rows] @ maps[c].t()
    return x, target


class LocalModels:
    """A gate and two-layer experts, their optimizer, and one training step."""

    def __init__(self, prototypes, out, hidden, k, tau, dtype=torch.bfloat16, lr=3e-3, seed=0):
        units, d = prototypes.shape
        g = torch.Generator().manual_seed(seed)

        def draw(*shape):
            return (torch.randn(*shape, generator=g) / shape[-1] ** 0.5).to(dtype).cuda()

        self.k, self.dtype = k, dtype
        self.gate_w, self.gate_b = local.gate_from_map(prototypes, tau, dtype)
        self.w1, self.w2 = draw(units, hidden, d), draw(units, out, hidden)
        self.b1 = torch.zeros(units, hidden, dtype=dtype, device="cuda")
        self.b2 = torch.zeros(units, out, dtype=dtype, device="cuda")
        self.params = [self.gate_w, self.gate_b, self.w1, self.b1, self.w2, self.b2]
        self.optimizer = local.AdamW(self.params, lr=lr, weight_decay=0.0, bits=8,
                                     master=dtype != torch.float32)

    def _route(self, x):
        scores = local.linear(x, self.gate_w, self.gate_b)
        return scores, local.route(scores, self.k)

    def answer(self, x):
        _, r = self._route(x)
        return local.experts(x, r, self.w1, self.b1, self.w2, self.b2)

    def step(self, x, target):
        """One step on the documents x; returns the error before it (a tensor)."""
        scores, r = self._route(x)
        y, kept = local.experts(x, r, self.w1, self.b1, self.w2, self.b2, keep=True)
        miss = y.float() - target
        dy = (miss * (2.0 / miss.numel())).to(self.dtype)
        d = local.experts_backward(dy, x, r, self.w1, self.b1, self.w2, self.b2, kept)
        dscores = local.route_backward(d.weight, scores, r)
        _, dgate_w, dgate_b = local.linear_backward(dscores, x, self.gate_w)
        self.optimizer.step([dgate_w, dgate_b, d.w1, d.b1, d.w2, d.b2])
        return miss.square().mean()


def run(n=8000, d=256, out=8, clusters=12, rows=6, cols=6, hidden=64, k=2, steps=300, batch=2000,
        say=print):
    x, target = make_task(n, d, out, clusters)
    m = som.Map(rows, cols, d, seed=0)
    m.train(x, 3, 0.5, 0.02, max(rows, cols) / 2, 0.5)
    bmu, qe, te = m.evaluate(x)
    say(f"map {rows} x {cols}: quantization error {qe:.4f}, topographic error {te:.4f}")
    ones = torch.cat([x, torch.ones(n, 1, device="cuda")], 1)
    fit = torch.linalg.lstsq(ones.double(), target.double()).solution
    linear = float((ones.double() @ fit - target).square().mean())
    say(f"one linear model: mean squared error {linear:.4f}")
    model = LocalModels(m.weights, out, hidden, k, tau=0.5 * qe ** 2 / d ** 0.5)
    xs = x.to(model.dtype)
    same = float((model._route(xs)[1].index[:, 0] == bmu).float().mean())
    say(f"the gate's first choice is the best-matching unit for {100 * same:.1f} % of the documents")
    first = last = None
    batch = min(batch, n)
    for s in range(steps):
        at = (s * batch) % (n - batch + 1)
        loss = model.step(xs[at:at + batch], target[at:at + batch])
        if s == 0 or (s + 1) % max(1, steps // 6) == 0:
            last = float(loss)
            first = last if first is None else first
            say(f"step {s + 1:4d}: mean squared error {last:.4f}")
    one = model.answer(xs[:1])
    every = model.answer(xs)
    say(f"one document alone and among all: answers differ by "
        f"{float((one - every[:1]).abs().max()):.1e}")
    return {"linear": linear, "first": first, "last": last, "same": same,
            "alone": float((one.float() - every[:1].float()).abs().max())}


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=300)
    p.add_argument("--documents", type=int, default=8000)
    a = p.parse_args()
    run(n=a.documents, steps=a.steps)


if __name__ == "__main__":
    main()
