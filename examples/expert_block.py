"""Train a residual classifier of expert blocks on one MI355X.

    python examples/expert_block.py [--steps N] [--blocks B] [--width D] [--experts E] [--k K] [--dtype bf16|fp32]

The block operators (paper_1710_02368_amd.block) as a training program uses
them, forwards and backwards, on a seeded synthetic workload (MNIST-shaped
stand-in data):

    r_0 = x W_in                                       h_0 = norm(r_0)
    block b:  route h_b to k of E experts; y = the experts' two-layer MLP with
              ReLU and dropout; f = the weighted sum of a row's experts
              r_{b+1} = r_b + alpha * gate * dropout(norm(f))    h_{b+1} = norm(r_{b+1})
    logits = h_B W_out

The input and output layers are the experts' product with one expert.  The
loss is the softmax cross-entropy; the update is plain SGD on float32 master
weights, with copies in the compute type.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

import workloads as W  # noqa: E402
from paper_1710_02368_amd import block  # noqa: E402


class ExpertBlocks:
    """Parameters, one training step and the forward pass of the model.  The
    pass and its gradients can be captured into a graph after a first eager call
    with as many rows; replays draw the masks of steps_done at the time."""

    def __init__(self, inputs, classes, blocks=2, width=256, hidden=256, experts=8, k=2, rate=0.1, alpha=0.5,
                 dtype=torch.bfloat16, seed=1):
        self.blocks, self.k, self.rate, self.alpha, self.dtype, self.seed = blocks, k, rate, alpha, dtype, seed
        self.steps_done = torch.zeros(1, dtype=torch.int32, device="cuda")  # moves the masks on
        g = torch.Generator().manual_seed(seed)
        normal = lambda *shape: (torch.randn(*shape, generator=g) * (2.0 / shape[-1]) ** 0.5).cuda()
        p = {"in.w": normal(1, width, inputs), "in.b": torch.zeros(1, width, device="cuda"),
             "out.w": normal(1, classes, width), "out.b": torch.zeros(1, classes, device="cuda"),
             "pre0": torch.ones(width, device="cuda")}
        for b in range(blocks):
            p.update({f"{b}.router": normal(1, experts, width) * 0.5,
                      f"{b}.w1": normal(experts, hidden, width), f"{b}.b1": torch.zeros(experts, hidden, device="cuda"),
                      f"{b}.w2": normal(experts, width, hidden), f"{b}.b2": torch.zeros(experts, width, device="cuda"),
                      f"{b}.gate": torch.ones(width, device="cuda"), f"{b}.post": torch.ones(width, device="cuda"),
                      f"{b}.pre": torch.ones(width, device="cuda")})
        self.params = p
        self.copies = {n: t.to(dtype) for n, t in p.items() if t.dim() == 3}  # what the products read
        self._offsets = {}

    def _all_rows(self, rows):
        """The offsets of a product with one expert, made once for a number of
        rows (by a copy from the host, which a graph cannot hold)."""
        if rows not in self._offsets:
            self._offsets[rows] = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        return self._offsets[rows]

    def forward(self, x, train=False):
        """Logits, and with train what the backward pass needs."""
        p, c = self.params, self.copies
        one = self._all_rows(x.shape[0])
        drop = lambda i: (self.rate, self.seed, i, self.steps_done) if train and self.rate else None
        r = block.experts(x, one, c["in.w"], p["in.b"])
        r, h, saved = block.norms(r, None, None, p["pre0"])
        kept = [(one, x, saved)]
        for b in range(self.blocks):
            logits = block.experts(h, one, c[f"{b}.router"])
            route = block.route(logits, self.k)
            xs = block.dispatch(h, route)
            a = block.experts(xs, route.offsets, c[f"{b}.w1"], p[f"{b}.b1"], relu=True, dropout=drop(2 * b))
            y = block.experts(a, route.offsets, c[f"{b}.w2"], p[f"{b}.b2"])
            f = block.combine(y, route)
            r, h2, saved = block.norms(r, f, p[f"{b}.post"], p[f"{b}.pre"], gate=p[f"{b}.gate"], alpha=self.alpha,
                                       dropout=drop(2 * b + 1))
            kept.append((h, logits, route, xs, a, y, f, r, saved, drop(2 * b + 1)))
            h = h2
        z = block.experts(h, one, c["out.w"], p["out.b"])
        return (z, (kept, h, r)) if train else z

    def gradients(self, x, labels):
        """(mean loss, gradients of all parameters) on one mini-batch."""
        p, c = self.params, self.copies
        z, (kept, h, r) = self.forward(x, train=True)
        logp = torch.log_softmax(z.float(), 1)
        loss = -logp.gather(1, labels.long()[:, None]).mean()
        dz = torch.exp(logp)
        dz.scatter_add_(1, labels.long()[:, None], torch.full_like(dz[:, :1], -1.0))
        dz = (dz / x.shape[0]).to(self.dtype)
        one, x, saved0 = kept[0]
        g = {}
        dh, g["out.w"], g["out.b"] = block.experts_backward(h, dz, one, c["out.w"])
        dr = None
        for b in reversed(range(self.blocks)):
            hb, logits, route, xs, a, y, f, rb, saved, drop = kept[b + 1]
            dr, df, g[f"{b}.gate"], g[f"{b}.post"], g[f"{b}.pre"] = block.norms_backward(
                dr, dh, rb, f, p[f"{b}.post"], p[f"{b}.pre"], saved, gate=p[f"{b}.gate"], alpha=self.alpha, dropout=drop)
            dy, dweights = block.combine_backward(df, y, route)
            da, g[f"{b}.w2"], g[f"{b}.b2"] = block.experts_backward(a, dy, route.offsets, c[f"{b}.w2"], relu_input=True,
                                                                    input_rate=self.rate)
            dxs, g[f"{b}.w1"], g[f"{b}.b1"] = block.experts_backward(xs, da, route.offsets, c[f"{b}.w1"])
            dlogits = block.route_backward(logits, route, dweights)
            dh, g[f"{b}.router"], _ = block.experts_backward(hb, dlogits, one, c[f"{b}.router"])
            dh = dh + block.dispatch_backward(dxs, route)
        dr, _, _, _, g["pre0"] = block.norms_backward(dr, dh, saved0.residual, None, None, p["pre0"], saved0)
        _, g["in.w"], g["in.b"] = block.experts_backward(x, dr, one, c["in.w"], need_dx=False)
        return loss, g

    def step(self, x, labels, eta):
        """One SGD step; returns the mini-batch's mean loss before it."""
        loss, g = self.gradients(x, labels)
        for n, t in self.params.items():
            t.add_(g[n], alpha=-eta)
            if n in self.copies:
                self.copies[n].copy_(t)
        self.steps_done += 2 * self.blocks
        return loss


def train(steps=60, batch=256, blocks=2, width=256, hidden=256, experts=8, k=2, rate=0.1, eta=0.05, dtype="bf16",
          dims=(784, 10), rows=8192, seed=1, log=None):
    """Train on a synthetic workload; returns the losses of the steps and the accuracy on the training rows."""
    wl = W.small_workload("expert_blocks", (dims[0], 64, dims[1]), n=1, lam=1, m=batch, eta=eta, rounds=1, N=rows,
                          data="sparse_teacher2", seed=seed)
    X, y = W.make_data(wl)
    t = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
    x, y = torch.from_numpy(X).cuda().to(t), torch.from_numpy(y).cuda()
    model = ExpertBlocks(dims[0], dims[1], blocks, width, hidden, experts, k, rate, dtype=t, seed=seed)
    losses = []
    for s in range(steps):
        at = torch.arange(s * batch, (s + 1) * batch, device="cuda") % rows
        losses.append(model.step(x[at], y[at], eta).item())
        if log and (s % 10 == 0 or s == steps - 1):
            log(f"step {s}: loss {losses[-1]:.4f}")
    accuracy = (model.forward(x).float().argmax(1) == y).float().mean().item()
    return losses, accuracy


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=256)
    ap.add_argument("--experts", type=int, default=8)
    ap.add_argument("--k", type=int, default=2)
    ap.add_argument("--eta", type=float, default=0.05)
    ap.add_argument("--rate", type=float, default=0.1)
    ap.add_argument("--dtype", choices=("bf16", "fp32"), default="bf16")
    a = ap.parse_args()
    _, acc = train(log=lambda s: print(s, flush=True), **vars(a))
    print(f"accuracy on the training rows: {acc:.4f}")
