"""Replicas of a residual classifier under Parallel Restarted SGD, with normalised rows and orthogonalised updates.

    python examples/residual_replicas.py [--workers 8] [--width 256] [--blocks 3] [--interval 8] [--epochs 24]

N workers hold a replica each, batched as [N][rows][cols], and take local steps on minibatches of their own shards; every
`interval` steps the average overwrites all replicas (Algorithm 1).  A block is

    s <- s + f,   y = s / rms(s) * w,   f = relu(y A) B        (prsgd_rms_norm and its gradients, a weight vector per worker)

and its matrices A and B move by updates of unit singular values (prsgd_muon_step); what is no hidden matrix (first and last
layer, norm weights) takes momentum SGD.  The averaged model is evaluated with its rows in fp32 and in 8 bits
(prsgd_rms_norm_fp8).  The other products are torch's.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1807_06629_amd import prsgd                      # noqa: E402
from workloads import get_workload, make_inputs             # noqa: E402


class ResidualNorm(torch.autograd.Function):
    """(y, s) of s = stream + f, y = s / rms(s) * w; rows of all workers one behind another, w [workers][width]."""

    @staticmethod
    def forward(ctx, stream, f, w):
        y, s, rstd = prsgd.prsgd_rms_norm(stream, w, residual=f)
        ctx.save_for_backward(s, rstd, w)
        return y, s

    @staticmethod
    def backward(ctx, dy, ds):
        s, rstd, w = ctx.saved_tensors
        dx, dw = prsgd.prsgd_rms_norm_backward(dy.contiguous(), s, rstd, w, dsum=None if ds is None else ds.contiguous())
        return dx, dx, dw


def by_worker(rows: torch.Tensor, matrices: torch.Tensor) -> torch.Tensor:
    """Every worker's rows times its own matrix."""
    n = matrices.shape[0]
    return torch.bmm(rows.view(n, -1, rows.shape[1]), matrices).view(rows.shape[0], matrices.shape[2])


def init(workers: int, d_in: int, width: int, blocks: int, classes: int, seed: int, device) -> dict:
    """The same point on every worker."""
    g = torch.Generator(device=device).manual_seed(seed)

    def matrix(rows, cols, scale=1.0):
        return (torch.randn((1, rows, cols), generator=g, device=device) * (scale / math.sqrt(rows))).repeat(workers, 1, 1)

    p = {"first": matrix(d_in, width), "last": matrix(width, classes)}
    for k in range(blocks):
        p["a%d" % k], p["b%d" % k] = matrix(width, width, math.sqrt(2.0)), matrix(width, width, 0.5)
    for k in range(blocks + 1):
        p["w%d" % k] = torch.ones((workers, width), device=device)
    return p


def logits(p: dict, rows: torch.Tensor, norm) -> torch.Tensor:
    """norm(stream, f, w) -> (y, stream)."""
    blocks = sum(k.startswith("a") for k in p)
    stream = by_worker(rows, p["first"])
    f = torch.zeros_like(stream)
    for k in range(blocks):
        y, stream = norm(stream, f, p["w%d" % k])
        f = by_worker(torch.relu(by_worker(y, p["a%d" % k])), p["b%d" % k])
    return by_worker(norm(stream, f, p["w%d" % blocks])[0], p["last"])


def norm_fp8(stream, f, w):
    """Rows in 8 bits, as a product in 8 bits would take them."""
    q, scales, s = prsgd.prsgd_rms_norm_fp8(stream, w, residual=f)
    return q.float() * scales[:, None], s


class Trainer:
    def __init__(self, features, labels, width, blocks, classes, batch, interval, seed=1, matrix_rate=0.02, rate=0.1, momentum=0.9):
        self.features, self.labels, self.batch, self.interval = features, labels, batch, interval
        self.matrix_rate, self.rate, self.momentum = matrix_rate, rate, momentum
        self.n, self.rows, d_in = features.shape
        self.seed, self.t = seed, 0
        self.p = init(self.n, d_in, width, blocks, classes, seed, features.device)
        self.m = {k: torch.zeros_like(v) for k, v in self.p.items()}
        self.hidden = [k for k in self.p if k[0] in "ab"]
        self.workspace = torch.empty(prsgd.prsgd_orthogonalize_workspace_bytes((self.n, width, width), torch.float32),
                                     dtype=torch.uint8, device=features.device)

    def gradients(self, x, y):
        """Minibatch loss of every worker and its gradients; x [N * batch][d], y [N * batch]."""
        leaves = {k: v.detach().requires_grad_() for k, v in self.p.items()}
        out = logits(leaves, x, ResidualNorm.apply)
        loss = torch.nn.functional.cross_entropy(out, y, reduction="none").view(self.n, -1).mean(1)
        grads = torch.autograd.grad(loss.sum(), list(leaves.values()))
        return loss.detach(), dict(zip(leaves, grads))

    def step(self):
        """A local step of every worker, and the restart behind every interval-th."""
        self.t += 1
        index = prsgd.prsgd_sample_indices(self.seed, self.n, self.batch, self.rows, self.t, 1, device=self.features.device)[0].long()
        worker = torch.arange(self.n, device=index.device)[:, None]
        loss, grads = self.gradients(self.features[worker, index].flatten(0, 1), self.labels[worker, index].flatten().long())
        for k, g in grads.items():
            if k in self.hidden:
                prsgd.prsgd_muon_step(self.p[k], g, self.m[k], self.matrix_rate, momentum=self.momentum, workspace=self.workspace)
            else:
                self.m[k].mul_(self.momentum).add_(g)
                self.p[k].add_(self.m[k], alpha=-self.rate)
        if self.t % self.interval == 0:
            for v in self.p.values():
                v.copy_(v.mean(0, keepdim=True).expand_as(v))
        return loss

    @torch.no_grad()
    def evaluate(self, norm):
        """Accuracy of the averaged model over all shards."""
        mean = {k: v.mean(0, keepdim=True) for k, v in self.p.items()}
        out = logits(mean, self.features.flatten(0, 1), norm)
        return float((out.argmax(1) == self.labels.flatten()).float().mean()), out


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--blocks", type=int, default=3)
    ap.add_argument("--interval", type=int, default=8)
    ap.add_argument("--epochs", type=int, default=24)
    ap.add_argument("--rows", type=int, default=1024)
    ap.add_argument("--noise", type=float, default=12.0, help="added to the mixture, whose classes lie 40 apart")
    a = ap.parse_args(argv)
    w = get_workload("c2").scaled(n_workers=a.workers, rows_per_worker=a.rows, dirichlet_alpha=0.3)
    data = make_inputs(w)
    features = torch.from_numpy(data["features"]).cuda()
    features += a.noise * torch.randn(features.shape, generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    t = Trainer(features, torch.from_numpy(data["targets"]).cuda(), a.width, a.blocks, w.n_classes, w.batch,
                a.interval)
    for epoch in range(a.epochs):
        for _ in range(a.interval):
            loss = t.step()
        print("epoch %2d  loss %.4f" % (epoch + 1, float(loss.mean())), flush=True)
    exact, in_fp32 = t.evaluate(ResidualNorm.apply)
    eight, in_fp8 = t.evaluate(norm_fp8)
    off = float((in_fp8 - in_fp32).norm() / in_fp32.norm())
    print("accuracy of the averaged model: %.4f, rows in 8 bits %.4f (logits %.4f apart)" % (exact, eight, off))
    return t, exact, eight, off


if __name__ == "__main__":
    main()
