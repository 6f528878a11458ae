"""Replicas of a recurrent language model under Parallel Restarted SGD.

    python examples/token_replicas.py [--workers 8] [--width 128] [--blocks 2] [--interval 8] [--steps 64] [--classes 512]

N workers hold a replica each and take local steps on sequences of their own shards; every `interval` steps the average overwrites
all replicas (Algorithm 1).  Rows of all workers stand one behind another.  A replica is

    s <- sqrt(width) E[token]                                       (prsgd_embedding)
    y <- s / rms(s) * w,  (v, gate) <- y A                          (prsgd_rms_norm)
    h <- gated scan of v along every sequence                       (prsgd_gated_scan)
    s <- s + dropout(h B)                                           (prsgd_dropout)
    loss <- cross entropy of (s / rms(s) * w) E^T                   (prsgd_linear_cross_entropy, the embedding's table once more)

with the gradients of each.  The matrices A and B move by updates of unit singular values (prsgd_muon_step), the rest by momentum SGD.  The averaged
model goes on from a prompt token by token, its scans' states in place.  The other products are torch's.
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

Function = torch.autograd.Function


class Embedding(Function):
    @staticmethod
    def forward(ctx, table, tokens):
        ctx.save_for_backward(table, tokens)
        return prsgd.prsgd_embedding(tokens, table, scale=math.sqrt(table.shape[2]))

    @staticmethod
    def backward(ctx, dy):
        table, tokens = ctx.saved_tensors
        return prsgd.prsgd_embedding_backward(dy.contiguous(), tokens, table, scale=math.sqrt(table.shape[2])), None


class Norm(Function):
    @staticmethod
    def forward(ctx, s, w):
        y, _, rstd = prsgd.prsgd_rms_norm(s, w)
        ctx.save_for_backward(s, rstd, w)
        return y

    @staticmethod
    def backward(ctx, dy):
        return prsgd.prsgd_rms_norm_backward(dy.contiguous(), *ctx.saved_tensors)


class Scan(Function):
    """Along sequences of equal length."""

    @staticmethod
    def forward(ctx, v, gate, sequences):
        h, _ = prsgd.prsgd_gated_scan(v, gate, sequences=sequences)
        ctx.save_for_backward(v, gate, h)
        ctx.sequences = sequences
        return h

    @staticmethod
    def backward(ctx, dh):
        dv, dgate, _ = prsgd.prsgd_gated_scan_backward(dh.contiguous(), *ctx.saved_tensors, sequences=ctx.sequences)
        return dv, dgate, None


class DropoutAdd(Function):
    """residual + dropout(x); the mask is made again from its counter."""

    @staticmethod
    def forward(ctx, x, residual, share, seed, step, layer):
        ctx.mask = share, seed, step, layer
        return prsgd.prsgd_dropout(x, share, seed, step=step, layer=layer, residual=residual)

    @staticmethod
    def backward(ctx, dy):
        share, seed, step, layer = ctx.mask
        dy = dy.contiguous()
        return prsgd.prsgd_dropout(dy, share, seed, step=step, layer=layer), dy, None, None, None, None


class LinearCrossEntropy(Function):
    """Loss of every row through the tables as last matrices."""

    @staticmethod
    def forward(ctx, h, table, labels):
        loss, lse = prsgd.prsgd_linear_cross_entropy(h, table, labels, classes_first=True)
        ctx.save_for_backward(h, table, labels, lse)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        return (*prsgd.prsgd_linear_cross_entropy_backward(dloss.contiguous(), *ctx.saved_tensors, classes_first=True), None)


class Kernels:
    """The operators as model() calls them."""
    embedding, norm, scan, cross_entropy = Embedding.apply, Norm.apply, Scan.apply, LinearCrossEntropy.apply
    dropout_add = DropoutAdd.apply


def by_worker(rows: torch.Tensor, matrices: torch.Tensor) -> torch.Tensor:
    """Every worker's rows times its own matrix."""
    return torch.bmm(rows.view(matrices.shape[0], -1, rows.shape[1]), matrices).view(rows.shape[0], matrices.shape[2])


def init(workers: int, width: int, blocks: int, classes: int, seed: int, device) -> dict:
    """The same point on every worker."""
    g = torch.Generator(device=device).manual_seed(seed)

    def matrix(rows, cols, scale):
        return (torch.randn((1, rows, cols), generator=g, device=device) * scale).repeat(workers, 1, 1)

    p = {"table": matrix(classes, width, width ** -0.5)}
    for k in range(blocks):
        p["a%d" % k], p["b%d" % k] = matrix(width, 2 * width, width ** -0.5), matrix(width, width, 0.5 * width ** -0.5)
    for k in range(blocks + 1):
        p["w%d" % k] = torch.ones((workers, width), device=device)
    return p


def blocks_of(p: dict) -> int:
    return sum(k.startswith("a") for k in p)


def model(p: dict, tokens, labels, sequences: int, dropout=(0.0, 0, 0), ops=Kernels) -> torch.Tensor:
    """Loss of every row; tokens and labels int32 [N * sequences of a worker * length]."""
    width = p["table"].shape[2]
    s = ops.embedding(p["table"], tokens)
    for k in range(blocks_of(p)):
        z = by_worker(ops.norm(s, p["w%d" % k]), p["a%d" % k])
        h = ops.scan(z[:, :width], z[:, width:], sequences)
        s = ops.dropout_add(by_worker(h, p["b%d" % k]), s, *dropout, k)
    return ops.cross_entropy(ops.norm(s, p["w%d" % blocks_of(p)]), p["table"], labels)


class Decoder:
    """One replica, one token of every sequence at a time."""

    def __init__(self, p: dict, sequences: int):
        self.p = p
        self.states = [torch.zeros((sequences, p["table"].shape[2]), device=p["table"].device) for _ in range(blocks_of(p))]

    @torch.no_grad()
    def step(self, tokens):
        """Rows in front of the last matrix; tokens int32 [sequences]."""
        p, width = self.p, self.p["table"].shape[2]
        s = prsgd.prsgd_embedding(tokens, p["table"], scale=math.sqrt(width))
        for k, state in enumerate(self.states):
            z = by_worker(prsgd.prsgd_rms_norm(s, p["w%d" % k])[0], p["a%d" % k])
            h, _ = prsgd.prsgd_gated_scan(z[:, :width], z[:, width:], initial=state, last=state)
            s = s + by_worker(h, p["b%d" % k])
        return prsgd.prsgd_rms_norm(s, p["w%d" % len(self.states)])[0]


class Trainer:
    def __init__(self, text, width, blocks, classes, sequences, length, interval, share=0.1, seed=1, matrix_rate=0.01, rate=0.5, momentum=0.9):
        """text: tokens of every worker's shard, [N][tokens]."""
        self.text, self.sequences, self.length, self.interval, self.share, self.seed = text, sequences, length, interval, share, seed
        self.matrix_rate, self.rate, self.momentum = matrix_rate, rate, momentum
        self.n, self.t = text.shape[0], 0
        self.p = init(self.n, width, blocks, classes, seed, text.device)
        self.m = {k: torch.zeros_like(v) for k, v in self.p.items()}

    def minibatch(self):
        """Tokens and the ones behind them, of sequences that start in the first places of a worker's shard (the sampler takes a power of two of these)."""
        places = 1 << ((self.text.shape[1] - self.length).bit_length() - 1)
        at = prsgd.prsgd_sample_indices(self.seed, self.n, self.sequences, places, self.t, 1, device=self.text.device)[0].long()
        at = at[:, :, None] + torch.arange(self.length + 1, device=at.device)
        rows = self.text.gather(1, at.flatten(1)).view(self.n, self.sequences, -1)
        return rows[:, :, :-1].reshape(-1), rows[:, :, 1:].reshape(-1)

    def gradients(self, tokens, labels):
        leaves = {k: v.detach().requires_grad_() for k, v in self.p.items()}
        loss = model(leaves, tokens, labels, self.n * self.sequences, (self.share, self.seed, self.t))
        loss = loss.view(self.n, -1).mean(1)
        grads = torch.autograd.grad(loss.sum(), list(leaves.values()))
        return loss.detach(), dict(zip(leaves, grads))

    def step(self):
        """A local step of every worker, and the restart behind every interval-th."""
        self.t += 1
        loss, grads = self.gradients(*self.minibatch())
        for k, g in grads.items():
            if k[0] in "ab":
                prsgd.prsgd_muon_step(self.p[k], g, self.m[k], self.matrix_rate, momentum=self.momentum)
            else:
                self.m[k].mul_(self.momentum).add_(g)
                self.p[k].add_(self.m[k], alpha=-self.rate)
        if self.t % self.interval == 0:
            for v in self.p.values():
                v.copy_(v.mean(0, keepdim=True).expand_as(v))
        return loss

    def average(self):
        return {k: v.mean(0, keepdim=True) for k, v in self.p.items()}

    @torch.no_grad()
    def go_on(self, prompt, count):
        """Likeliest continuation of prompts [sequences][length] by the averaged model."""
        p = self.average()
        decoder, out = Decoder(p, prompt.shape[0]), []
        for t in range(prompt.shape[1]):
            y = decoder.step(prompt[:, t].contiguous())
        for _ in range(count):
            out.append((y @ p["table"][0].t()).argmax(1).to(torch.int32))
            y = decoder.step(out[-1])
        return torch.stack(out, 1)


def shards(workers: int, tokens: int, classes: int, device, seed=3):
    """Texts in which a token mostly follows from the one before it, by the same rule everywhere, from places of their own."""
    g = torch.Generator(device=device).manual_seed(seed)
    noise = torch.randint(0, 3, (workers, tokens), generator=g, device=device)
    step = 1 + (torch.arange(workers, device=device)[:, None] % 2)
    return ((noise + step).cumsum(1) % classes).to(torch.int32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--width", type=int, default=128)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--classes", type=int, default=512)
    ap.add_argument("--sequences", type=int, default=8, help="of a worker's minibatch")
    ap.add_argument("--length", type=int, default=64)
    ap.add_argument("--interval", type=int, default=8)
    ap.add_argument("--steps", type=int, default=64)
    a = ap.parse_args(argv)
    text = shards(a.workers, 4096, a.classes, "cuda")
    t = Trainer(text, a.width, a.blocks, a.classes, a.sequences, a.length, a.interval)
    for k in range(a.steps):
        loss = t.step()
        if (k + 1) % a.interval == 0:
            print("step %3d  loss %.4f" % (k + 1, float(loss.mean())), flush=True)
    more = t.go_on(text[:, :32], 8)
    print("continuations:", more.tolist()[:2])
    return t, more


if __name__ == "__main__":
    main()
