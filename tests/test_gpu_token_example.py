"""Replicas of a language model in examples/: all the operators together, their gradients against autograd in 64 bits, single tokens against whole sequences, restarts."""
import importlib.util
import math
import os

import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    spec = importlib.util.spec_from_file_location("token_replicas", os.path.join(ROOT, "examples", "token_replicas.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


class Plain:
    """The operators by elementary operations, for autograd in 64 bits."""

    @staticmethod
    def embedding(table, tokens):
        worker = torch.arange(table.shape[0]).repeat_interleave(tokens.numel() // table.shape[0])
        real = (tokens >= 0) & (tokens < table.shape[1])
        return table[worker, torch.where(real, tokens.long(), 0)] * real[:, None] * float(torch.tensor(math.sqrt(table.shape[2]), dtype=torch.float32))

    @staticmethod
    def norm(s, w):
        return s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6) * w.repeat_interleave(s.shape[0] // w.shape[0], 0)

    @staticmethod
    def scan(v, gate, sequences):
        f, v = torch.sigmoid(gate).view(sequences, -1, v.shape[1]), v.reshape(sequences, -1, v.shape[1])
        h, out = torch.zeros_like(v[:, 0]), []
        for t in range(v.shape[1]):
            h = f[:, t] * h + (1 - f[:, t]) * v[:, t]
            out.append(h)
        return torch.stack(out, 1).flatten(0, 1)

    @staticmethod
    def dropout_add(x, residual, share, seed, step, layer):
        keep, q = O.kept(x.shape[0], x.shape[1], share, seed, step, layer)
        return residual + x * keep / (1 - q)

    @staticmethod
    def cross_entropy(h, table, labels):
        z = torch.bmm(h.view(table.shape[0], -1, h.shape[1]), table.transpose(1, 2)).flatten(0, 1)
        real = (labels >= 0) & (labels < table.shape[1])
        picked = z.gather(1, torch.where(real, labels.long(), 0)[:, None])[:, 0]
        return torch.where(real, torch.logsumexp(z, 1) - picked, 0.0)


def _trainer(E, n=3, classes=37, width=40, blocks=2, sequences=4, length=21):
    t = E.Trainer(E.shards(n, 400, classes, "cuda"), width, blocks, classes, sequences, length, 3, share=0.25)
    g = torch.Generator(device="cuda").manual_seed(5)
    for v in t.p.values():                                  # unlike replicas
        v.add_(0.1 * torch.randn(v.shape, generator=g, device="cuda"))
    return t


def test_gradients_are_autograds_in_64_bits(E):
    """fp32 sums of 21 to 84 terms through two blocks: 1e-4 of the largest gradient of a tensor.  Some tokens and labels are padding."""
    t = _trainer(E)
    t.t = 7
    tokens, labels = t.minibatch()
    tokens[5], labels[20], labels[21] = -1, -1, t.p["table"].shape[1]
    loss, grads = t.gradients(tokens, labels)
    leaves = {k: v.double().cpu().requires_grad_() for k, v in t.p.items()}
    want = E.model(leaves, tokens.cpu(), labels.cpu(), t.n * t.sequences, (t.share, t.seed, t.t), ops=Plain).view(t.n, -1).mean(1)
    exact = torch.autograd.grad(want.sum(), list(leaves.values()))
    assert torch.allclose(loss.double().cpu(), want.detach(), rtol=1e-5)
    for (k, g), e in zip(grads.items(), exact):
        assert float((g.double().cpu() - e).abs().max()) <= 1e-4 * float(e.abs().max()), k


def test_single_tokens_are_the_whole_sequence(E):
    """Each of fp32 sums of 80 terms at most: 1e-4 of the largest value."""
    t = _trainer(E, n=1, sequences=5)
    tokens, _ = t.minibatch()
    width, s = t.p["table"].shape[2], None
    with torch.no_grad():
        s = E.Embedding.apply(t.p["table"], tokens)
        for k in range(2):
            z = E.by_worker(E.Norm.apply(s, t.p["w%d" % k]), t.p["a%d" % k])
            s = s + E.by_worker(E.Scan.apply(z[:, :width], z[:, width:], 5), t.p["b%d" % k])
        whole = E.Norm.apply(s, t.p["w2"]).view(5, -1, width)
    decoder = E.Decoder(t.p, 5)
    for k in range(t.length):
        y = decoder.step(tokens.view(5, -1)[:, k].contiguous())
        assert float((y - whole[:, k]).abs().max()) <= 1e-4 * float(whole.abs().max()), k


def test_training_and_restarts(E, capsys):
    t, more = E.main(["--workers", "3", "--width", "64", "--blocks", "2", "--classes", "50", "--length", "30", "--interval", "4", "--steps", "8"])
    losses = [float(l.split()[-1]) for l in capsys.readouterr().out.splitlines() if l.startswith("step")]
    assert len(losses) == 2 and all(math.isfinite(x) for x in losses)
    for v in t.p.values():                                  # the last step was a restart
        assert all(torch.equal(v[0], v[i]) for i in range(1, v.shape[0])) and bool(v.isfinite().all())
    assert more.shape == (3, 8) and bool(((more >= 0) & (more < 50)).all())
