"""The residual classifier of examples/: its gradients against autograd in 64 bits, its training, restarts and 8-bit evaluation."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    spec = importlib.util.spec_from_file_location("residual_replicas", os.path.join(ROOT, "examples", "residual_replicas.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _plain_norm(stream, f, w):
    s = stream + f
    y = s / torch.sqrt((s * s).mean(1, keepdim=True) + 1e-6)
    return y * w.repeat_interleave(y.shape[0] // w.shape[0], 0), s


def test_gradients_are_autograds_in_64_bits(E):
    """fp32 products of depth 24 to 40 through three blocks: 1e-4 of the largest gradient of a tensor."""
    torch.manual_seed(0)
    n, b, d, width, classes = 3, 5, 24, 40, 7
    x = torch.randn(n, 16, d, device="cuda")
    y = torch.randint(classes, (n, 16), device="cuda", dtype=torch.int32)
    t = E.Trainer(x, y, width, 3, classes, b, 4)
    for v in t.p.values():
        v.add_(0.1 * torch.randn_like(v))                   # unlike replicas
    rows, labels = x[:, :b].flatten(0, 1).contiguous(), y[:, :b].flatten().long()
    loss, grads = t.gradients(rows, labels)
    leaves = {k: v.double().cpu().requires_grad_() for k, v in t.p.items()}
    out = E.logits(leaves, rows.double().cpu(), _plain_norm)
    want = torch.nn.functional.cross_entropy(out, labels.cpu(), reduction="none").view(n, -1).mean(1)
    exact = torch.autograd.grad(want.sum(), list(leaves.values()))
    assert torch.allclose(loss.double().cpu(), want.detach(), rtol=1e-5)
    for (k, g), e in zip(grads.items(), exact):
        assert float((g.double().cpu() - e).abs().max()) <= 1e-4 * float(e.abs().max()), k


def test_training_restarts_and_eight_bit_rows(E, capsys):
    t, exact, eight, off = E.main(["--workers", "4", "--width", "96", "--blocks", "2", "--interval", "4", "--epochs", "10", "--rows", "256",
                                   "--noise", "6"])
    losses = [float(l.split()[-1]) for l in capsys.readouterr().out.splitlines() if l.startswith("epoch")]
    assert losses[-1] < 0.5 * losses[0]
    for v in t.p.values():                                  # the last step was a restart
        assert all(torch.equal(v[0], v[i]) for i in range(1, v.shape[0]))
    assert exact > 0.9
    # an e4m3 row is off by 2^-4 / sqrt(3) of its values at most, through three norms and the layers behind them
    assert abs(eight - exact) <= 0.05 and off <= 0.1
