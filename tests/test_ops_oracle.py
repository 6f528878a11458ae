"""The 64-bit forms of the operators, held to what their definitions say (no GPU)."""
import pytest
import torch

import ops_oracle as O


@pytest.mark.parametrize("shape", [(3, 4), (7, 3), (1, 5), (6, 6)])
def test_the_products_are_the_polynomial_of_the_singular_values(shape):
    torch.manual_seed(1)
    g = torch.randn((1,) + shape, dtype=torch.float64)
    u, s, vt = torch.linalg.svd(g[0], full_matrices=False)
    s = s / (torch.linalg.norm(s) + 1e-7)
    a, b, c = (float(torch.tensor(v)) for v in O.NS)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert torch.allclose(O.orthogonalize(g)[0], u @ torch.diag(s) @ vt, rtol=0, atol=1e-8)
    assert 0.6 < float(s.min()) and float(s.max()) < 1.2


def test_singular_values_from_two_thousandths_on_come_out_near_one():
    # the local maximum of p is 1.2024 (at 0.554), and p(1.2024) = 0.6818 is the least that any later step leaves
    a, b, c = O.NS
    s = torch.logspace(-2.69, 0, 2000, dtype=torch.float64)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    assert 0.68 < float(s.min()) and float(s.max()) < 1.21


@pytest.mark.parametrize("workers,rows,width", [(1, 1, 1), (1, 3, 5), (2, 4, 7), (3, 1, 2)])
@pytest.mark.parametrize("shared", [False, True])
def test_norm_gradients_are_those_of_differences_and_of_autograd(workers, rows, width, shared):
    torch.manual_seed(2)
    n = workers * rows
    x, res = torch.randn(n, width, dtype=torch.float64), torch.randn(n, width, dtype=torch.float64)
    w = torch.randn(width, dtype=torch.float64) if shared else torch.randn(workers, width, dtype=torch.float64)
    dy, ds = torch.randn(n, width, dtype=torch.float64), torch.randn(n, width, dtype=torch.float64)

    def objective(x, res, w):
        y, s, _ = O.rms_norm(x, w, res)
        return float((y * dy).sum() + (s * ds).sum())

    _, s, rstd = O.rms_norm(x, w, res)
    dx, dw = O.rms_norm_backward(dy, s, rstd, w, ds)
    h = 1e-6
    for t, grad, at in ((x, dx, 0), (res, dx, 1), (w, dw, 2)):
        for i in range(t.numel()):
            args = [x.clone(), res.clone(), w.clone()]
            args[at].view(-1)[i] += h
            up = objective(*args)
            args[at].view(-1)[i] -= 2 * h
            assert (up - objective(*args)) / (2 * h) == pytest.approx(float(grad.reshape(-1)[i]), rel=1e-5, abs=1e-7)
    x, w = x.requires_grad_(), w.requires_grad_()
    y, s, _ = O.rms_norm(x, w, res)
    ((y * dy).sum() + (s * ds).sum()).backward()
    assert torch.allclose(x.grad, dx, atol=1e-12) and torch.allclose(w.grad, dw, atol=1e-12)
