"""Updates whose norm is small beside eps: X_0 = G / (||G|| + eps) is as small, and as exact, as its type allows.

X_0's relative rounding is that of any other matrix, a step's linear part makes both larger alike, and what the other parts add is
smaller the smaller X_0 is: tolerances are those of test_gpu_orthogonalize.py.
"""
import pytest
import torch

import ops_oracle as O
from test_gpu_orthogonalize import BF16, F32, P, TOL, _err, _matrices   # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu
EPS = 1e-7


def _of_norm(count, rows, cols, dtype, ratio, seed=0):
    g = _matrices(count, rows, cols, F32, seed=seed)
    return (g * (ratio * EPS / g.flatten(1).norm(dim=1)).view(-1, 1, 1)).to(dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ratio", [1.0, 1e-2, 1e-4, 1e-5, 1e-7, 1e-10, 1e-20])
@pytest.mark.parametrize("rows,cols", [(12, 200), (70, 100), (100, 70), (300, 301), (1000, 1000)])
def test_norms_below_eps(P, rows, cols, ratio, dtype):                                         # noqa: F811
    g = _of_norm(2, rows, cols, dtype, ratio, seed=rows)
    assert _err(P.prsgd_orthogonalize(g, eps=EPS), O.orthogonalize(g, eps=EPS)) <= TOL[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_matrices_of_every_size_in_one_call(P, dtype):                                         # noqa: F811
    """Each goes by its own norm."""
    g = torch.cat([_of_norm(1, 90, 130, dtype, r, seed=k) for k, r in enumerate((1e6, 0.0, 1.0, 1e-6, 1e-12, 1e3, 1e-3))])
    out, want = P.prsgd_orthogonalize(g, eps=EPS), O.orthogonalize(g.cpu(), eps=EPS)
    assert bool((out[1] == 0).all())
    keep = [0, 2, 3, 4, 5, 6]
    assert _err(out[keep], want[keep]) <= TOL[dtype]
    for k in keep:
        assert torch.equal(P.prsgd_orthogonalize(g[k:k + 1].contiguous(), eps=EPS)[0], out[k])


@pytest.mark.parametrize("coefficients,steps", [(O.NS, 1), (O.NS, 2), (O.NS, 7), ((1.5, -0.5, 0.0), 12), ((0.5, 0.5, 0.0), 5)])
@pytest.mark.parametrize("ratio", [1e-5, 1e-9])
def test_other_coefficients_and_steps(P, ratio, coefficients, steps):                          # noqa: F811
    """A rounding grows as the matrix does while it is small: the steps behind the seventh at 1e-5 would be past that."""
    g = _of_norm(2, 80, 120, F32, ratio, seed=3)
    assert _err(P.prsgd_orthogonalize(g, coefficients=coefficients, steps=steps, eps=EPS),
                O.orthogonalize(g.cpu(), coefficients, steps, EPS)) <= TOL[F32]


@pytest.mark.parametrize("rows,cols", [(70, 100), (130, 90)])
def test_steps_with_small_gradients(P, rows, cols):                                            # noqa: F811
    g, m = _of_norm(3, rows, cols, F32, 1e-4, seed=5), _of_norm(3, rows, cols, F32, 1e-3, seed=6)
    x = torch.zeros(3, rows, cols, device="cuda")
    want, _ = O.muon_step(x.cpu(), g.cpu(), m.cpu(), lr=1.0, mu=0.9, nesterov=True, weight_decay=0.0, scale=1.0, eps=EPS)
    P.prsgd_muon_step(x, g, m, 1.0, momentum=0.9, scale=1.0, eps=EPS)
    assert _err(x, want) <= TOL[F32]
