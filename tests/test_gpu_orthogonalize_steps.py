"""Many steps on short sides, against the definition where it determines the result."""
import pytest
import torch

import ops_oracle as O
from test_gpu_orthogonalize import F32, P, _err, _matrices        # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu
DEFICIENT = [(60, 128, 16), (128, 60, 16), (10, 200, 9), (200, 10, 9), (32, 100, 1), (48, 300, 8), (2000, 64, 20), (5, 7, 2), (70, 100, 8)]


# what a rounding of 2^-23 grows to: the sum of a^j over the later steps, against ||O|| >= 0.68 ||X_0||
@pytest.mark.parametrize("steps", [6, 8, 10])
@pytest.mark.parametrize("rows,cols,rank", DEFICIENT)
def test_rank_deficient_matrices_while_the_result_is_determined(P, rows, cols, rank, steps):     # noqa: F811
    g = _matrices(3, rows, cols, F32, seed=rows, rank=rank)
    # every matrix off by its own rounding already: that of the product which made it
    tol = sum(O.NS[0] ** k for k in range(steps)) * 2.0 ** -23 / 0.68
    assert _err(P.prsgd_orthogonalize(g, steps=steps), O.orthogonalize(g.cpu(), steps=steps)) <= tol


SIDES = [(1, 1), (1, 7), (5, 1), (2, 2), (33, 17), (16, 500), (64, 64), (64, 4001), (4001, 64), (31, 1000), (100, 70)]


@pytest.mark.parametrize("coefficients,steps", [((1.5, -0.5, 0.0), 40), ((2.0, -1.5, 0.5), 30), ((1.875, -1.25, 0.375), 64)])
@pytest.mark.parametrize("rows,cols", SIDES)
def test_many_steps_that_converge(P, rows, cols, coefficients, steps):                         # noqa: F811
    """Singular values from 0.5 to 1 of the largest: X_0's are at least 1 / 16 and grow by 16 at most on their way to 1.  Six roundings of
    2^-22 a step (operands and sums of three products) that no later step makes smaller: 64 * 6 * 17 * 2^-22 = 1.6e-3."""
    torch.manual_seed(rows * cols)
    r = min(rows, cols)
    g = torch.empty(2, rows, cols)
    for k in range(2):
        u, v = (torch.linalg.qr(torch.randn(n, r, dtype=torch.float64))[0] for n in (rows, cols))
        g[k] = (u * torch.linspace(0.5, 1.0, r, dtype=torch.float64)) @ v.t()
    out = P.prsgd_orthogonalize(g.cuda(), coefficients=coefficients, steps=steps)
    assert _err(out, O.orthogonalize(g, coefficients, steps)) <= 1.6e-3
