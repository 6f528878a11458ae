"""Sides up to the largest.  A matrix of one entry to a row and a column, all of one size, has singular values that are all alike: the result
is the same pattern at what the polynomial makes of 1 / sqrt(side), wherever in 2^30 elements an entry lies.

Tolerances of the entries as in test_gpu_orthogonalize.py; elsewhere sums are of zeros alone.
"""
import math

import pytest
import torch

import ops_oracle as O
from test_gpu_orthogonalize import BF16, F32, P, TOL                    # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu
LARGEST = 32768


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(LARGEST, LARGEST), (LARGEST, 64), (7, LARGEST), (LARGEST, 70), (1000, LARGEST), (LARGEST, 5000)])
def test_the_largest_sides(P, rows, cols, dtype):                                              # noqa: F811
    r = min(rows, cols)
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    row = torch.randperm(rows, generator=g, device="cuda")[:r]
    col = torch.randperm(cols, generator=g, device="cuda")[:r]
    sign = torch.randint(2, (r,), generator=g, device="cuda") * 2.0 - 1.0
    x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
    x[row, col] = (0.5 * sign).to(dtype)
    out = P.prsgd_orthogonalize(x)
    a, b, c = O.NS
    s = 0.5 / (0.5 * math.sqrt(r) + 1e-7)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    got = out[row, col].double() * sign.double()
    assert float((got / s - 1.0).abs().max()) <= TOL[dtype]
    out[row, col] = 0
    assert not bool(out.any())
