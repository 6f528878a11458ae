"""bf16 matrices of full rank to the error that their products' bits leave, not only to its bound.

Limits before the first run, from a model of the products on the CPU (operands in half precision, sums exact, result rounded to bfloat16),
over three draws of each shape up to 721: result's rounding alone 1.64e-3 to 1.66e-3; sides below 200 1.79e-3 to 2.02e-3, 2.48e-3 and more
without B's diagonal in 22 bits, 3.7e-3 with the correction's sign turned; sides from 300 to 2048 1.80e-3 to 1.87e-3, 2.05e-3 and more
without, 2.55e-3 turned.
"""
import pytest

import ops_oracle as O
from test_gpu_orthogonalize import BF16, P, _err, _matrices             # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu


# tiles of 64, of 128 in four and in eight wavefronts, and of 256
@pytest.mark.parametrize("count,rows,cols,limit", [(2, 70, 80, 2.2e-3), (2, 80, 70, 2.2e-3), (20, 65, 65, 2.2e-3), (2, 100, 300, 2.2e-3),
                                                   (2, 300, 301, 1.97e-3), (4, 512, 512, 1.97e-3), (6, 1000, 500, 1.97e-3),
                                                   (10, 700, 721, 1.97e-3), (16, 700, 721, 1.97e-3), (8, 2048, 2048, 1.97e-3)])
def test_errors_of_full_rank_matrices(P, count, rows, cols, limit):                            # noqa: F811
    g = _matrices(count, rows, cols, BF16, seed=rows + cols)
    assert _err(P.prsgd_orthogonalize(g), O.orthogonalize(g)) <= limit
