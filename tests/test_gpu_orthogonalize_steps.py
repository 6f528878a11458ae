"""Many steps on short and on rank-deficient matrices, against the definition where it determines the result.

Directions in which a matrix is zero hold rounding, which every step makes larger by a until it is as large as the others: from some
number of steps on their result is any direction, but no singular value may pass what the polynomial leaves, 1.2024 at the default
coefficients.  Tolerances before the first run: singular values of fp32 results 1.21; bf16 adds three operand roundings of 2^-12 in front
of factors of norm 2.8 at most, and the result's rounding, 2^-9 of a norm of up to 1.2 sqrt(64): 1.25.
"""
import pytest
import torch

import ops_oracle as O
from test_gpu_orthogonalize import BF16, F32, P, _err, _matrices        # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu
MOST = {F32: 1.21, BF16: 1.25}
DEFICIENT = [(60, 128, 16), (128, 60, 16), (10, 200, 9), (200, 10, 9), (32, 100, 1), (48, 300, 8), (2000, 64, 20), (5, 7, 2), (70, 100, 8)]


def _largest(out):
    assert bool(out.isfinite().all())
    return float(torch.linalg.svdvals(out.double().cpu()).max())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("steps", [12, 16, 20, 33, 64])
@pytest.mark.parametrize("rows,cols,rank", DEFICIENT)
def test_many_steps_keep_singular_values_in_their_range(P, rows, cols, rank, steps, dtype):    # noqa: F811
    g = _matrices(3, rows, cols, dtype, seed=rows + steps, rank=rank)
    assert _largest(P.prsgd_orthogonalize(g, steps=steps)) <= MOST[dtype]


@pytest.mark.parametrize("coefficients", [(2.0, -1.5, 0.5), (1.875, -1.25, 0.375), (1.5, -0.5, 0.0)])
@pytest.mark.parametrize("steps", [24, 40, 64])
@pytest.mark.parametrize("rows,cols,rank", [(60, 128, 16), (100, 32, 1), (16, 300, 8)])
def test_many_steps_of_other_coefficients(P, rows, cols, rank, steps, coefficients):            # noqa: F811
    """Singular values come from below and end at 1."""
    g = _matrices(3, rows, cols, F32, seed=rows + steps, rank=rank)
    assert _largest(P.prsgd_orthogonalize(g, coefficients=coefficients, steps=steps)) <= 1.01


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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,rank", [(128, 60, 16), (10, 200, 9), (300, 48, 8)])
def test_steps_of_replicas_stay_bounded(P, rows, cols, rank, dtype):                            # noqa: F811
    """Twenty products a step: the update of finite matrices is finite and no larger than its rate allows."""
    g, m = _matrices(3, rows, cols, dtype, seed=4, rank=rank), torch.zeros(3, rows, cols, device="cuda")
    x = torch.zeros(3, rows, cols, dtype=dtype, device="cuda")
    for _ in range(2):
        before = x.clone()
        P.prsgd_muon_step(x, g, m, 0.5, momentum=0.9, scale=2.0, steps=20)
        # bf16 parameters of size 2 at most are rounded again
        slack = 0.0 if dtype == F32 else 2.0 ** -8 * float(x.float().flatten(1).norm(dim=1).max())
        assert _largest(x.float() - before.float()) <= MOST[dtype] + slack


def test_a_recording_of_many_steps(P):                                                          # noqa: F811
    g = _matrices(4, 128, 20, F32, rank=6)
    ws = torch.empty(P.prsgd_orthogonalize_workspace_bytes(g.shape, g.dtype, steps=30), dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(g)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        P.prsgd_orthogonalize(g, out=out, steps=30, workspace=ws)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        P.prsgd_orthogonalize(g, out=out, steps=30, workspace=ws)
    for k in range(3):
        g.copy_(_matrices(4, 128, 20, F32, seed=40 + k, rank=6))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, P.prsgd_orthogonalize(g, steps=30)), k
        (g @ g.transpose(1, 2)).sum().item()
