"""Short sides in every form of their launches: one launch over several chunks of the long side, slices of it with one to sixteen blocks of
a Gram matrix, and more matrices than the device holds workgroups.  Tolerances as in test_gpu_orthogonalize.py."""
import pytest
import torch

import ops_oracle as O
from test_gpu_orthogonalize import BF16, F32, P, STEP, TOL, _err, _matrices     # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu
SHAPES = [(2, 64, 1000), (4, 50, 4001), (2, 16, 1500), (2, 10, 400), (2, 60, 200), (600, 12, 700), (300, 64, 400), (3, 20, 5000), (2, 40, 3001),
          (3, 1, 9000), (513, 3, 1030)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("count,side,longer", SHAPES)
def test_short_sides_in_every_form(P, count, side, longer, tall, dtype):                       # noqa: F811
    rows, cols = (longer, side) if tall else (side, longer)
    g = _matrices(count, rows, cols, dtype, seed=side)
    want = O.orthogonalize(g.cpu())
    out = P.prsgd_orthogonalize(g)
    assert _err(out, want) <= TOL[dtype]
    again = g.clone()
    assert torch.equal(P.prsgd_orthogonalize(again, out=again), out)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tall", [False, True])
@pytest.mark.parametrize("count,side,longer", SHAPES)
def test_steps_on_short_sides_in_every_form(P, count, side, longer, tall, dtype):              # noqa: F811
    """The momentum moves on once, whichever launch reads the update first."""
    rows, cols = (longer, side) if tall else (side, longer)
    g, m = _matrices(count, rows, cols, dtype, seed=1), _matrices(count, rows, cols, F32, seed=2) * 3
    x = (_matrices(count, rows, cols, F32, seed=3) * 100).to(dtype)
    want_x, want_m = O.muon_step(x.cpu(), g.cpu(), m.cpu(), nesterov=True, **STEP)
    o = (want_x - (1 - STEP["lr"] * STEP["weight_decay"]) * x.cpu().double()).flatten(1).norm(dim=1)
    P.prsgd_muon_step(x, g, m, STEP["lr"], momentum=STEP["mu"], weight_decay=STEP["weight_decay"], scale=STEP["scale"])
    # as in test_muon_step: one rounding of mu M + G; the update's error and the roundings of x
    assert float(((m.cpu().double() - want_m).abs() / (want_m.abs() + 1e-3 * want_m.abs().max())).max()) <= 2.0 ** -23 * 1e3
    rounding = 2.0 ** (-8 if dtype == BF16 else -23) * want_x.flatten(1).norm(dim=1)
    assert bool(((x.cpu().double() - want_x).flatten(1).norm(dim=1) <= TOL[dtype] * o + rounding).all())
