"""Norms whose arrays pass the caches (non-temporal loads and stores), and more rows than one launch has workgroups.

Tolerances as in test_gpu_rms_norm.py.  Rows lie apart and off alignment; results are also taken in place.
"""
import pytest
import torch

import ops_oracle as O
from test_gpu_rms_norm import BF16, F32, P, ROUND, SUMS, _close, _weights      # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu


def _apart(n, width, dtype, seed, offset, size=1.0):
    ld = width + 3
    base = torch.empty(n * ld + 16, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = base[offset:offset + n * ld].view(n, ld)[:, 1:width + 1]
    t.copy_(torch.randn(n, width, generator=g, device="cuda").mul_(size))
    return t


# rows * width * element size * 4 > 512 MB; a row in 4, 16, 64, 256, 512 and 1024 threads
@pytest.mark.parametrize("dtype,n,width", [(BF16, 16500, 4097), (F32, 8300, 4099), (BF16, 4200000, 17), (BF16, 68000, 1000), (F32, 700000, 52),
                                           (F32, 36000, 1001), (F32, 5200, 6581), (BF16, 9000, 8191), (F32, 2100, 16383), (BF16, 4200, 16384)])
def test_rows_past_the_caches(P, dtype, n, width):                                             # noqa: F811
    assert n * width * (2 if dtype == BF16 else 4) * 4 > 512 << 20
    x, res, w = _apart(n, width, dtype, 1, 1), _apart(n, width, dtype, 2, 0, 0.5), _weights(2, width)
    y, s = _apart(n, width, dtype, 3, 3), _apart(n, width, dtype, 4, 2)
    want = O.rms_norm(x, w, res)
    P.prsgd_rms_norm(x, w, residual=res, out=y, sum_out=s)
    _close(y, want[0], dtype)
    _close(s, want[1], dtype)

    q, scales, s8 = P.prsgd_rms_norm_fp8(x, w, residual=res)
    assert torch.equal(s8, s)
    scale = want[0].abs().amax(1).clamp(min=2.0 ** -100) / 448.0
    assert float((scales.double() / scale - 1).abs().max()) <= SUMS
    off = (q.float().double() * scales.double()[:, None] - want[0]).abs()
    assert bool((off <= torch.maximum(want[0].abs() * 2.0 ** -4, 2.0 ** -10 * scales.double()[:, None]) * (1 + 1e-4)).all())
    del q, off

    dy, rstd = _apart(n, width, dtype, 5, 1, 1e-2), want[2].float()
    dx, dw = P.prsgd_rms_norm_backward(dy, s, rstd, w, dsum=res)
    grads = O.rms_norm_backward(dy, s, rstd, w, res)
    parts = O.rms_norm_backward(dy.abs(), s.abs(), rstd, w.abs())[1]
    size = (rstd.double()[:, None] * dy.double().abs() * w.double().abs().amax()).amax(1, keepdim=True) * 2 + res.double().abs().amax()
    assert bool(((dx.double() - grads[0]).abs() <= ROUND[dtype] * grads[0].abs() + SUMS * size).all())
    # a column's rows are added in runs: 2^-24 for each that a thread adds, 1024 runs at most
    assert bool(((dw.double() - grads[1]).abs() <= (SUMS + 2.0 ** -24 * (n / 2 / 512 + 64)) * parts + 1e-37).all())
    del grads, parts, size

    keep = (y.clone(), s.clone())
    P.prsgd_rms_norm(x, w, residual=res, out=x, sum_out=res)
    assert torch.equal(x, keep[0]) and torch.equal(res, keep[1])
    over, gw = P.prsgd_rms_norm_backward(dy, s, rstd, w, dsum=None, dx=dy.clone())
    again, gw2 = P.prsgd_rms_norm_backward(dy, s, rstd, w, dsum=None, dx=dy)
    assert again is dy and torch.equal(over, again) and torch.equal(gw, gw2)


def test_more_rows_than_workgroups(P):                                                         # noqa: F811
    """256 threads to a row and 2^20 workgroups at most: the first rows' workgroups take the last ones as well."""
    n, width, part = (1 << 20) + 5000, 1030, 1 << 16
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(n, width, dtype=BF16, device="cuda")
    for a in range(0, n, part):
        x[a:a + part] = torch.randn(min(part, n - a), width, generator=g, device="cuda")
    x[7] = 0
    x[(1 << 20) + 7] = 3e38                                          # squares past fp32, behind a row of zeros in the same workgroup
    w = _weights(8, width)
    y, _, rstd = P.prsgd_rms_norm(x, w)
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w)
    per = n // 8
    assert n % 8 == 0
    for a in range(0, n, part):
        rows = slice(a, min(n, a + part))
        owner = torch.arange(rows.start, rows.stop, device="cuda") // per
        v = x[rows].double()
        r = 1.0 / torch.sqrt((v * v).mean(1) + 1e-6)
        want = v * r[:, None] * w.double()[owner]
        _close(y[rows], want, BF16)
        assert float((rstd[rows].double() / r - 1).abs().max()) <= SUMS
        scale = want.abs().amax(1).clamp(min=2.0 ** -100) / 448.0
        assert float((scales[rows].double() / scale - 1).abs().max()) <= SUMS
        off = (q[rows].float().double() * scales[rows].double()[:, None] - want).abs()
        assert bool((off <= torch.maximum(want.abs() * 2.0 ** -4, 2.0 ** -10 * scales[rows].double()[:, None]) * (1 + 1e-4)).all())
