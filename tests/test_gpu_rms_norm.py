"""prsgd_rms_norm, prsgd_rms_norm_fp8 and prsgd_rms_norm_backward against their definitions in 64 bits.

Tolerances before the first run: a row's sums are at most 64 fp32 roundings deep (16 per thread, ten levels over threads, the rest
products), and what follows them six more: 2^-24 * 70 relative to the row, 5e-6; bfloat16 outputs add 2^-8 of the element.
"""
import pytest
import torch

import ops_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
SUMS = 5e-6
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8}          # half a step of 24 and of 8 significant bits


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rows(n, width, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (size * torch.randn(n, width, generator=g, device="cuda")).to(dtype)


def _weights(workers, width, seed=9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 1.0 + 0.3 * torch.randn(workers, width, generator=g, device="cuda")


def _close(got, want, dtype, slack=SUMS):
    got, want = got.double(), want.double()
    top = want.abs().amax(dim=-1, keepdim=True)
    assert got.shape == want.shape
    assert bool(((got - want).abs() <= ROUND[dtype] * want.abs() + slack * top + 1e-37).all())


WIDTHS = [1, 2, 3, 7, 8, 9, 63, 64, 65, 100, 255, 256, 257, 1000, 1001, 1024, 2047, 4096, 4097, 8191, 16383, 16384]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", WIDTHS)
def test_forward_of_every_width(P, width, dtype):
    for workers, rows in ((1, 1), (3, 5), (2, 300)):
        n = workers * rows
        x, res, w = _rows(n, width, dtype, 1), _rows(n, width, dtype, 2, 0.5), _weights(workers, width)
        y, s, rstd = P.prsgd_rms_norm(x, w, residual=res)
        want = O.rms_norm(x, w, res)
        _close(y, want[0], dtype)
        _close(s, want[1], dtype)
        assert float((rstd.double() / want[2] - 1).abs().max()) <= SUMS
        y, s, rstd = P.prsgd_rms_norm(x, w[0], eps=0.5)
        want = O.rms_norm(x, w[0], eps=0.5)
        _close(y, want[0], dtype)
        assert s is x


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", WIDTHS)
def test_eight_bits_of_every_width(P, width, dtype):
    for workers, rows in ((1, 1), (3, 5), (2, 300)):
        n = workers * rows
        x, res, w = _rows(n, width, dtype, 3), _rows(n, width, dtype, 4, 0.5), _weights(workers, width)
        q, scales, s = P.prsgd_rms_norm_fp8(x, w, residual=res)
        y, want_s, _ = O.rms_norm(x, w, res)
        _close(s, want_s, dtype)
        top = y.abs().amax(1)                                      # at width 1 a residual may cancel its row
        want = top.clamp(min=2.0 ** -100) / 448.0
        assert float((scales.double() / want - 1).abs().max()) <= SUMS
        # nearest of e4m3: half a step, 2^-4 of the value or 2^-10 below the normal numbers
        got = q.float().double() * scales.double()[:, None]
        step = torch.maximum(y.abs() * 2.0 ** -4, 2.0 ** -10 * scales.double()[:, None])
        assert bool(((got - y).abs() <= step * (1 + 1e-4)).all())
        assert torch.equal(q.float().abs().amax(1), torch.where(top > 0, 448.0, 0.0).float())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", WIDTHS)
def test_backward_of_every_width(P, width, dtype):
    for workers, rows in ((1, 1), (3, 5), (2, 301)):
        n = workers * rows
        s, w = _rows(n, width, dtype, 5), _weights(workers, width)
        dy, ds = _rows(n, width, dtype, 6, 1e-2), _rows(n, width, dtype, 7, 1e-2)
        rstd = O.rms_norm(s, w)[2].float()
        for dsum in (ds, None):
            dx, dw = P.prsgd_rms_norm_backward(dy, s, rstd, w, dsum=dsum)
            want = O.rms_norm_backward(dy, s, rstd, w, dsum)
            parts = O.rms_norm_backward(dy.abs(), s.abs(), rstd, w.abs())[1]
            # single elements of one column may cancel: against the size of what is summed
            size = (rstd.double()[:, None] * dy.double().abs() * w.double().abs().amax()).amax(1, keepdim=True) * 2 + ds.double().abs().amax()
            assert bool(((dx.double() - want[0]).abs() <= ROUND[dtype] * want[0].abs() + SUMS * size).all())
            assert bool(((dw.double() - want[1]).abs() <= SUMS * parts + 1e-37).all())
        dx, dw = P.prsgd_rms_norm_backward(dy, s, rstd, w[0], dsum=ds)
        want = O.rms_norm_backward(dy, s, rstd, w[0], ds)
        parts = O.rms_norm_backward(dy.abs(), s.abs(), rstd, w[0].abs())[1]
        assert dw.shape == (width,) and bool(((dw.double() - want[1]).abs() <= SUMS * parts + 1e-37).all())


def test_backward_is_the_slope_of_forward(P):
    """Both in fp32, along a direction: a difference over 2h is off by h^2 of the third derivative and 2^-22 / h of the values."""
    n, width = 12, 40
    x, w = _rows(n, width, F32, 1), _weights(3, width)
    dy, ds, d, dw_dir = _rows(n, width, F32, 2), _rows(n, width, F32, 3), _rows(n, width, F32, 4), _weights(3, width, 5)
    _, s, rstd = P.prsgd_rms_norm(x, w)
    dx, dw = P.prsgd_rms_norm_backward(dy, s, rstd, w, dsum=ds)
    h = 2.0 ** -8
    val = lambda x, w: float((P.prsgd_rms_norm(x, w)[0].double() * dy.double()).sum() + (x.double() * ds.double()).sum())     # noqa: E731
    slope = (val(x + h * d, w) - val(x - h * d, w)) / (2 * h)
    size = float((dy.double().abs() * 4).sum())
    assert abs(slope - float((dx.double() * d.double()).sum())) <= (h * h + 2.0 ** -22 / h) * size
    slope = (val(x, w + h * dw_dir) - val(x, w - h * dw_dir)) / (2 * h)
    assert abs(slope - float((dw.double() * dw_dir.double()).sum())) <= (h * h + 2.0 ** -22 / h) * size


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [5, 37, 200, 1030, 5000])
def test_rows_apart_off_alignment_and_in_place(P, width, dtype):
    n, ld = 14, width + 3
    def apart(seed, offset):                                       # noqa: E306
        base = torch.full((n * ld + 16,), 5.0, dtype=dtype, device="cuda")
        t = base[offset:offset + n * ld].view(n, ld)[:, 1:width + 1]
        t.copy_(_rows(n, width, dtype, seed))
        return base, t
    (_, x), (_, res), (yb, y), (sb, s) = apart(1, 1), apart(2, 0), apart(3, 3), apart(4, 2)
    wide = _weights(2, width + 2)
    w = wide[:, 1:width + 1]
    want = O.rms_norm(x, w, res)
    P.prsgd_rms_norm(x, w, residual=res, out=y, sum_out=s)
    _close(y, want[0], dtype)
    _close(s, want[1], dtype)
    for base, t in ((yb, y), (sb, s)):
        t.fill_(5.0)
        assert bool((base == 5.0).all())                           # nothing beside the rows was written
    # the sum over the residual or over x, y over x
    x0, r0 = x.clone(), res.clone()
    P.prsgd_rms_norm(x, w, residual=res, out=x, sum_out=res)
    _close(x, want[0], dtype)
    _close(res, want[1], dtype)
    x.copy_(x0)
    res.copy_(r0)
    P.prsgd_rms_norm(x, w, residual=res, out=y, sum_out=x)
    _close(x, want[1], dtype)
    rstd = want[2].float()
    dyb, dy = apart(5, 1)
    dsb, ds = apart(6, 2)
    grads = O.rms_norm_backward(dy, x, rstd, w, ds)
    dx, dw = P.prsgd_rms_norm_backward(dy, x, rstd, w, dsum=ds, dw=torch.empty(2, width + 9, device="cuda")[:, 4:width + 4])
    for over in (dy, ds):
        keep = over.clone()
        got, gw = P.prsgd_rms_norm_backward(dy, x, rstd, w, dsum=ds, dx=over)
        assert torch.equal(got, dx) and torch.equal(gw, dw)
        over.copy_(keep)
    top = float(grads[0].abs().max())
    assert bool(((dx.double() - grads[0]).abs() <= ROUND[dtype] * grads[0].abs() + SUMS * 4 * top).all())
    q = torch.empty(n, width + 3, dtype=torch.uint8, device="cuda").fill_(9)
    qv = q.view(torch.float8_e4m3fn)[:, 2:width + 2]
    P.prsgd_rms_norm_fp8(x0, w, residual=r0, out=qv)
    assert torch.equal(qv.float(), P.prsgd_rms_norm_fp8(x0, w, residual=r0)[0].float())
    assert bool((q[:, :2] == 9).all()) and bool((q[:, width + 2:] == 9).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [9, 100, 3000, 9000])
def test_rows_that_are_empty_of_numbers(P, width, dtype):
    """Zeros, NaN, infinities and the type's lowest value, beside rows that must not notice."""
    x, w = _rows(8, width, dtype, 1), _weights(2, width)
    clean = [t.clone() for t in P.prsgd_rms_norm(x, w)]
    clean8 = [t.clone() for t in P.prsgd_rms_norm_fp8(x, w)]
    x[1] = 0
    x[2, width // 2] = float("nan")
    x[5, 0] = float("inf")
    x[6] = torch.finfo(dtype).min
    y, _, rstd = P.prsgd_rms_norm(x, w)
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w)
    assert bool((y[1] == 0).all()) and float(rstd[1]) == pytest.approx(1e3) and bool((q[1].float() == 0).all()) and float(scales[1]) > 0
    assert bool(y[2].isnan().all()) and bool(q[2].float().isnan().all()) and bool(scales[2].isnan())
    assert bool(y[5, 0].isnan()) and bool((y[5, 1:] == 0).all()) and float(rstd[5]) == 0.0
    assert bool(scales[5].isnan()) and bool(q[5].float().isnan().all())
    want = O.rms_norm(x[6:7], w[1])
    _close(y[6:7], want[0], dtype)
    assert abs(float(rstd[6].double() / want[2][0] - 1)) <= SUMS
    got = q[6].float().double() * scales[6].double()
    assert bool(((got - want[0][0]).abs() <= want[0][0].abs() * 2.0 ** -4 * (1 + 1e-4) + 2.0 ** -10 * scales[6].double()).all())
    for k in (0, 3, 4, 7):
        assert torch.equal(y[k], clean[0][k]) and torch.equal(q[k].float(), clean8[0][k].float()) and scales[k] == clean8[1][k]
    zero = torch.zeros(4, width, dtype=dtype, device="cuda")
    assert bool((P.prsgd_rms_norm(zero, w, eps=1e-6)[0] == 0).all())


def test_no_rows(P):
    w = _weights(2, 30)
    x = torch.empty(0, 30, device="cuda")
    y, _, rstd = P.prsgd_rms_norm(x, w)
    assert y.shape == (0, 30) and rstd.shape == (0,)
    dw = torch.full((2, 30), 4.0, device="cuda")
    P.prsgd_rms_norm_backward(x, x, rstd, w, dw=dw)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_rows_and_many_workers(P, dtype):
    for workers, rows, width in ((1, 70001, 17), (500, 3, 130), (3, 4099, 256), (64, 128, 1024)):
        n = workers * rows
        x, w = _rows(n, width, dtype, 1), _weights(workers, width)
        dy = _rows(n, width, dtype, 2)
        y, s, rstd = P.prsgd_rms_norm(x, w)
        _close(y, O.rms_norm(x, w)[0], dtype)
        dx, dw = P.prsgd_rms_norm_backward(dy, x, rstd, w)
        want = O.rms_norm_backward(dy, x, rstd, w)
        parts = O.rms_norm_backward(dy.abs(), x.abs(), rstd, w)[1].abs()
        assert bool(((dw.double() - want[1]).abs() <= (SUMS + 2.0 ** -24 * 64) * parts).all())
        again = P.prsgd_rms_norm_backward(dy, x, rstd, w)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_offsets_beyond_32_bits(P):
    """The last rows of a buffer of 5 GB."""
    n, width = 3, 1000
    base = torch.zeros(2500 * 1000 * 1000, dtype=BF16, device="cuda")
    apart = base.as_strided((n, width), (1_200_000_000, 1))
    apart.copy_(_rows(n, width, BF16, 1))
    w = _weights(1, width)
    y, _, _ = P.prsgd_rms_norm(apart, w)
    assert torch.equal(y, P.prsgd_rms_norm(apart.contiguous(), w)[0])


def test_another_stream_and_recorded_calls(P):
    s = torch.cuda.Stream()
    x, w = _rows(24, 300, F32, 1), _weights(2, 300)
    dy = _rows(24, 300, F32, 2)
    y, rstd, dx, dw = torch.empty_like(x), torch.empty(24, device="cuda"), torch.empty_like(x), torch.empty_like(w)
    ws = torch.empty(P.prsgd_rms_norm_backward_workspace_bytes(dy, w), dtype=torch.uint8, device="cuda")

    def both():
        P.prsgd_rms_norm(x, w, out=y, rstd=rstd)
        P.prsgd_rms_norm_backward(dy, x, rstd, w, dx=dx, dw=dw, workspace=ws)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        both()
    for k in range(4):
        x.copy_(_rows(24, 300, F32, 30 + k))
        dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, rstd, dx, dw)]
        both()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, rstd, dx, dw))), k
        (x * x).sum().item()


def test_what_the_binding_refuses(P):
    x, w = _rows(6, 20, F32, 1), _weights(2, 20)
    for bad in (lambda: P.prsgd_rms_norm(x.double(), w), lambda: P.prsgd_rms_norm(x, w.double()), lambda: P.prsgd_rms_norm(x, _weights(4, 20)),
                lambda: P.prsgd_rms_norm(x, w, residual=x.to(BF16)), lambda: P.prsgd_rms_norm(x.t().contiguous().t(), w),
                lambda: P.prsgd_rms_norm(x, w, rstd=torch.empty(5, device="cuda")),
                lambda: P.prsgd_rms_norm_fp8(x, w, out=torch.empty_like(x)),
                lambda: P.prsgd_rms_norm_backward(x, x[:4], torch.empty(6, device="cuda"), w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(P.PrsgdError):
        P.prsgd_rms_norm(x, w, eps=-1.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [9, 100, 1000, 9000])
@pytest.mark.parametrize("size", [1e3, 1e18, 1e30])
def test_eight_bits_of_weights_whose_products_overflow(P, width, dtype, size):
    """s w passes fp32 where y does not: scales go by y."""
    x, w = _rows(6, width, dtype, 1, size), 1e36 * _weights(2, width)
    x[0] = 1.0                                                      # a row beside that needs nothing of it
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w)
    y = O.rms_norm(x, w)[0]
    assert float((scales.double() / (y.abs().amax(1) / 448.0) - 1).abs().max()) <= SUMS
    got = q.float().double() * scales.double()[:, None]
    step = torch.maximum(y.abs() * 2.0 ** -4, 2.0 ** -10 * scales.double()[:, None])
    assert bool(((got - y).abs() <= step * (1 + 1e-4)).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("eps", [1e-12, 1e-30])
def test_eight_bits_of_zeros_under_a_small_eps(P, dtype, eps):
    """rstd over the least scale passes fp32: zeros stay zeros."""
    x = torch.zeros(5, 200, dtype=dtype, device="cuda")
    x[3] = _rows(1, 200, dtype, 1, 1e-3)[0]
    w = _weights(1, 200)
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w, eps=eps)
    assert bool((q[[0, 1, 2, 4]].float() == 0).all()) and bool(((scales[[0, 1, 2, 4]].double() * 448 * 2.0 ** 100 - 1).abs() <= 2.0 ** -23).all())
    y = O.rms_norm(x[3:4], w, eps=eps)[0]
    got = q[3:4].float().double() * float(scales[3])
    assert bool(((got - y).abs() <= torch.maximum(y.abs() * 2.0 ** -4, torch.full_like(y, 2.0 ** -10 * float(scales[3]))) * (1 + 1e-4)).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [5, 300, 5000])
def test_result_over_the_residual_and_gradient_over_the_rows(P, width, dtype):
    x, res, w, dy = _rows(14, width, dtype, 1), _rows(14, width, dtype, 2), _weights(2, width), _rows(14, width, dtype, 3)
    y, s, rstd = P.prsgd_rms_norm(x, w, residual=res)
    over = res.clone()
    again = P.prsgd_rms_norm(x, w, residual=over, out=over)
    assert again[0] is over and torch.equal(over, y) and torch.equal(again[1], s)
    dx, dw = P.prsgd_rms_norm_backward(dy, s, rstd, w)
    over, gw = P.prsgd_rms_norm_backward(dy, s, rstd, w, dx=s)
    assert torch.equal(over, dx) and torch.equal(gw, dw) and over.data_ptr() == s.data_ptr()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [9, 100, 1000, 9000])
@pytest.mark.parametrize("size,eps", [(1e-15, 0.0), (1e-20, 1e-39), (1e-25, 0.0), (1e-35, 0.0), (1e-17, 1e-34)])
def test_rows_whose_squares_vanish(P, width, dtype, size, eps):
    x, w = _rows(6, width, dtype, 1, size), _weights(2, width)
    x[0] = 1.0
    y, _, rstd = P.prsgd_rms_norm(x, w, eps=eps)
    want = O.rms_norm(x, w, eps=eps)
    _close(y, want[0], dtype)
    assert float((rstd.double() / want[2] - 1).abs().max()) <= SUMS
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w, eps=eps)
    assert float((scales.double() / (want[0].abs().amax(1) / 448.0) - 1).abs().max()) <= SUMS


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width,size,weight,eps", [(9, 1e-21, 1e-22, 1e-27), (100, 1e-21, 1e-22, 1e-27), (1000, 1e-21, 1e-22, 1e-27),
                                                   (9000, 1e-21, 1e-22, 1e-27), (16384, 2.0 ** -51, 2.0 ** -98, 1e-40),
                                                   (16384, 2.0 ** -51, 2.0 ** -100, 1e-40)])
def test_eight_bits_of_weights_whose_products_vanish(P, width, size, weight, eps, dtype):
    """s w is below fp32's normal numbers, or nothing at all, where y is not: scales go by y."""
    x, w = _rows(6, width, dtype, 1, size), weight * _weights(2, width)
    x[0] = 1.0                                                      # rows beside that need nothing of it
    x[3] = 0.0
    q, scales, _ = P.prsgd_rms_norm_fp8(x, w, eps=eps)
    y = O.rms_norm(x, w, eps=eps)[0]
    want = y.abs().amax(1).clamp(min=2.0 ** -100) / 448.0
    assert float((scales.double() / want - 1).abs().max()) <= SUMS
    got = q.float().double() * scales.double()[:, None]
    step = torch.maximum(y.abs() * 2.0 ** -4, 2.0 ** -10 * scales.double()[:, None])
    assert bool(((got - y).abs() <= step * (1 + 1e-4)).all())
