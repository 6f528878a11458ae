"""prsgd_linear_cross_entropy and its gradients against their definitions in 64 bits.

Tolerances before the first run, in roundings u = 2^-24: a logit is a sum of `width` products in fp32, off by at most (width + 2) u of sum |h| |w|; lse by the largest such
error, and by (classes + 8) u for its own sum of positive terms (counted relative: u of 1) and u of itself; a loss by both.  dz = dloss (p - onehot): p is off
by the logit's error and lse's (given, so none), exp's and the product's 4 u; it is then rounded to the rows' type.  Sums over classes or rows add (their number + 2) u of the
sizes; the result is rounded once more.
"""
import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
ROUND = {F32: U, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rand(seed, *shape, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _case(workers, rows, width, classes, dtype, first, seed=1, spread=2.0):
    h = _rand(seed, workers * rows, width, dtype=dtype)
    shape = (workers, classes, width) if first else (workers, width, classes)
    w = (_rand(seed + 1, *shape) * (spread / width ** 0.5)).to(dtype)
    labels = torch.randint(-1, classes + 1, (workers * rows,), generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
    return h, w, labels


def _logit_error(size, width):
    return (width + 2) * U * size


def _check_forward(P, h, w, labels, first, **kw):
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first, **kw)
    want, want_lse, size = O.linear_cross_entropy(h, w, labels, first)
    classes = w.shape[-2] if first else w.shape[-1]
    off = _logit_error(size, h.shape[1])
    lse_off = off + (classes + 8) * U + 2 * U * want_lse.abs()
    assert bool(((lse.double() - want_lse).abs() <= lse_off).all())
    assert bool(((loss.double() - want).abs() <= lse_off + off + 2 * U * want.abs()).all())
    assert not loss[(labels < 0) | (labels >= classes)].any()
    return lse


def _check_backward(P, dloss, h, w, labels, lse, first, **kw):
    dh, dw = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first, **kw)
    assert dh.shape == h.shape and dw.shape == w.shape and dh.dtype == h.dtype and dw.dtype == h.dtype
    dtype, classes, rows = h.dtype, w.shape[-2] if first else w.shape[-1], h.shape[0] // (w.shape[0] if w.dim() == 3 else 1)
    want_h, want_w, size_h, size_w = O.linear_cross_entropy_backward(dloss, h, w, labels, lse, first)
    z = float(_logit_error(O.linear_cross_entropy(h, w, labels, first)[2], h.shape[1]).max())
    part = ROUND[dtype] + 1.1 * z + 6 * U
    assert bool(((dh.double() - want_h).abs() <= ROUND[dtype] * want_h.abs() + (part + (classes + 2) * U) * size_h + 1e-37).all())
    assert bool(((dw.double() - want_w).abs() <= ROUND[dtype] * want_w.abs() + (part + (rows + 2) * U) * size_w + 1e-37).all())
    return dh, dw


def _check(P, workers, rows, width, classes, dtype, first, **kw):
    h, w, labels = _case(workers, rows, width, classes, dtype, first, **kw)
    lse = _check_forward(P, h, w, labels, first)
    return _check_backward(P, _rand(9, workers * rows), h, w, labels, lse, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 2, 7, 8, 31, 32, 33, 64, 65, 128, 250, 256])
def test_every_width(P, width, dtype, first):
    for workers, rows, classes in ((1, 1, 5), (3, 9, 40), (2, 130, 136)):
        _check(P, workers, rows, width, classes, dtype, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("classes", [1, 2, 10, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 1001, 2500])
def test_every_number_of_classes(P, classes, dtype, first):
    _check(P, 2, 17, 72, classes, dtype, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 2, 15, 16, 31, 33, 64, 100, 127, 128, 129, 255, 257, 300])
def test_every_number_of_rows(P, rows, dtype, first):
    _check(P, 2, rows, 64, 200, dtype, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_whole_tiles(P, dtype, first):
    _check(P, 2, 256, 512, 1024, dtype, first)
    _check(P, 1, 520, 1024, 776, dtype, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("workers,rows,width,classes", [(33, 256, 512, 1024), (40, 250, 520, 1000), (40, 300, 264, 1004), (3, 2000, 1032, 1928), (130, 70, 200, 136)])
def test_tiles_of_every_size(P, workers, rows, width, classes, first):
    """Enough tiles for the larger ones, whole and ragged; rows without a label in every tile, in whole tiles, and nowhere."""
    h, w, labels = _case(workers, rows, width, classes, BF16, first)
    by_worker = labels.view(workers, rows)
    by_worker[0] = by_worker[0].clamp(0, classes - 1)
    by_worker[1, rows // 2:] = -1
    by_worker[2, :rows // 2] = -1
    h.view(workers, rows, width)[1, rows // 2:] = float("nan")
    lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)[1]
    clean = h.clone()
    clean.view(workers, rows, width)[1, rows // 2:] = 0.0
    _check_forward(P, clean, w, labels, first)
    got = P.prsgd_linear_cross_entropy_backward(_rand(9, workers * rows), h, w, labels, lse, classes_first=first)
    want = _check_backward(P, _rand(9, workers * rows), clean, w, labels, torch.where(lse.isnan(), 0.0, lse), first)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_several_pieces_of_the_classes(P, dtype, first):
    """256 MiB of dz are less than these classes take."""
    rows, classes, width = 80000, 2000, 24
    h, w, labels = _case(1, rows, width, classes, dtype, first)
    assert P.prsgd_linear_cross_entropy_backward_workspace_bytes(h, w, first) < rows * classes * h.element_size()
    lse = _check_forward(P, h, w, labels, first)
    _check_backward(P, _rand(9, rows), h, w, labels, lse, first)


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("workers,rows,width,classes", [(2, 191, 33, 1001), (2, 192, 33, 1001), (3, 300, 250, 129), (2, 200, 264, 7), (1, 230, 1023, 515), (600, 192, 1001, 515)])
def test_rows_of_no_whole_eights(P, workers, rows, width, classes, first):
    """bf16 that is copied for its products; the last case in several pieces of the classes, forward too."""
    _check(P, workers, rows, width, classes, BF16, first)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("rows,width,classes", [(2, 18, 15255), (1, 3, 9001), (3330, 9, 30), (700, 5, 3), (33, 4001, 2), (4100, 20, 33), (20, 51, 9000)])
def test_few_tiles_and_long_sums(P, rows, width, classes, dtype, first):
    _check(P, 1, rows, width, classes, dtype, first)
    _check(P, 3, rows, width, classes, dtype, first)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
def test_strides_that_are_multiples_of_nothing(P, dtype, first):
    workers, rows, width, classes = 2, 40, 48, 72
    h, w, labels = _case(workers, rows, width, classes, dtype, first)
    r, c = w.shape[1:]
    apart_h = torch.full((workers * rows, width + 5), 7.0, device="cuda", dtype=dtype)
    apart_w = torch.full((workers, r + 3, c + 9), 7.0, device="cuda", dtype=dtype)
    apart_h[:, 3:3 + width], apart_w[:, 1:1 + r, 5:5 + c] = h, w
    hv, wv = apart_h[:, 3:3 + width], apart_w[:, 1:1 + r, 5:5 + c]
    lse = _check_forward(P, hv, wv, labels, first)
    dh, dw = torch.full_like(apart_h, 9.0), torch.full_like(apart_w, 9.0)
    dloss = _rand(9, workers * rows)
    _check_backward(P, dloss, hv, wv, labels, lse, first, dh=dh[:, 3:3 + width], dw=dw[:, 1:1 + r, 5:5 + c])
    assert int((dh == 9).sum()) == dh.numel() - h.numel() and int((dw == 9).sum()) == dw.numel() - w.numel()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
def test_a_shared_matrix_and_repeated_rows(P, dtype, first):
    h, w, labels = _case(3, 10, 40, 50, dtype, first)
    shared = w[:1].expand(3, *w.shape[1:])
    lse = _check_forward(P, h, shared, labels, first)
    dw = torch.empty_like(w)
    _check_backward(P, _rand(9, 30), h, shared, labels, lse, first, dw=dw)
    spread = h[:1].expand(30, 40)
    lse = _check_forward(P, spread, w, labels, first)
    _check_backward(P, _rand(9, 30), spread, w, labels, lse, first, dh=torch.empty_like(h))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
def test_padding_holds_anything(P, dtype, first):
    h, w, labels = _case(2, 70, 64, 96, dtype, first)
    labels[60:70], labels[135:] = -1, -100
    lse = _check_forward(P, h, w, labels, first)
    dloss = _rand(9, 140)
    want = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first)
    none = (labels < 0) | (labels >= 96)
    h[none], lse[none], dloss[none] = float("nan"), float("inf"), float("nan")
    got = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[0][none].any()
    loss, _ = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)
    assert not loss[none].any()


def test_no_row_has_a_label(P):
    h, w, labels = _case(2, 5, 16, 24, F32, False)
    labels[:] = -1
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels)
    dh, dw = P.prsgd_linear_cross_entropy_backward(torch.ones(10, device="cuda"), h, w, labels, lse)
    assert not loss.any() and not dh.any() and not dw.any() and bool(lse.isfinite().all())


def test_logits_far_from_zero(P):
    """exp of logits of +-200 overflows without the row's maximum; a class far below the others adds nothing."""
    h = torch.ones(3, 8, device="cuda")
    w = torch.zeros(8, 300, device="cuda")
    w[0] = 200.0
    w[0, 7], w[0, 150], w[0, 299] = 230.0, -200.0, 229.0
    labels = torch.tensor([7, 150, 299], dtype=torch.int32, device="cuda")
    lse = _check_forward(P, h, w, labels, False)
    _check_backward(P, torch.ones(3, device="cuda"), h, w, labels, lse, False)
    lse = _check_forward(P, h, -w, labels, False)
    _check_backward(P, torch.ones(3, device="cuda"), h, -w, labels, lse, False)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_classes_of_minus_infinity_take_no_part(P, dtype):
    h, w, labels = _case(1, 6, 16, 200, dtype, True)
    w = w[0]
    h[:, 0], w[:, 0] = 1.0, 0.0
    w[40:190, 0] = float("-inf")
    w[40:190, 1:] = 0.0
    labels[:] = torch.tensor([0, 39, 190, 199, 3, -1])
    keep = torch.cat([torch.arange(40), torch.arange(190, 200)]).cuda()
    small = torch.tensor([0, 39, 40, 49, 3, -1], dtype=torch.int32, device="cuda")
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=True)
    want, want_lse = P.prsgd_linear_cross_entropy(h, w[keep].contiguous(), small, classes_first=True)
    assert bool(((lse - want_lse).abs() <= 400 * U).all()) and bool(((loss - want).abs() <= 400 * U).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
def test_what_is_no_number_stays_in_its_row_and_its_worker(P, dtype, first):
    h, w, labels = _case(3, 20, 40, 150, dtype, first)
    labels.clamp_(0, 149)
    clean_loss, clean_lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)
    dloss = _rand(9, 60)
    want = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, clean_lse, classes_first=first)
    h[25, 3] = float("nan")
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)
    others = torch.arange(60, device="cuda") != 25
    assert bool(loss[25].isnan()) and bool(lse[25].isnan()) and torch.equal(loss[others], clean_loss[others]) and torch.equal(lse[others], clean_lse[others])
    dh, dw = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first)
    assert bool(dh[25].isnan().all()) and torch.equal(dh[others], want[0][others]) and torch.equal(dw[[0, 2]], want[1][[0, 2]]) and bool(dw[1].isnan().all())


@pytest.mark.parametrize("first", [False, True])
def test_gradients_are_the_slopes(P, first):
    """fp32 along a direction: a difference over 2 d is off by d^2 of the third derivative and 2^-22 / d of the values."""
    h, w, labels = _case(2, 12, 24, 30, F32, first)
    dloss, a, b = _rand(9, 24), _rand(10, *h.shape), _rand(11, *w.shape) / 24 ** 0.5
    _, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)
    dh, dw = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first)
    d = 2.0 ** -7
    value = lambda t: float((P.prsgd_linear_cross_entropy(h + t * a, w + t * b, labels, classes_first=first)[0].double() * dloss.double()).sum())    # noqa: E731
    along = float((dh.double() * a).sum() + (dw.double() * b).sum())
    size = float((dh.abs().double() * a.abs()).sum() + (dw.abs().double() * b.abs()).sum())
    assert abs((value(d) - value(-d)) / (2 * d) - along) <= 2e-3 * size


def test_without_rows_the_gradient_is_zero(P):
    w, none = _rand(1, 2, 20, 30), torch.empty(0, dtype=torch.int32, device="cuda")
    h, f = torch.empty(0, 20, device="cuda"), torch.empty(0, device="cuda")
    loss, lse = P.prsgd_linear_cross_entropy(h, w, none)
    assert loss.shape == (0,) and lse.shape == (0,)
    dh, dw = P.prsgd_linear_cross_entropy_backward(f, h, w, none, lse)
    assert dh.shape == (0, 20) and dw.shape == w.shape and not dw.any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("first", [False, True])
def test_runs_agree_bit_for_bit_and_workspaces_may_hold_anything(P, dtype, first):
    h, w, labels = _case(2, 90, 100, 400, dtype, first)
    dloss = _rand(9, 180)
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first)
    dh, dw = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first)
    for fill in (0, 0xFF, 0x7F):
        ws = torch.full((P.prsgd_linear_cross_entropy_workspace_bytes(h, w, first),), fill, dtype=torch.uint8, device="cuda")
        again = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=first, workspace=ws)
        assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
        ws = torch.full((P.prsgd_linear_cross_entropy_backward_workspace_bytes(h, w, first),), fill, dtype=torch.uint8, device="cuda")
        again = P.prsgd_linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=first, workspace=ws)
        assert torch.equal(again[0], dh) and torch.equal(again[1], dw)


def test_the_binding_refuses_other_shapes_and_types(P):
    h, w, labels = _case(2, 4, 16, 24, F32, False)
    lse, d = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    for call in (lambda: P.prsgd_linear_cross_entropy(h, w, labels, classes_first=True), lambda: P.prsgd_linear_cross_entropy(h, w.bfloat16(), labels),
                 lambda: P.prsgd_linear_cross_entropy(h, w, labels.long()), lambda: P.prsgd_linear_cross_entropy(h, w, labels[:7]),
                 lambda: P.prsgd_linear_cross_entropy(h[:7], w, labels[:7]), lambda: P.prsgd_linear_cross_entropy(h, w.transpose(1, 2), labels),
                 lambda: P.prsgd_linear_cross_entropy(h, w, labels, loss=lse[:7]), lambda: P.prsgd_linear_cross_entropy(h.half(), w.half(), labels),
                 lambda: P.prsgd_linear_cross_entropy_backward(d[:7], h, w, labels, lse), lambda: P.prsgd_linear_cross_entropy_backward(d, h, w, labels, None),
                 lambda: P.prsgd_linear_cross_entropy_backward(d, h, w, labels, lse, dw=w[0]), lambda: P.prsgd_linear_cross_entropy_backward(d, h, w, labels, lse, dh=h[:, :8])):
        with pytest.raises(ValueError):
            call()
