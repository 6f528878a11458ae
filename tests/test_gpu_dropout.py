"""prsgd_dropout against its definition: masks equal, values to three fp32 roundings (scale, product, sum) and the result's own."""
import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rand(seed, *shape, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _check(P, x, p, seed, residual=None, **kw):
    got = P.prsgd_dropout(x, p, seed, residual=residual, **kw)
    want = O.dropout(x, p, seed, residual=residual, **kw)
    size = O.dropout(x.abs(), p, seed, residual=None if residual is None else residual.abs(), **kw)
    assert bool(((got.double() - want).abs() <= ROUND[x.dtype] * want.abs() + 4 * 2.0 ** -24 * size).all())
    if residual is None:
        assert torch.equal(got == 0, ~O.kept(*x.shape, p, seed, **kw)[0].to(x.device) | (x == 0))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 15, 64, 100, 1000, 2047, 2048, 2056, 4097])
def test_every_width(P, width, dtype):
    for rows in (1, 3, 70):
        x = _rand(1, rows, width, dtype=dtype)
        _check(P, x, 0.1, 7)
        _check(P, x, 0.5, 7, step=3, layer=2, residual=_rand(2, rows, width, dtype=dtype))


@pytest.mark.parametrize("seed,step,layer", [(0, 0, 0), (2 ** 64 - 1, 2 ** 64 - 1, 32767), (2 ** 32, 2 ** 32, 1), (2 ** 63, 5, 100)])
def test_every_word_of_the_counter(P, seed, step, layer):
    x = torch.ones(20, 50, device="cuda")
    _check(P, x, 0.25, seed, step=step, layer=layer)


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.1, 0.5, 0.9, 1.0 - 2.0 ** -16, 0.99999])
def test_every_share(P, p):
    x = _rand(1, 300, 100)
    _check(P, x, p, 3)
    if p == 0.0:
        assert torch.equal(P.prsgd_dropout(x, p, 3), x)


def test_the_step_may_lie_on_the_device(P):
    x = _rand(1, 30, 40)
    at = torch.tensor([(1 << 40) + 5], device="cuda")
    assert torch.equal(P.prsgd_dropout(x, 0.3, 9, step=at), P.prsgd_dropout(x, 0.3, 9, step=(1 << 40) + 5))
    at.fill_(-1)
    assert torch.equal(P.prsgd_dropout(x, 0.3, 9, step=at), P.prsgd_dropout(x, 0.3, 9, step=2 ** 64 - 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_strides(P, dtype):
    x, r = _rand(1, 50, 61, dtype=dtype)[:, 3:58], _rand(2, 50, 70, dtype=dtype)[:, 1:56]
    want = P.prsgd_dropout(x.contiguous(), 0.2, 5, residual=r.contiguous())
    assert torch.equal(P.prsgd_dropout(x, 0.2, 5, residual=r), want)
    a, b = x.contiguous(), r.contiguous()
    assert P.prsgd_dropout(a, 0.2, 5, residual=r.contiguous(), out=a) is not None and torch.equal(a, want)
    P.prsgd_dropout(x, 0.2, 5, residual=b, out=b)
    assert torch.equal(b, want)
    out = torch.full((50, 60), 9.0, device="cuda", dtype=dtype)
    P.prsgd_dropout(x, 0.2, 5, residual=r, out=out[:, 2:57])
    assert torch.equal(out[:, 2:57], want) and int((out == 9).sum()) == 50 * 5
    spread = x[:1].expand(50, 55)
    assert torch.equal(P.prsgd_dropout(spread, 0.2, 5), P.prsgd_dropout(spread.contiguous(), 0.2, 5))


def test_dropped_places_take_nothing(P):
    keep = O.kept(20, 30, 0.5, 1)[0].cuda()
    x = torch.full((20, 30), float("nan"), device="cuda")
    r = _rand(1, 20, 30)
    y = P.prsgd_dropout(x, 0.5, 1)
    assert bool(y[keep].isnan().all()) and not y[~keep].any()
    y = P.prsgd_dropout(x, 0.5, 1, residual=r)
    assert bool(y[keep].isnan().all()) and torch.equal(y[~keep], r[~keep])


def test_the_gradient_has_the_mask(P):
    """Linear in x: the gradient of sum(y dy) is the same call on dy."""
    x, dy = _rand(1, 40, 100), _rand(2, 40, 100)
    a = float((P.prsgd_dropout(x, 0.3, 8, step=2).double() * dy.double()).sum())
    b = float((x.double() * P.prsgd_dropout(dy, 0.3, 8, step=2).double()).sum())
    assert abs(a - b) <= 2.0 ** -22 * float((x.double() * dy.double()).abs().sum()) * 2


def test_no_rows(P):
    assert P.prsgd_dropout(torch.empty(0, 5, device="cuda"), 0.3, 1).shape == (0, 5)


def test_the_binding_refuses_other_shapes_and_types(P):
    x = _rand(1, 6, 8)
    for call in (lambda: P.prsgd_dropout(x[0], 0.1, 1), lambda: P.prsgd_dropout(x.half(), 0.1, 1), lambda: P.prsgd_dropout(x, 0.1, 1, residual=x[:5]),
                 lambda: P.prsgd_dropout(x, 0.1, 1, residual=x.bfloat16()), lambda: P.prsgd_dropout(x, 0.1, 1, step=torch.tensor([1, 2], device="cuda")),
                 lambda: P.prsgd_dropout(x, 0.1, 1, step=torch.tensor(1)), lambda: P.prsgd_dropout(x.t(), 0.1, 1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: P.prsgd_dropout(x, 1.0, 1), lambda: P.prsgd_dropout(x, 0.1, 1, layer=40000)):
        with pytest.raises(P.PrsgdError):
            call()
    with pytest.raises(OverflowError):
        P.prsgd_dropout(x, 0.1, -1)
