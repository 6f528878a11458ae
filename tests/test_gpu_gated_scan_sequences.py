"""Numbers of sequences: those that are none are refused, whatever else says how many there are; many short ones."""
import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


@pytest.mark.parametrize("sequences", [0, -1, -2, -2 ** 31])
def test_numbers_below_one_are_refused(P, sequences):
    v, state = torch.ones(6, 8, device="cuda"), torch.ones(2, 8, device="cuda")
    starts = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    refused = (ValueError, P.PrsgdError)
    for kw in ({}, {"initial": state}, {"starts": starts}):
        with pytest.raises(refused):
            P.prsgd_gated_scan(v, v, sequences=sequences, **kw)
        with pytest.raises(refused):
            P.prsgd_gated_scan_backward(v, v, v, v, sequences=sequences, **kw)
    for kw in ({"last": state}, {"last": state, "initial": state}):
        with pytest.raises(refused):
            P.prsgd_gated_scan(v, v, sequences=sequences, **kw)
    with pytest.raises(refused):
        P.prsgd_gated_scan_backward(v, v, v, v, sequences=sequences, dlast=state)
    assert bool((state == 1).all())


def test_a_number_beyond_32_bits_is_refused(P):
    v = torch.ones(6, 8, device="cuda")
    for n in (2 ** 31, 2 ** 32 + 1, -2 ** 40):
        with pytest.raises((ValueError, P.PrsgdError)):
            P.prsgd_gated_scan(v, v, sequences=n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", [64, 61])
@pytest.mark.parametrize("length", [17, 33, 64, 65])
def test_many_short_sequences(P, length, width, dtype):
    """1024 of them, of up to 64 rows, which a wavefront each walks."""
    n, few = 1024, 16
    g = torch.Generator(device="cuda").manual_seed(length)
    v, gate, dh = (torch.randn(n * length, width, generator=g, device="cuda").to(dtype) for _ in range(3))
    initial, dlast = (torch.randn(n, width, generator=g, device="cuda") for _ in range(2))
    h, last = P.prsgd_gated_scan(v, gate, sequences=n, initial=initial)
    back = P.prsgd_gated_scan_backward(dh, v, gate, h, sequences=n, initial=initial, dlast=dlast)
    unit, step = 16 * 2.0 ** -24, 2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8
    for first in (0, 500, n - few):
        rows, at = slice(first * length, (first + few) * length), slice(first, first + few)
        kw = dict(sequences=few, initial=initial[at], unit=unit)
        want, want_last, off, far = O.gated_scan(v[rows], gate[rows], **kw)
        assert bool(((h[rows].double() - want).abs() <= step * want.abs() + 1.001 * off + 1e-37).all())
        assert bool(((last[at].double() - want_last).abs() <= 2.0 ** -24 * want_last.abs() + 1.001 * far + 1e-37).all())
        want, off = O.gated_scan_backward(dh[rows], v[rows], gate[rows], h[rows], dlast=dlast[at], **kw)
        for got, w, o, r in zip((back[0][rows], back[1][rows], back[2][at]), want, off, (step, step, 2.0 ** -24)):
            assert bool(((got.double() - w).abs() <= r * w.abs() + 1.001 * o + 1e-37).all())
