"""Numbers of sequences that are none: refused, whatever else says how many there are."""
import pytest
import torch

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
