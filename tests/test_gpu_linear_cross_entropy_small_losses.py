"""Losses of likely labels far from zero: as small as they are, however large the logits.

The logits are whole numbers that products and sums hold exactly.  A loss is log of a sum of exponentials of differences from the row's maximum: `classes` terms of at most 1, each
off by at most (20 + 2) roundings of itself (differences down to -20, where it counts), one rounding a sum, and the logarithm's and the last sum's: (classes + 30) 2^-24 of what is at most
a few, whatever the logits' size.  lse itself has a rounding of that size.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("classes", [2, 5, 40, 100, 300, 3000])
def test_a_likely_label_among_large_logits(P, classes, first, dtype):
    rows, width, top = 12, 8, 128.0
    g = torch.Generator().manual_seed(classes)
    below = torch.randint(3, 21, (classes,), generator=g).double()       # how far a class lies below the label
    label = classes // 2
    below[label] = 0.0
    w = torch.zeros(classes, width, dtype=torch.float64)
    w[:, 0], w[:, 1] = top, -below
    h = torch.zeros(rows, width, dtype=torch.float64)
    h[:, 0] = torch.arange(rows, dtype=torch.float64) * 12 - 4           # logits from -512 to 16384
    h[:, 1] = 1.0
    labels = torch.full((rows,), label, dtype=torch.int32)
    labels[3] = (label + 1) % classes                                    # and an unlikely one
    z = h @ w.t()
    want_lse = torch.logsumexp(z, 1)
    want = torch.log(torch.exp(z - z.amax(1, keepdim=True)).sum(1)) + (z.amax(1) - z[torch.arange(rows), labels.long()])
    m = (w if first else w.t().contiguous()).to(dtype).cuda()
    assert torch.equal(m.double().cpu(), w if first else w.t())
    loss, lse = P.prsgd_linear_cross_entropy(h.to(dtype).cuda(), m, labels.cuda(), classes_first=first)
    assert bool(((loss.double().cpu() - want).abs() <= (classes + 30) * U + 4 * U * want).all())
    assert bool(((lse.double().cpu() - want_lse).abs() <= (classes + 30) * U + 2 * U * want_lse.abs()).all())
