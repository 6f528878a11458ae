"""Calls whose launches would have 2^32 threads and more, which no axis of a grid holds.

A scan's workgroups of 512 threads, 2^23 of them, and the logits' tiles of rows shorter than 16 bytes, 2^24 workgroups of 256.  Tolerances are those of the operators' own tests.
"""
import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rand(seed, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _pick(n, sequences):
    """The first, the last, those around 2^22, and some."""
    some = torch.randint(0, sequences, (n,), generator=torch.Generator().manual_seed(1)).tolist()
    return sorted({0, 1, sequences - 1, sequences - 2, (1 << 22) - 1, 1 << 22, (1 << 22) + 1} | set(some))


@pytest.mark.parametrize("packed", [False, True])
def test_scan(P, packed):
    sequences, length, width = (1 << 23) + 3, 17, 8
    rows = sequences * length + (5 if packed else 0)
    v, gate = _rand(1, rows, width, dtype=torch.bfloat16), _rand(2, rows, width, dtype=torch.bfloat16)
    starts = torch.arange(sequences + 1, dtype=torch.int32, device="cuda") * length + 2 if packed else None
    initial = _rand(3, sequences, width)
    h, last = P.prsgd_gated_scan(v, gate, sequences=sequences, starts=starts, initial=initial)
    dh, dlast = _rand(4, rows, width, dtype=torch.bfloat16), _rand(5, sequences, width)
    back = P.prsgd_gated_scan_backward(dh, v, gate, h, sequences=sequences, starts=starts, initial=initial, dlast=dlast)
    first = 2 if packed else 0
    if packed:
        for t in (h, *back[:2]):
            assert not t[:2].any() and not t[rows - 3:].any()
    at = torch.tensor(_pick(200, sequences), device="cuda")
    take = (at[:, None] * length + first + torch.arange(length, device="cuda")).flatten()
    kw = dict(sequences=at.numel(), unit=16 * U)
    want, want_last, off, far = O.gated_scan(v[take], gate[take], initial=initial[at], **kw)
    assert bool(((h[take].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.001 * off + 1e-37).all())
    assert bool(((last[at].double() - want_last).abs() <= U * want_last.abs() + 1.001 * far + 1e-37).all())
    want, off = O.gated_scan_backward(dh[take], v[take], gate[take], h[take], initial=initial[at], dlast=dlast[at], **kw)
    for got, w, o, r in zip((back[0][take], back[1][take], back[2][at]), want, off, (2.0 ** -8, 2.0 ** -8, U)):
        assert bool(((got.double() - w).abs() <= r * w.abs() + 1.001 * o + 1e-37).all())


def test_logits_of_short_rows(P):
    rows, width, classes = (1 << 17) + 33, 3, 1 << 17
    h, w = _rand(1, rows, width), _rand(2, classes, width)
    labels = torch.randint(-1, classes + 1, (rows,), generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    loss, lse = P.prsgd_linear_cross_entropy(h, w, labels, classes_first=True)
    assert bool(lse.isfinite().all()) and not loss[(labels < 0) | (labels >= classes)].any()
    at = torch.tensor(_pick(60, rows)[:-3] + [rows - 1], device="cuda").clamp(max=rows - 1).unique()
    want, want_lse, size = O.linear_cross_entropy(h[at], w, labels[at], True)
    off = (width + 2) * U * size
    lse_off = off + (classes + 8) * U + 2 * U * want_lse.abs()
    assert bool(((lse[at].double() - want_lse).abs() <= lse_off).all())
    assert bool(((loss[at].double() - want).abs() <= lse_off + off + 2 * U * want.abs()).all())
