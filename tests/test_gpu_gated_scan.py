"""prsgd_gated_scan and its gradients against the recurrence in 64 bits.

Tolerances before the first run: f and 1 - f are off by at most 5 roundings (exp 2, sum 1, quotient 1, product 1), a step's products and sum by 3 more,
and a composition takes every product once more: 16 * 2^-24 of the step's terms, carried on by f as the state is (the oracle's E); outputs add their own rounding.
"""
import pytest
import torch

import token_oracle as O

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROUND = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
UNIT = 16 * 2.0 ** -24


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rand(seed, *shape, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def _near(got, want, off, dtype):
    return bool(((got.double() - want).abs() <= ROUND[dtype] * want.abs() + off * (1 + 1e-3) + 1e-37).all())


def _check(P, rows, width, dtype, sequences=1, starts=None, states=True, shift=1.0):
    v, gate = _rand(1, rows, width, dtype=dtype), (2 * _rand(2, rows, width) + shift).to(dtype)
    initial = _rand(3, sequences, width) if states else None
    kw = dict(sequences=sequences, starts=starts, initial=initial)
    h, last = P.prsgd_gated_scan(v, gate, **kw)
    want, want_last, off, far = O.gated_scan(v, gate, unit=UNIT, **kw)
    assert _near(h, want, off, dtype) and _near(last, want_last, far, F32)
    dh, dlast = _rand(4, rows, width, dtype=dtype), _rand(5, sequences, width) if states else None
    got = P.prsgd_gated_scan_backward(dh, v, gate, h, dlast=dlast, **kw)
    want, off = O.gated_scan_backward(dh, v, gate, h, dlast=dlast, unit=UNIT, **kw)
    for g, w, o, t in zip(got, want, off, (dtype, dtype, F32)):
        assert _near(g, w, o, t)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 3, 7, 8, 9, 63, 64, 65, 130])
def test_every_width(P, width, dtype):
    for sequences, length in ((1, 1), (3, 1), (2, 2), (3, 33), (1, 150)):
        _check(P, sequences * length, width, dtype, sequences)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length", [15, 16, 17, 31, 32, 34, 127, 128, 129, 255, 256, 257, 700])
def test_every_length(P, length, dtype):
    _check(P, length, 10, dtype)
    _check(P, 2 * length, 10, dtype, 2, states=False, shift=6.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cuts", [[0, 40], [3, 3, 3, 40], [0, 1, 2, 3, 40], [5, 5], [0, 0, 0], [40, 40], [2, 300, 301, 560, 599], [0, 600], [590, 600]])
def test_packed_sequences_and_empty_ones(P, cuts, dtype):
    rows = 40 if cuts[-1] <= 40 else 600
    _check(P, rows, 70, dtype, len(cuts) - 1, torch.tensor(cuts, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cuts", [(1024, None), (1100, None), (2500, None), (2200, [1, 2190]), (4400, [0, 4000, 4001, 4001, 4390])])
def test_few_long_sequences_are_cut_into_parts(P, rows, cuts, dtype):
    n = 1 if cuts is None else len(cuts) - 1
    assert P.prsgd_gated_scan_workspace_bytes(torch.empty(rows, 12, device="cuda", dtype=dtype), n) > 0
    _check(P, rows, 12, dtype, n, None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device="cuda"), shift=3.0)


def test_parts_and_any_workspace(P):
    """Bits are those of any run, whatever the workspace held."""
    v, gate, dh = (_rand(k, 3000, 40, dtype=BF16) for k in (1, 2, 3))
    h, last = P.prsgd_gated_scan(v, gate)
    back = P.prsgd_gated_scan_backward(dh, v, gate, h, dlast=last)
    n = P.prsgd_gated_scan_workspace_bytes(v, 1)
    for fill in (0, 0xFF):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        again = P.prsgd_gated_scan(v, gate, workspace=ws)
        assert torch.equal(h, again[0]) and torch.equal(last, again[1])
        assert all(torch.equal(a, b) for a, b in zip(back, P.prsgd_gated_scan_backward(dh, v, gate, h, dlast=last, workspace=ws)))
    with pytest.raises(ValueError):
        P.prsgd_gated_scan(v, gate, workspace=torch.empty(n - 8, dtype=torch.uint8, device="cuda"))


def _many_cuts(rows, sequences, seed):
    """Sequences of any length, empty ones, ones of a row and ones that end where tables of 512 rows and parts do."""
    cuts = torch.randint(7, rows - 9, (sequences - 9,), generator=torch.Generator().manual_seed(seed)).tolist()
    return torch.tensor(sorted(cuts + [7, 7, 8, 512, 513, 1024, 1024 + 7, 1024 + 7, rows - 9, rows - 9]), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("width,dtype", [(5, F32), (20, BF16), (72, F32), (72, BF16)])
def test_many_sequences_of_any_length_are_cut_too(P, width, dtype):
    rows, n = 9000, 30
    starts = _many_cuts(rows, n, width)
    assert starts.numel() == n + 1 and P.prsgd_gated_scan_workspace_bytes(torch.empty(rows, width, device="cuda", dtype=dtype), n) > 0
    _check(P, rows, width, dtype, n, starts, shift=3.0)
    _check(P, rows, width, dtype, n, starts, states=False, shift=3.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [(2600, 8136), (2100, 7001), (300, 3000), (256, 513), (513, 2002)])
def test_long_walks_of_few_workgroups(P, rows, width, dtype):
    """Wide rows of a long sequence that is not cut: workgroups have 32 channels there."""
    assert P.prsgd_gated_scan_workspace_bytes(torch.empty(rows, width, device="cuda", dtype=dtype), 1) == 0
    _check(P, rows, width, dtype, shift=3.0)


def test_parts_keep_sequences_apart_and_states_in_place(P):
    rows, n, width = 9000, 30, 20
    starts = _many_cuts(rows, n, 3)
    v, gate, initial, dlast = _rand(1, rows, width), _rand(2, rows, width) + 2, _rand(3, n, width), _rand(4, n, width)
    out = torch.full((rows, width), 9.0, device="cuda")
    h, last = P.prsgd_gated_scan(v, gate, starts=starts, initial=initial, out=out)
    assert bool((h[:7] == 9).all()) and bool((h[rows - 9:] == 9).all())
    state = initial.clone()
    again, s = P.prsgd_gated_scan(v, gate, starts=starts, initial=state, last=state)
    assert torch.equal(again[7:rows - 9], h[7:rows - 9]) and not again[:7].any() and not again[rows - 9:].any() and torch.equal(s, last)
    dh = _rand(5, rows, width)
    a = P.prsgd_gated_scan_backward(dh, v, gate, h, starts=starts, initial=initial, dlast=dlast)
    b = P.prsgd_gated_scan_backward(dh, v, gate, h, starts=starts, initial=initial, dlast=dlast, dinitial=dlast)
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and not a[0][:7].any() and not a[1][rows - 9:].any()
    # what is no number, in one channel of the longest sequence, also where it is its state
    lengths = (starts[1:] - starts[:-1]).tolist()
    k = lengths.index(max(lengths))
    first, end = int(starts[k]), int(starts[k + 1])
    v[first + 3, 4], initial[k, 6] = float("nan"), float("inf")
    bad, bad_last = P.prsgd_gated_scan(v, gate, starts=starts, initial=initial, out=out.clone())
    touched = torch.zeros_like(v, dtype=torch.bool)
    touched[first + 3:end, 4] = True
    touched[first:end, 6] = True
    assert bool(bad[touched].isfinite().logical_not().all()) and torch.equal(bad[~touched], h[~touched])
    assert torch.equal(bad_last[:k], last[:k]) and torch.equal(bad_last[k + 1:], last[k + 1:])


def test_rows_that_no_sequence_has(P):
    rows, width = 50, 20
    starts = torch.tensor([7, 20, 41], dtype=torch.int32, device="cuda")
    v, gate, dh, initial = _rand(1, rows, width), _rand(2, rows, width), _rand(3, rows, width), _rand(4, 2, width)
    v[:7], gate[41:], dh[45] = float("nan"), float("inf"), float("nan")
    h, last = P.prsgd_gated_scan(v, gate, starts=starts, initial=initial)
    assert not h[:7].any() and not h[41:].any() and bool(h.isfinite().all()) and bool(last.isfinite().all())
    out = torch.full((rows, width), 5.0, device="cuda")
    P.prsgd_gated_scan(v, gate, starts=starts, initial=initial, out=out)
    assert bool((out[:7] == 5).all()) and bool((out[41:] == 5).all()) and torch.equal(out[7:41], h[7:41])
    dv, dgate, _ = P.prsgd_gated_scan_backward(dh, v, gate, h, starts=starts, initial=initial, dgate=out)
    assert not dv[:7].any() and not dv[41:].any() and bool((dgate[:7] == 5).all()) and bool((dgate[41:] == 5).all())
    assert bool(dv.isfinite().all()) and bool(dgate.isfinite().all())


def test_starts_past_the_rows_read_and_write_nothing_else(P):
    v, gate = _rand(1, 30, 9), _rand(2, 30, 9)
    want, _ = P.prsgd_gated_scan(v, gate, starts=torch.tensor([0, 12, 30], dtype=torch.int32, device="cuda"))
    got, _ = P.prsgd_gated_scan(v, gate, starts=torch.tensor([-5, 12, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want)


def test_one_token_at_a_time_is_the_whole_sequence(P):
    """State in place; what differs is the order of the products."""
    n, length, width = 3, 40, 100
    v, gate = _rand(1, n * length, width), _rand(2, n * length, width)
    h, last = P.prsgd_gated_scan(v, gate, sequences=n)
    _, _, off, far = O.gated_scan(v, gate, n, unit=UNIT)
    state = torch.zeros(n, width, device="cuda")
    for t in range(length):
        y, s = P.prsgd_gated_scan(v[t::length], gate[t::length], sequences=n, initial=state, last=state)
        assert s.data_ptr() == state.data_ptr() and torch.equal(y, state)
        assert bool(((y - h[t::length]).abs() <= 2 * off[t::length]).all())
    assert bool(((state - last).abs() <= 2 * far).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_pieces_carry_the_state(P, dtype):
    v, gate = _rand(1, 500, 33, dtype=dtype), _rand(2, 500, 33, dtype=dtype)
    h, last = P.prsgd_gated_scan(v, gate)
    a, mid = P.prsgd_gated_scan(v[:201], gate[:201])
    b, end = P.prsgd_gated_scan(v[201:], gate[201:], initial=mid)
    want, want_last, off, far = O.gated_scan(v, gate, unit=UNIT)
    assert _near(torch.cat([a, b]), want, off, dtype) and _near(end, want_last, far, F32)


def test_strides(P):
    v, gate, dh = _rand(1, 60, 50)[:, 3:44], _rand(2, 60, 70)[:, 1:42], _rand(3, 60, 41)
    initial = _rand(4, 2, 90)[:, 7:48]
    out, last = torch.full((60, 45), 9.0, device="cuda"), torch.full((2, 50), 9.0, device="cuda")
    h, end = P.prsgd_gated_scan(v, gate, initial=initial, out=out[:, 2:43], last=last[:, 1:42])
    want, want_end = P.prsgd_gated_scan(v.contiguous(), gate.contiguous(), initial=initial.contiguous())
    assert torch.equal(h, want) and torch.equal(end, want_end) and int((out == 9).sum()) == 60 * 4 and int((last == 9).sum()) == 2 * 9
    spread = dh[:1].expand(60, 41)
    got = P.prsgd_gated_scan_backward(spread, v, gate, h, initial=initial, dlast=initial)
    for x, y in zip(got, P.prsgd_gated_scan_backward(spread.contiguous(), v.contiguous(), gate.contiguous(), want, initial=initial.contiguous(),
                                                     dlast=initial.contiguous())):
        assert torch.equal(x, y)


def test_what_is_no_number_stays_in_its_channel_of_its_sequence(P):
    n, length, width = 3, 300, 20
    v, gate = _rand(1, n * length, width), _rand(2, n * length, width)
    clean, _ = P.prsgd_gated_scan(v, gate, sequences=n)
    v[length + 70, 4] = float("nan")
    h, last = P.prsgd_gated_scan(v, gate, sequences=n)
    touched = torch.zeros_like(v, dtype=torch.bool)
    touched[length + 70:2 * length, 4] = True
    assert bool(h[touched].isnan().all()) and torch.equal(h[~touched], clean[~touched]) and bool(last[1, 4].isnan())
    dv, dgate, d0 = P.prsgd_gated_scan_backward(_rand(3, n * length, width), v, gate, h, sequences=n)
    assert bool(dv.isfinite().all()) and bool(d0.isfinite().all()) and int(dgate.isnan().sum()) == int(dgate[length + 70:2 * length, 4].isnan().sum())


def test_gates_that_are_shut_or_open(P):
    """sigmoid of +-100 and +-inf: f is 1 or 0 to fp32, and no state is lost or kept by a difference from 1."""
    v = torch.ones(4, 8, device="cuda")
    initial = torch.full((1, 8), 3.0, device="cuda")
    for size in (100.0, 1e30, float("inf")):
        assert torch.equal(P.prsgd_gated_scan(v, torch.full_like(v, size), initial=initial)[0], torch.full_like(v, 3.0))
        assert torch.equal(P.prsgd_gated_scan(v, torch.full_like(v, -size), initial=initial)[0], v)
    h, _ = P.prsgd_gated_scan(v, torch.full_like(v, 40.0))
    want = torch.arange(1, 5, device="cuda", dtype=torch.float64)[:, None] * torch.exp(torch.tensor(-40.0, dtype=torch.float64))
    assert float((h.double() / want - 1).abs().max()) < 1e-5


def test_gradients_are_the_slopes(P):
    """fp32 along a direction: a difference over 2 d is off by d^2 of the third derivative and 2^-22 / d of the values."""
    rows, width = 40, 12
    v, gate, dh = _rand(1, rows, width), _rand(2, rows, width), _rand(3, rows, width)
    initial, dlast = _rand(4, 2, width), _rand(5, 2, width)
    a, b, c = _rand(6, rows, width), _rand(7, rows, width), _rand(8, 2, width)
    h, _ = P.prsgd_gated_scan(v, gate, initial=initial)
    dv, dgate, d0 = P.prsgd_gated_scan_backward(dh, v, gate, h, initial=initial, dlast=dlast)

    def value(t):
        y, last = P.prsgd_gated_scan(v + t * a, gate + t * b, initial=initial + t * c)
        return float((y.double() * dh.double()).sum() + (last.double() * dlast.double()).sum())
    d = 2.0 ** -7
    slope = (value(d) - value(-d)) / (2 * d)
    along = float((dv.double() * a).sum() + (dgate.double() * b).sum() + (d0.double() * c).sum())
    size = float((dv.abs().double() * a.abs()).sum() + (dgate.abs().double() * b.abs()).sum() + (d0.abs().double() * c.abs()).sum())
    assert abs(slope - along) <= 1e-3 * size


def test_runs_agree_and_states_may_be_in_place(P):
    v, gate, initial = _rand(1, 600, 70, dtype=BF16), _rand(2, 600, 70, dtype=BF16), _rand(3, 2, 70)
    h, last = P.prsgd_gated_scan(v, gate, initial=initial)
    state = initial.clone()
    again, s = P.prsgd_gated_scan(v, gate, initial=state, last=state)
    assert torch.equal(h, again) and torch.equal(s, last) and s.data_ptr() == state.data_ptr()
    dh, dlast = _rand(4, 600, 70, dtype=BF16), _rand(5, 2, 70)
    a = P.prsgd_gated_scan_backward(dh, v, gate, h, initial=initial, dlast=dlast)
    b = P.prsgd_gated_scan_backward(dh, v, gate, h, initial=initial, dlast=dlast, dinitial=dlast)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_without_rows_states_pass_through(P):
    none, state = torch.empty(0, 9, device="cuda"), _rand(1, 4, 9)
    h, last = P.prsgd_gated_scan(none, none, initial=state)
    assert h.shape == (0, 9) and torch.equal(last, state)
    assert not P.prsgd_gated_scan(none, none, sequences=4)[1].any()
    assert torch.equal(P.prsgd_gated_scan_backward(none, none, none, none, dlast=state)[2], state)


def test_the_binding_refuses_other_shapes_and_types(P):
    v, s = _rand(1, 6, 8), _rand(2, 2, 8)
    starts = torch.tensor([0, 3, 6], dtype=torch.int32, device="cuda")
    for call in (lambda: P.prsgd_gated_scan(v, v[:5]), lambda: P.prsgd_gated_scan(v, v.bfloat16()), lambda: P.prsgd_gated_scan(v, v, sequences=2, starts=starts[:2]),
                 lambda: P.prsgd_gated_scan(v, v, starts=starts.long()), lambda: P.prsgd_gated_scan(v, v, sequences=3, initial=s),
                 lambda: P.prsgd_gated_scan(v, v, initial=s.bfloat16()), lambda: P.prsgd_gated_scan(v, v, initial=s[:, :7]),
                 lambda: P.prsgd_gated_scan(v.t(), v.t()), lambda: P.prsgd_gated_scan(v, v, starts=starts[:1])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: P.prsgd_gated_scan(v, v, sequences=4), lambda: P.prsgd_gated_scan(v, v, sequences=0), lambda: P.prsgd_gated_scan(v, _rand(3, 6, 8), out=v)):
        with pytest.raises(P.PrsgdError):
            call()
