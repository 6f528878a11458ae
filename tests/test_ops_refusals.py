"""What the operators refuse, before anything reaches a device (no GPU): the addresses are never read."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 20                                       # an aligned address that is no buffer


@pytest.fixture(scope="module")
def P():
    if not os.path.exists(os.path.join(ROOT, "paper_1807_06629_amd", "libprsgd.so")):
        from paper_1807_06629_amd.build import build
        build()
    from paper_1807_06629_amd import prsgd
    return prsgd


def _orth(P, **kw):
    base = dict(dtype=P.PRSGD_F32, count=2, rows=40, cols=50, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7)
    base.update(kw)
    return P.prsgd_orth_config(*(base[k] for k, _ in P.prsgd_orth_config._fields_))


def _norm(P, **kw):
    base = dict(dtype=P.PRSGD_F32, workers=2, rows_per_worker=3, width=50, eps=1e-6)
    base.update(kw)
    return P.prsgd_norm_config(*(base[k] for k, _ in P.prsgd_norm_config._fields_))


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(count=-1), dict(count=65536), dict(rows=0), dict(cols=0), dict(rows=32769), dict(steps=0),
    dict(steps=65), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(a=NAN), dict(b=INF),
    dict(a=5.0), dict(b=20.0), dict(c=40.0),               # singular values or the middle factor leave the range
])
def test_orthogonalize_refuses_its_configuration(P, kw):
    cfg = _orth(P, **kw)
    assert P._lib.prsgd_orthogonalize_workspace_bytes(ctypes.byref(cfg)) == 0
    assert P._lib.prsgd_orthogonalize(ctypes.byref(cfg), AT, 2000, 50, AT, 2000, 50, AT, None) == P.PRSGD_EINVAL
    assert P._lib.prsgd_muon_step(ctypes.byref(cfg), AT, 2000, 50, 2 * AT, 2000, 50, 3 * AT, 2000, 50, 0.1, 0.9, 1, 0.0, 1.0, AT,
                                  None) == P.PRSGD_EINVAL
    assert "orthogonalize" in P.prsgd_last_error(None)


@pytest.mark.parametrize("coefficients", [(3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (2.0, -1.5, 0.5), (1.875, -1.25, 0.375)])
@pytest.mark.parametrize("steps", [1, 5, 64])
def test_common_coefficients_are_taken(P, coefficients, steps):
    a, b, c = coefficients
    assert P._lib.prsgd_orthogonalize_workspace_bytes(ctypes.byref(_orth(P, a=a, b=b, c=c, steps=steps))) > 0


@pytest.mark.parametrize("args", [
    (None, 2000, 50, AT, 2000, 50, AT), (AT, 2000, 50, None, 2000, 50, AT), (AT, 2000, 50, AT, 2000, 50, None),
    (AT + 2, 2000, 50, AT, 2000, 50, AT), (AT, 2000, 50, AT + 1, 2000, 50, AT), (AT, 2000, 50, AT, 2000, 50, AT + 128),
    (AT, 2000, 49, 2 * AT, 2000, 50, AT), (AT, 1999, 50, 2 * AT, 2000, 50, AT), (AT, 2000, -50, 2 * AT, 2000, 50, AT),
    (AT, 2000, 50, 2 * AT, 2000, 49, AT), (AT, 2000, 50, 2 * AT, 2009, 51, AT), (AT, 2000, 50, AT, 2001, 50, AT),
    (AT, 1 << 41, 50, 2 * AT, 2000, 50, AT),
])
def test_orthogonalize_refuses_its_buffers(P, args):
    assert P._lib.prsgd_orthogonalize(ctypes.byref(_orth(P)), *args, None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("lr,mu,wd,scale", [(NAN, 0.9, 0.0, 1.0), (INF, 0.9, 0.0, 1.0), (0.1, 1.0, 0.0, 1.0), (0.1, -0.1, 0.0, 1.0),
                                            (0.1, NAN, 0.0, 1.0), (0.1, 0.9, NAN, 1.0), (0.1, 0.9, 0.0, INF)])
def test_muon_step_refuses_its_rates(P, lr, mu, wd, scale):
    assert P._lib.prsgd_muon_step(ctypes.byref(_orth(P)), AT, 2000, 50, 2 * AT, 2000, 50, 3 * AT, 2000, 50, lr, mu, 1, wd, scale, AT,
                                  None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("x,g,m,ws", [(None, 2, 3, 4), (1, None, 3, 4), (1, 2, None, 4), (1, 2, 3, None), (1, 1, 3, 4), (1, 2, 1, 4),
                                      (1, 2, 2, 4)])
def test_muon_step_refuses_its_buffers(P, x, g, m, ws):
    at = [None if v is None else v * AT for v in (x, g, m, ws)]
    assert P._lib.prsgd_muon_step(ctypes.byref(_orth(P)), at[0], 2000, 50, at[1], 2000, 50, at[2], 2000, 50, 0.1, 0.9, 1, 0.0, 1.0,
                                  at[3], None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("kw", [dict(dtype=-1), dict(workers=0), dict(workers=65536), dict(rows_per_worker=-1),
                                dict(rows_per_worker=1 << 30), dict(width=0), dict(width=16385), dict(eps=-1e-9), dict(eps=NAN),
                                dict(eps=INF)])
def test_norms_refuse_their_configuration(P, kw):
    cfg = _norm(P, **kw)
    row = (AT, 50, None, 0, AT, 50, None, 0, 2 * AT, 50)
    assert P._lib.prsgd_rms_norm(ctypes.byref(cfg), *row, None, None) == P.PRSGD_EINVAL
    assert P._lib.prsgd_rms_norm_fp8(ctypes.byref(cfg), *row, AT, None) == P.PRSGD_EINVAL
    assert P._lib.prsgd_rms_norm_backward_workspace_bytes(ctypes.byref(cfg)) == 0
    assert P._lib.prsgd_rms_norm_backward(ctypes.byref(cfg), AT, 50, None, 0, AT, 50, AT, AT, 50, 2 * AT, 50, AT, 50, AT,
                                          None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("args", [
    (None, 50, None, 0, AT, 50, None, 0, AT, 50), (AT, 50, None, 0, None, 50, None, 0, AT, 50), (AT, 50, None, 0, AT, 50, None, 0, None, 50),
    (AT + 2, 50, None, 0, AT, 50, None, 0, AT, 50), (AT, 50, AT + 1, 50, AT, 50, None, 0, AT, 50), (AT, 50, None, 0, AT + 2, 50, None, 0, AT, 50),
    (AT, 50, None, 0, AT, 50, AT + 2, 50, 2 * AT, 50), (AT, 49, None, 0, AT, 50, None, 0, 2 * AT, 50), (AT, 50, AT, 7, AT, 50, None, 0, 2 * AT, 50),
    (AT, 50, None, 0, AT, 49, None, 0, 2 * AT, 50), (AT, 50, None, 0, AT, 50, 3 * AT, 0, 2 * AT, 50), (AT, 50, None, 0, AT, 50, None, 0, 2 * AT, 0),
    (AT, 50, None, 0, AT, 50, AT, 51, 2 * AT, 50), (AT, 50, None, 0, AT, 50, None, 0, AT, 51), (AT, -50, None, 0, AT, 50, None, 0, 2 * AT, 50),
])
def test_norms_refuse_their_buffers(P, args):
    assert P._lib.prsgd_rms_norm(ctypes.byref(_norm(P)), *args, None, None) == P.PRSGD_EINVAL
    assert "norm" in P.prsgd_last_error(None)


def test_norm_fp8_needs_scales(P):
    assert P._lib.prsgd_rms_norm_fp8(ctypes.byref(_norm(P)), AT, 50, None, 0, AT, 50, None, 0, 2 * AT, 50, None, None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("hole", [0, 4, 6, 7, 9, 11, 13])
def test_norm_backward_refuses_null_buffers(P, hole):
    args = [AT, 50, None, 0, AT, 50, AT, AT, 50, 2 * AT, 50, AT, 50, AT]
    args[hole] = None
    assert P._lib.prsgd_rms_norm_backward(ctypes.byref(_norm(P)), *args, None) == P.PRSGD_EINVAL


def test_nothing_to_do_is_no_error(P):
    assert P._lib.prsgd_orthogonalize(ctypes.byref(_orth(P, count=0)), None, 0, 0, None, 0, 0, None, None) == P.PRSGD_OK
    assert P._lib.prsgd_orthogonalize_workspace_bytes(ctypes.byref(_orth(P, count=0))) == 0
    assert P._lib.prsgd_rms_norm(ctypes.byref(_norm(P, rows_per_worker=0)), None, 50, None, 0, AT, 50, None, 0, None, 50, None,
                                 None) == P.PRSGD_OK


def test_the_binding_refuses_what_has_no_kernel(P):
    import torch
    with pytest.raises(ValueError):
        P.prsgd_orthogonalize(torch.zeros(3, 4, dtype=torch.float64))
    with pytest.raises(ValueError):
        P.prsgd_orthogonalize(torch.zeros(3, 4))                       # no device tensor
    with pytest.raises(ValueError):
        P.prsgd_rms_norm(torch.zeros(3, 4), torch.ones(4))


@pytest.mark.parametrize("args", [
    (AT, 50, 3 * AT, 50, AT, 50, 2 * AT, 50, 2 * AT, 50), (AT, 50, 3 * AT, 50, AT, 50, None, 0, 3 * AT, 51),
    (AT, 50, 3 * AT, 0, AT, 50, None, 0, 3 * AT, 50), (AT, 50, 3 * AT, 50, AT, 50, 3 * AT, 50, 3 * AT, 50),
])
def test_norms_refuse_outputs_on_each_other_or_elsewhere_in_place(P, args):
    assert P._lib.prsgd_rms_norm(ctypes.byref(_norm(P)), *args, None, None) == P.PRSGD_EINVAL


@pytest.mark.parametrize("y", [AT, 2 * AT, 3 * AT])
def test_norm_fp8_is_not_in_place(P, y):
    assert P._lib.prsgd_rms_norm_fp8(ctypes.byref(_norm(P)), AT, 50, 2 * AT, 50, AT, 50, 3 * AT, 50, y, 50, AT, None) == P.PRSGD_EINVAL


def test_norm_backward_refuses_other_distances_in_place(P):
    for dx in (AT, 2 * AT, 3 * AT):                                    # dy, dsum and s
        args = [AT, 50, 2 * AT, 50, 3 * AT, 50, AT, AT, 50, dx, 51, AT, 50, AT]
        assert P._lib.prsgd_rms_norm_backward(ctypes.byref(_norm(P)), *args, None) == P.PRSGD_EINVAL


def test_norms_refuse_distances_whose_last_row_is_past_64_bits(P):
    """The last of 2^31 - 1 rows of 2^40 elements' distance would start at 2^71."""
    many = _norm(P, workers=1, rows_per_worker=(1 << 31) - 1)
    far, ok = 1 << 40, (AT, 50)
    for at in range(4):
        d = [far if at == k else 50 for k in range(4)]
        args = (AT, d[0], 2 * AT, d[1], AT, 50, 3 * AT, d[2], 4 * AT, d[3])
        assert P._lib.prsgd_rms_norm(ctypes.byref(many), *args, None, None) == P.PRSGD_EINVAL
        assert P._lib.prsgd_rms_norm_fp8(ctypes.byref(many), *args, AT, None) == P.PRSGD_EINVAL
        back = (AT, d[0], 2 * AT, d[1], 3 * AT, d[2], AT, *ok, 4 * AT, d[3], *ok, AT)
        assert P._lib.prsgd_rms_norm_backward(ctypes.byref(many), *back, None) == P.PRSGD_EINVAL
