"""What the token operators refuse, before anything reaches a device (no GPU): the addresses are never read."""
import ctypes
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A, B, C, D, E, F, G = (k << 20 for k in range(1, 8))       # aligned addresses that are no buffers
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def P():
    if not os.path.exists(os.path.join(ROOT, "paper_1807_06629_amd", "libprsgd.so")):
        from paper_1807_06629_amd.build import build
        build()
    from paper_1807_06629_amd import prsgd
    return prsgd


def _make(kind, base, kw):
    base.update(kw)
    return kind(*(base[k] for k, _ in kind._fields_))


def _emb(P, **kw):
    return _make(P.prsgd_embedding_config, dict(dtype=0, workers=2, rows_per_worker=3, classes=7, width=50, scale=1.0), kw)


def _scan(P, **kw):
    return _make(P.prsgd_scan_config, dict(dtype=0, sequences=2, rows=6, width=50, clear=0), kw)


def _drop(P, **kw):
    return _make(P.prsgd_dropout_config, dict(dtype=0, layer=0, rows=6, width=50, p=0.1, seed=1, step=0), kw)


def _xent(P, **kw):
    return _make(P.prsgd_xent_config, dict(dtype=0, workers=2, rows_per_worker=3, width=50, classes=7, classes_first=0), kw)


def _call(P, name, cfg, args):
    rc = getattr(P._lib, name)(None if cfg is None else ctypes.byref(cfg), *args, None)
    return rc


def _vary(good, changes):
    """The argument list with one of them changed, for every (place, value)."""
    return [[v if i == at else g for i, g in enumerate(good)] for at, v in changes]


EMB = [A, B, 350, 50, C, 50]                                 # tokens, table, matrix, row, y, row
EMB_BACK = [A, B, 50, C, 350, 50, D]                         # tokens, dy, row, dtable, matrix, row, workspace
SCAN = [None, A, 50, B, 50, C, 50, D, 50, E, 50, None]       # starts, v, gate, initial, h, last, workspace
SCAN_BACK = [None, A, 50, B, 50, C, 50, D, 50, E, 50, F, 50, G, 50, 8 * A, 50, 9 * A, 50, None]
DROP = [None, A, 50, B, 50, C, 50]                           # step, x, res, y
XENT = [A, 50, B, 350, 7, C, D, E, F]                        # h, w, labels, loss, lse, workspace
XENT_BACK = [A, B, 50, C, 350, 7, D, E, F, 50, G, 350, 7, 8 * A]      # dloss, h, w, labels, lse, dh, dw, workspace


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(workers=0), dict(workers=65536), dict(rows_per_worker=-1), dict(rows_per_worker=1 << 30),
                                dict(classes=0), dict(classes=(1 << 20) + 1), dict(width=0), dict(width=32769), dict(scale=NAN), dict(scale=INF)])
def test_embedding_refuses_its_configuration(P, kw):
    cfg = _emb(P, **kw)
    assert _call(P, "prsgd_embedding", cfg, EMB) == P.PRSGD_EINVAL
    assert _call(P, "prsgd_embedding_backward", cfg, EMB_BACK) == P.PRSGD_EINVAL
    assert P._lib.prsgd_embedding_backward_workspace_bytes(ctypes.byref(cfg)) == 0
    assert "embedding" in P.prsgd_last_error(None)


def test_embedding_gradients_of_too_many_rows_are_refused(P):
    cfg = _emb(P, workers=1, rows_per_worker=(1 << 24) + 1)
    assert P._lib.prsgd_embedding_backward_workspace_bytes(ctypes.byref(cfg)) == 0
    assert _call(P, "prsgd_embedding_backward", cfg, EMB_BACK) == P.PRSGD_EINVAL


@pytest.mark.parametrize("args", _vary(EMB, [(0, None), (0, A + 2), (1, None), (1, B + 2), (2, 349), (2, -350), (2, 1 << 41), (3, 49), (3, 0), (3, 1 << 41),
                                             (4, None), (4, C + 1), (4, B), (4, A), (5, 49), (5, 0), (5, -50), (5, 1 << 41)]))
def test_embedding_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_embedding", _emb(P), args) == P.PRSGD_EINVAL


@pytest.mark.parametrize("args", _vary(EMB_BACK, [(0, None), (0, A + 1), (1, None), (1, B + 2), (2, 49), (2, -50), (3, None), (3, C + 2), (3, B), (3, A),
                                                  (4, 349), (4, 0), (5, 49), (5, 0), (6, None), (6, D + 128)]))
def test_embedding_backward_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_embedding_backward", _emb(P), args) == P.PRSGD_EINVAL


@pytest.mark.parametrize("kw", [dict(dtype=-1), dict(sequences=0), dict(sequences=(1 << 24) + 1), dict(sequences=4), dict(rows=-1), dict(rows=(1 << 30) + 2),
                                dict(width=0), dict(width=32769), dict(sequences=1 << 23, rows=1 << 23, width=32768), dict(clear=-1), dict(clear=4)])
def test_scan_refuses_its_configuration(P, kw):
    cfg = _scan(P, **kw)
    assert _call(P, "prsgd_gated_scan", cfg, SCAN) == P.PRSGD_EINVAL
    assert _call(P, "prsgd_gated_scan_backward", cfg, SCAN_BACK) == P.PRSGD_EINVAL
    assert "gated_scan" in P.prsgd_last_error(None)


@pytest.mark.parametrize("args", _vary(SCAN, [(0, A + 2), (1, None), (1, A + 1), (2, 49), (3, None), (3, B + 2), (4, 49), (5, C + 2), (6, 49), (6, -50), (7, None),
                                              (7, D + 2), (7, A), (7, B), (7, C), (7, E), (8, 0), (8, 49), (9, E + 2), (9, A), (10, 49), (10, 0)]) +
                         [[None, A, 50, B, 50, C, 50, D, 50, C, 51, None], SCAN[:11] + [F + 64]])
def test_scan_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_gated_scan", _scan(P), args) == P.PRSGD_EINVAL
    assert _call(P, "prsgd_gated_scan", _scan(P, clear=2), SCAN) == P.PRSGD_EINVAL


@pytest.mark.parametrize("args", _vary(SCAN_BACK, [(1, None), (3, None), (5, None), (7, None), (13, None), (15, None), (1, A + 2), (7, D + 1), (9, E + 2),
                                                   (13, A), (13, B), (13, D), (13, 8 * A), (15, C), (15, E), (17, E), (17, A), (17, G), (2, 49), (8, 7), (14, 0),
                                                   (16, 49), (18, 0), (12, 3)]) +
                         [[None, A, 50, B, 50, C, 50, D, 50, E, 50, F, 50, G, 50, 8 * A, 50, F, 51, None]])
def test_scan_backward_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_gated_scan_backward", _scan(P), args) == P.PRSGD_EINVAL


def test_long_sequences_need_a_workspace(P):
    """For what parts of 128 rows at least compose, up to 512 of them, and for the sequences' states."""
    cfg = _scan(P, sequences=1, rows=1 << 15)
    n = P._lib.prsgd_gated_scan_workspace_bytes(ctypes.byref(cfg))
    assert 0 < n <= 256 * 50 * 8 + 50 * 4
    assert _call(P, "prsgd_gated_scan", cfg, SCAN) == P.PRSGD_EINVAL and _call(P, "prsgd_gated_scan_backward", cfg, SCAN_BACK) == P.PRSGD_EINVAL
    assert P._lib.prsgd_gated_scan_workspace_bytes(ctypes.byref(_scan(P))) == 0
    assert P._lib.prsgd_gated_scan_workspace_bytes(ctypes.byref(_scan(P, width=0))) == 0 and "width" in P.prsgd_last_error(None)


@pytest.mark.parametrize("kw", [dict(dtype=3), dict(layer=-1), dict(layer=32768), dict(rows=-1), dict(rows=1 << 31), dict(width=0), dict(width=32769), dict(p=-0.1),
                                dict(p=NAN), dict(p=1.0), dict(p=0.999995)])
def test_dropout_refuses_its_configuration(P, kw):
    assert _call(P, "prsgd_dropout", _drop(P, **kw), DROP) == P.PRSGD_EINVAL
    assert "dropout" in P.prsgd_last_error(None)


@pytest.mark.parametrize("args", _vary(DROP, [(0, A + 4), (0, C), (1, None), (1, A + 2), (2, 49), (2, -1), (3, B + 2), (4, 7), (5, None), (5, C + 1), (6, 0), (6, 49)]) +
                         [[None, A, 50, B, 50, A, 51], [None, A, 50, B, 50, B, 51], [None, A, 0, B, 50, A, 50]])
def test_dropout_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_dropout", _drop(P), args) == P.PRSGD_EINVAL


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(workers=0), dict(workers=65536), dict(rows_per_worker=-1), dict(rows_per_worker=1 << 30), dict(width=0),
                                dict(width=32769), dict(classes=0), dict(classes=(1 << 20) + 1), dict(classes_first=2),
                                dict(workers=1, rows_per_worker=(1 << 31) - 1, classes=1 << 20), dict(workers=65535, rows_per_worker=1, classes=1 << 20, width=2048)])
def test_cross_entropy_refuses_its_configuration(P, kw):
    cfg = _xent(P, **kw)
    assert _call(P, "prsgd_linear_cross_entropy", cfg, XENT) == P.PRSGD_EINVAL
    assert _call(P, "prsgd_linear_cross_entropy_backward", cfg, XENT_BACK) == P.PRSGD_EINVAL
    assert P._lib.prsgd_linear_cross_entropy_workspace_bytes(ctypes.byref(cfg)) == 0
    assert P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg)) == 0
    assert "linear_cross_entropy" in P.prsgd_last_error(None)


@pytest.mark.parametrize("args", _vary(XENT, [(0, None), (0, A + 2), (1, 49), (2, None), (2, B + 1), (3, 349), (4, 6), (4, 0), (5, None), (5, C + 2), (6, None), (6, D + 2),
                                              (6, E), (6, A), (6, C), (7, None), (7, B), (8, None), (8, F + 64)]))
def test_cross_entropy_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_linear_cross_entropy", _xent(P), args) == P.PRSGD_EINVAL


@pytest.mark.parametrize("args", _vary(XENT_BACK, [(0, None), (0, A + 2), (1, None), (2, 3), (3, None), (4, 349), (5, 6), (6, None), (7, None), (7, E + 1), (8, None), (8, B),
                                                   (8, D), (8, G), (9, 0), (9, 49), (10, None), (10, C), (10, E), (11, 0), (11, 349), (12, 6), (13, None), (13, 8 * A + 16)]))
def test_cross_entropy_backward_refuses_its_buffers(P, args):
    assert _call(P, "prsgd_linear_cross_entropy_backward", _xent(P), args) == P.PRSGD_EINVAL


def test_classes_first_has_its_own_distances(P):
    """[7][50]: rows of 50 and matrices of 350."""
    bad = [A, 50, B, 350, 7, C, D, E, F]
    assert _call(P, "prsgd_linear_cross_entropy", _xent(P, classes_first=1), bad) == P.PRSGD_EINVAL


def test_null_configurations_are_refused(P):
    for name, args in (("prsgd_embedding", EMB), ("prsgd_embedding_backward", EMB_BACK), ("prsgd_gated_scan", SCAN), ("prsgd_gated_scan_backward", SCAN_BACK),
                       ("prsgd_dropout", DROP), ("prsgd_linear_cross_entropy", XENT), ("prsgd_linear_cross_entropy_backward", XENT_BACK)):
        assert _call(P, name, None, args) == P.PRSGD_EINVAL


def test_nothing_to_do_is_no_error(P):
    assert _call(P, "prsgd_embedding", _emb(P, rows_per_worker=0), [None, None, 0, 0, None, 0]) == P.PRSGD_OK
    assert _call(P, "prsgd_dropout", _drop(P, rows=0), [None, None, 0, None, 0, None, 0]) == P.PRSGD_OK
    assert _call(P, "prsgd_linear_cross_entropy", _xent(P, rows_per_worker=0), [None, 0, None, 0, 0, None, None, None, None]) == P.PRSGD_OK


def test_workspaces_stay_bounded(P):
    """Of the logits' gradients 256 MiB are held, or 256 classes of them; with them dh's sums, parts of products of few tiles
    (512 tiles of 64 x 64 in fp32), a bit a row, and what rounds each up to 256 bytes."""
    parts = 512 * 64 * 64 * 4
    cfg = _xent(P, dtype=1, workers=8, rows_per_worker=8192, width=64, classes=1 << 20)
    assert P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg)) <= (256 << 20) + 8 * 8192 * 64 * 4 + 8 * 8192 // 8 + parts + 4096
    cfg = _xent(P, dtype=0, workers=1, rows_per_worker=1 << 20, width=64, classes=1000)
    assert P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg)) <= (1 << 20) * (256 + 64) * 4 + (1 << 20) // 8 + parts + 4096


def test_the_binding_refuses_what_has_no_kernel(P):
    rows, ids = torch.zeros(4, 6), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: P.prsgd_embedding(ids, torch.zeros(9, 6)), lambda: P.prsgd_embedding_backward(rows, ids, torch.zeros(9, 6)),
                 lambda: P.prsgd_gated_scan(rows, rows), lambda: P.prsgd_gated_scan_backward(rows, rows, rows, rows),
                 lambda: P.prsgd_dropout(rows, 0.1, 1), lambda: P.prsgd_linear_cross_entropy(rows, torch.zeros(6, 9), ids),
                 lambda: P.prsgd_linear_cross_entropy_backward(torch.zeros(4), rows, torch.zeros(6, 9), ids, torch.zeros(4)),
                 lambda: P.prsgd_linear_cross_entropy_workspace_bytes(rows, torch.zeros(6, 9))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        P.prsgd_dropout(rows.requires_grad_(), 0.1, 1)
