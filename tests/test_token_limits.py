"""Sizes at the ends of the token operators' documented ranges: refused one past them, with bounded workspaces up to them (no GPU; the addresses are never read)."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 1 << 20                                                # an aligned address that is no buffer


@pytest.fixture(scope="module")
def P():
    if not os.path.exists(os.path.join(ROOT, "paper_1807_06629_amd", "libprsgd.so")):
        from paper_1807_06629_amd.build import build
        build()
    from paper_1807_06629_amd import prsgd
    return prsgd


def _xent(P, **kw):
    base = dict(dtype=P.PRSGD_F32, workers=1, rows_per_worker=3, width=8, classes=8, classes_first=0)
    base.update(kw)
    return P.prsgd_xent_config(*(base[k] for k, _ in P.prsgd_xent_config._fields_))


def _xent_bytes(P, cfg):
    return (P._lib.prsgd_linear_cross_entropy_workspace_bytes(ctypes.byref(cfg)),
            P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg)))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("first", [0, 1])
@pytest.mark.parametrize("short", [1, 2, 31, 32, 127, 255])
def test_cross_entropy_refuses_rows_that_no_tile_can_count(P, short, first, dtype):
    """Rows rounded up to a tile of 256 have to stay in 32 bits."""
    cfg = _xent(P, dtype=dtype, rows_per_worker=2 ** 31 - short, classes_first=first)
    assert _xent_bytes(P, cfg) == (0, 0) and "rows" in P.prsgd_last_error(None)
    assert P._lib.prsgd_linear_cross_entropy(ctypes.byref(cfg), A, 8, 2 * A, 64, 8, 3 * A, 4 * A, 5 * A, 6 * A, None) == P.PRSGD_EINVAL
    assert P._lib.prsgd_linear_cross_entropy_backward(ctypes.byref(cfg), A, 2 * A, 8, 3 * A, 64, 8, 4 * A, 5 * A, 6 * A, 8, 7 * A, 64, 8, 8 * A, None) == P.PRSGD_EINVAL
    most = _xent(P, dtype=dtype, rows_per_worker=2 ** 31 - 256, classes_first=first)
    assert min(_xent_bytes(P, most)) > 0


def test_rows_of_all_workers_may_be_more(P):
    assert min(_xent_bytes(P, _xent(P, workers=7, rows_per_worker=(2 ** 31 - 1) // 7))) > 0


@pytest.mark.parametrize("dtype,first,workers,rows,width,classes", [(1, 1, 8, 8192, 1024, 131072), (1, 0, 8, 8192, 1024, 131072), (0, 1, 8, 8192, 1024, 131072),
                                                                    (1, 0, 2, 4096, 2047, 32767), (0, 0, 1, 65536, 250, 50001)])
def test_statistics_of_large_launches_take_what_their_tiles_write(P, dtype, first, workers, rows, width, classes):
    """Tiles of 128 classes at least: 8 bytes a row and tile, 4 a row for the label's logit, and copies of what is not aligned."""
    cfg = _xent(P, dtype=dtype, workers=workers, rows_per_worker=rows, width=width, classes=classes, classes_first=first)
    n, eights = workers * rows, lambda k: (k + 7) // 8 * 8
    copies = 2 * (n * eights(width) + workers * eights(width) * eights(classes)) if dtype == 1 and (width % 8 or classes % 8) else 0
    assert P._lib.prsgd_linear_cross_entropy_workspace_bytes(ctypes.byref(cfg)) <= 8 * n * ((classes + 127) // 128) + 4 * n + copies + 2048


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,classes", [(1 << 20, 1), (1 << 20, 2), (1 << 20, 10), (1 << 18, 100), (1 << 16, 333)])
def test_gradients_of_few_classes_take_what_they_hold(P, rows, classes, dtype):
    """A row's classes rounded up to 64 (to 8 below that), the parts of products of few tiles (512 of 64 x 64 in fp32), a copy of W and a bit a row."""
    cfg = _xent(P, dtype=dtype, rows_per_worker=rows, width=64, classes=classes)
    each = (classes + 7) // 8 * 8 if classes < 64 else (classes + 63) // 64 * 64
    n = P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(cfg))
    assert n <= rows * each * (2 if dtype == 1 else 4) + 512 * 64 * 64 * 4 + rows // 8 + 2 * 64 * each + 4096


@pytest.mark.parametrize("dtype", [0, 1])
def test_the_embeddings_gradient_of_few_rows_needs_no_workspace(P, dtype):
    """Up to 256 rows a worker one launch does without: what every call asks for at least is all. Beyond, sorted tokens with their rows, and two fp32 rows for eight tokens."""
    def need(rows, workers=5, width=250):
        return P._lib.prsgd_embedding_backward_workspace_bytes(ctypes.byref(P.prsgd_embedding_config(dtype, workers, rows, 1000, width, 1.0)))
    assert [need(r) for r in (0, 1, 8, 255, 256)] == [256] * 5
    assert 5 * 257 * 8 < need(257) <= 5 * (257 * 8 + 33 * 2 * 256 * 4) + 3 * 256


@pytest.mark.parametrize("workers,rows,width,classes", [(8, 128, 1024, 1000), (8, 128, 2048, 1000), (64, 16, 1024, 100), (4, 64, 1024, 512)])
def test_short_contractions_of_bf16_stay_whole(P, workers, rows, width, classes):
    """No room is asked for parts that would take longer to add than they save: dz, a bit a row, and roundings to 256 bytes alone."""
    n = P._lib.prsgd_linear_cross_entropy_backward_workspace_bytes(ctypes.byref(_xent(P, dtype=1, workers=workers, rows_per_worker=rows, width=width, classes=classes)))
    assert n <= workers * rows * ((classes + 63) // 64 * 64) * 2 + workers * ((rows + 63) // 64 * 8) + 1024
