"""Rows and matrices that lie far from the first ones, past 2^32 bytes and (bfloat16) elements, and the most rows that an embedding's gradient takes."""
import pytest
import torch

import token_oracle as O
from test_gpu_linear_cross_entropy import _case, _check_backward, _check_forward

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
ROWS = 44


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


@pytest.fixture(scope="module")
def room():
    """Bytes for 44 rows that lie 2^28 and some apart."""
    yield torch.empty(ROWS * ((1 << 28) + 4096), dtype=torch.uint8, device="cuda")
    torch.cuda.empty_cache()


def _rand(seed, *shape, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


class Far:
    """Places in the room for rows far apart, one set behind another."""

    def __init__(self, room, dtype):
        self.room, self.at, self.far = room.view(dtype), 0, ((1 << 28) + 4096) // dtype.itemsize

    def like(self, t):
        """A copy of rows [n][width] or matrices [n][rows][cols], the first axis far apart."""
        inner = t[0].numel()
        v = self.room.as_strided(t.shape, (self.far, *(t.stride()[1:])), self.at)
        self.at += inner + 3
        v.copy_(t)
        return v


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_and_dropout(P, room, dtype):
    f = Far(room, dtype)
    assert f.far * (ROWS - 1) * dtype.itemsize > 1 << 33
    v, gate, dh = (_rand(k, ROWS, 45, dtype=dtype) for k in (1, 2, 3))
    far = [f.like(t) for t in (v, gate, dh)]
    out = [f.like(torch.zeros_like(v)) for _ in range(4)]
    h, last = P.prsgd_gated_scan(v, gate, sequences=2)
    got, got_last = P.prsgd_gated_scan(far[0], far[1], sequences=2, out=out[0])
    assert torch.equal(got, h) and torch.equal(got_last, last)
    want = P.prsgd_gated_scan_backward(dh, v, gate, h, sequences=2)
    back = P.prsgd_gated_scan_backward(far[2], far[0], far[1], got, sequences=2, dv=out[1], dgate=out[2])
    assert all(torch.equal(a, b) for a, b in zip(back, want))
    assert torch.equal(P.prsgd_dropout(far[0], 0.3, 5, residual=far[1], out=out[3]), P.prsgd_dropout(v, 0.3, 5, residual=gate))
    one = P.prsgd_gated_scan(v, gate, sequences=ROWS)[0]
    assert torch.equal(P.prsgd_gated_scan(far[0], far[1], sequences=ROWS, out=out[0])[0], one)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows", [ROWS // 4, ROWS])
def test_embedding(P, room, rows, dtype):
    """Rows of y and dy far apart, rows of the table, and tables."""
    f = Far(room, dtype)
    tokens = torch.tensor([(7 * k) % 41 - 1 for k in range(rows)], dtype=torch.int32, device="cuda")
    table, dy = _rand(1, 40, 37, dtype=dtype), _rand(2, rows, 37, dtype=dtype)
    y = P.prsgd_embedding(tokens, table, 1.5)
    assert torch.equal(P.prsgd_embedding(tokens, f.like(table), 1.5, out=f.like(torch.zeros_like(y))), y)
    want = P.prsgd_embedding_backward(dy, tokens, table, 1.5)
    assert torch.equal(P.prsgd_embedding_backward(f.like(dy), tokens, table, 1.5, dtable=f.like(torch.ones_like(table))), want)
    tables = _rand(3, rows, 5, 9, dtype=dtype)              # of a worker a row
    some = tokens.remainder(6)
    assert torch.equal(P.prsgd_embedding(some, f.like(tables)), P.prsgd_embedding(some, tables))
    d = dy[:, :9].contiguous()
    assert torch.equal(P.prsgd_embedding_backward(d, some, tables, dtable=f.like(torch.ones_like(tables))), P.prsgd_embedding_backward(d, some, tables))


@pytest.mark.parametrize("first", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_cross_entropy(P, room, dtype, first):
    """Rows of h and dh, rows of one worker's matrices, then the workers' matrices far apart."""
    f = Far(room, dtype)
    h, w, labels = _case(1, ROWS, 40, 37, dtype, first)
    dloss = _rand(9, ROWS)
    far_h, far_w = f.like(h), f.like(w[0])
    lse = _check_forward(P, far_h, far_w, labels, first)
    _check_backward(P, dloss, far_h, far_w, labels, lse, first, dh=f.like(torch.zeros_like(h)), dw=f.like(torch.zeros_like(w[0])))
    h, w, labels = _case(ROWS, 3, 24, 50, dtype, first)
    far_w = f.like(w)
    lse = _check_forward(P, h, far_w, labels, first)
    _check_backward(P, _rand(9, 3 * ROWS), h, far_w, labels, lse, first, dw=f.like(torch.zeros_like(w)))


def test_the_most_rows_of_an_embeddings_gradient(P):
    """2^24 rows of a worker: 8192 sorted tiles, chunks of 65536 rows.  Sums of k rows in fp32 are off by (k + 2) 2^-24 of the sum of sizes."""
    rows, classes, width = 1 << 24, 1000, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    tokens = (torch.rand(rows, generator=g, device="cuda") ** 4 * 1002 - 1).floor().to(torch.int32)
    dy, table = torch.randn(rows, width, generator=g, device="cuda"), torch.empty(classes, width, device="cuda")
    got = P.prsgd_embedding_backward(dy, tokens, table)
    real = (tokens >= 0) & (tokens < classes)
    at, order = tokens[real].long().sort()
    ends = torch.bincount(at, minlength=classes).cumsum(0)
    count = torch.diff(ends, prepend=ends.new_zeros(1)).double()[:, None]

    def sums(x):                                            # differences of running sums in 64 bits, whose own roundings are 2^-29 of an fp32 one of all that came before
        running = torch.cat([torch.zeros(1, width, dtype=torch.float64, device="cuda"), x[real][order].double().cumsum(0)])
        return torch.diff(running[ends], dim=0, prepend=running[:1])
    want, size = sums(dy), sums(dy.abs())
    assert bool(((got.double() - want).abs() <= 2.0 ** -24 * (want.abs() + (count + 2) * size)).all())
    # of whole numbers exactly: each row once, none of another token's
    ones = torch.ones(rows, 1, device="cuda")
    counted = P.prsgd_embedding_backward(ones, tokens, torch.empty(classes, 1, device="cuda"))
    assert torch.equal(counted.double(), count)
