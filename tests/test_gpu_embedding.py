"""prsgd_embedding and prsgd_embedding_backward against their definitions in 64 bits.

Tolerances before the first run: a lookup is one product, rounded once; in bfloat16 that product is rounded to fp32 first, where a halfway case may move by one step more than
half: compared with the same two roundings, exactly.  A sum of k rows in fp32 in any order is off by at most (k - 1) 2^-24 of the sum of sizes, its scale by 2^-24, then
the result's own rounding.
"""
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


def _tokens(seed, n, classes, kind="any"):
    g = torch.Generator().manual_seed(seed)
    t = torch.randint(-1, classes + 1, (n,), generator=g)
    if kind == "few":                                      # most tokens are one of three
        t = torch.where(torch.rand(n, generator=g) < 0.9, torch.randint(0, min(3, classes), (n,), generator=g), t)
    if kind == "one":
        t[:] = classes - 1
    if kind == "none":
        t[:] = -1
    return t.to(torch.int32).cuda()


def _check_gradient(P, dy, tokens, table, scale, **kw):
    got = P.prsgd_embedding_backward(dy, tokens, table, scale=scale, **kw)
    want = O.embedding_backward(dy, tokens, table, scale)
    size = O.embedding_backward(dy.abs(), tokens, table, abs(scale))
    most = int(torch.bincount(tokens.long().clamp(min=0)).max()) if tokens.numel() else 0
    assert got.shape == table.shape and got.dtype == table.dtype
    assert bool(((got.double() - want).abs() <= ROUND[table.dtype] * want.abs() + (most + 2) * 2.0 ** -24 * size).all())
    return got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 3, 7, 8, 9, 64, 65, 250, 512, 513, 1024, 2049])
def test_every_width(P, width, dtype):
    for workers, rows, classes in ((1, 1, 1), (3, 5, 7), (2, 100, 30)):
        table = _rand(1, workers, classes, width, dtype=dtype)
        tokens = _tokens(2, workers * rows, classes)
        y = P.prsgd_embedding(tokens, table, scale=1.7)
        real = ((tokens >= 0) & (tokens < classes))[:, None]
        at = torch.arange(workers, device="cuda").repeat_interleave(rows), tokens.long().clamp(0, classes - 1)
        assert torch.equal(y, torch.where(real, table[at].float() * torch.tensor(1.7), 0.0).to(dtype))
        _check_gradient(P, _rand(3, workers * rows, width, dtype=dtype), tokens, table, 1.7)


@pytest.mark.parametrize("kind", ["any", "few", "one", "none"])
@pytest.mark.parametrize("rows", [2, 63, 64, 65, 129, 1000, 2047, 2048, 2049, 4096, 6500])
def test_gradients_of_every_length_and_of_common_tokens(P, rows, kind):
    for workers, classes in ((1, 50), (2, 4000)):
        table = _rand(1, workers, classes, 12, dtype=BF16)
        _check_gradient(P, _rand(3, workers * rows, 12, dtype=BF16), _tokens(rows, workers * rows, classes, kind), table, 0.5)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["any", "few", "one", "none"])
@pytest.mark.parametrize("rows", [1, 5, 127, 128, 130, 255, 256, 257])
def test_gradients_of_few_rows(P, rows, kind, dtype):
    """A launch has ranges of the table's rows up to 256 rows of a worker; tables of one range, of many and of ranges of a row each."""
    for workers, classes, width in ((1, 7, 530), (3, 1000, 41), (1, 20000, 16), (600 if rows < 10 else 4, 3, 9)):
        table = _rand(1, workers, classes, width, dtype=dtype)
        _check_gradient(P, _rand(3, workers * rows, width, dtype=dtype), _tokens(rows, workers * rows, classes, kind), table, 1.5)


def test_chunks_grow_with_the_rows(P):
    """More than 256 chunks of 64 sorted tokens: chunks are larger then."""
    rows, classes = 40001, 11
    tokens = _tokens(4, rows, classes, "few")
    dy, table = _rand(5, rows, 24), _rand(6, classes, 24)
    got = P.prsgd_embedding_backward(dy, tokens, table)
    want = torch.zeros((classes, 24), dtype=torch.float64, device="cuda")
    size = want.clone()
    real = (tokens >= 0) & (tokens < classes)
    want.index_add_(0, tokens[real].long(), dy[real].double())
    size.index_add_(0, tokens[real].long(), dy[real].double().abs())
    assert bool(((got.double() - want).abs() <= 40001 * 2.0 ** -24 * size).all())


def test_largest_token_ids(P):
    classes = 1 << 20
    table = _rand(1, classes, 8, dtype=BF16)
    tokens = torch.tensor([classes - 1, 0, classes, 2 ** 31 - 1, -2 ** 31, classes - 1] + 3000 * [classes - 2], dtype=torch.int32, device="cuda")
    y = P.prsgd_embedding(tokens, table)
    assert torch.equal(y[0], table[classes - 1]) and torch.equal(y[1], table[0]) and not y[2:5].any() and torch.equal(y[7], table[classes - 2])
    dy = torch.ones(tokens.numel(), 8, device="cuda", dtype=BF16)
    d = P.prsgd_embedding_backward(dy, tokens, table)
    assert float(d[classes - 1, 0]) == 2.0 and float(d[0, 0]) == 1.0 and float(d[classes - 2, 3]) == 3008.0 and float(d.float().sum()) == 8 * 3011.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_and_a_shared_table(P, dtype):
    base = _rand(1, 3, 20, 47, dtype=dtype)
    table = base[:, 2:19, 3:44]                            # rows of 41, odd places
    rows = _rand(2, 30, 60, dtype=dtype)[:, 5:46]
    tokens = _tokens(3, 30, 17)
    out = torch.full((30, 50), 9.0, device="cuda", dtype=dtype)
    assert P.prsgd_embedding(tokens, table, out=out[:, 1:42]).data_ptr() == out[:, 1:42].data_ptr()
    assert torch.equal(out[:, 1:42], P.prsgd_embedding(tokens, table.contiguous()))
    assert bool((out[:, 0] == 9).all()) and bool((out[:, 42:] == 9).all())
    d = torch.full((3, 20, 47), 9.0, device="cuda", dtype=dtype)
    got = P.prsgd_embedding_backward(rows, tokens, table, dtable=d[:, 2:19, 3:44])
    assert torch.equal(got, P.prsgd_embedding_backward(rows.contiguous(), tokens, table.contiguous()))
    assert int((d == 9).sum()) == 3 * (20 * 47 - 17 * 41)
    shared = table[:1].expand(3, 17, 41)                   # a table that all workers read
    assert torch.equal(P.prsgd_embedding(tokens, shared), P.prsgd_embedding(tokens, table[0].contiguous()))
    spread = rows[:1].expand(30, 41)                       # one row of gradients for all
    assert torch.equal(P.prsgd_embedding_backward(spread, tokens, table), P.prsgd_embedding_backward(spread.contiguous(), tokens, table))


def test_what_is_no_number_stays_in_its_row(P):
    table = _rand(1, 2, 9, 10)
    table[0, 3] = float("nan")
    table[1, 3, 2] = float("inf")
    tokens = torch.tensor([3, -1, 4, 8, 3, -1], dtype=torch.int32, device="cuda")
    y = P.prsgd_embedding(tokens, table)
    assert bool(y[0].isnan().all()) and not y[1].any() and bool(y[2:4].isfinite().all()) and bool(y[4, 2].isinf()) and not y[5].any()
    dy = _rand(2, 6, 10)
    dy[1] = float("nan")                                   # of padding
    dy[4] = float("inf")
    d = P.prsgd_embedding_backward(dy, tokens, table)
    assert bool(d[0].isfinite().all()) and bool(d[1, 3].isinf().all()) and bool(torch.cat([d[1, :3], d[1, 4:]]).isfinite().all())


def test_without_rows_the_gradient_is_zero(P):
    table = _rand(1, 2, 9, 10)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert P.prsgd_embedding(none, table).shape == (0, 10)
    assert not P.prsgd_embedding_backward(torch.empty(0, 10, device="cuda"), none, table).any()


def test_runs_agree_bit_for_bit_and_workspaces_may_hold_anything(P):
    tokens, table, dy = _tokens(1, 10000, 300, "few"), _rand(2, 2, 300, 40), _rand(3, 10000, 40)
    first = P.prsgd_embedding_backward(dy, tokens, table)
    n = P.prsgd_embedding_backward_workspace_bytes(tokens, table)
    for fill in (0, 0xFF, 0x7F):
        ws = torch.full((n,), fill, dtype=torch.uint8, device="cuda")
        assert torch.equal(first, P.prsgd_embedding_backward(dy, tokens, table, workspace=ws))
    with pytest.raises(ValueError):
        P.prsgd_embedding_backward(dy, tokens, table, workspace=torch.empty(n - 256, dtype=torch.uint8, device="cuda"))


def test_the_binding_refuses_other_shapes_and_types(P):
    table, tokens, dy = _rand(1, 2, 9, 10), _tokens(1, 6, 9), _rand(2, 6, 10)
    for call in (lambda: P.prsgd_embedding(tokens.long(), table), lambda: P.prsgd_embedding(tokens[:5], table), lambda: P.prsgd_embedding(tokens, table.half()),
                 lambda: P.prsgd_embedding(tokens[::2], table[0]), lambda: P.prsgd_embedding(tokens, table.transpose(1, 2)), lambda: P.prsgd_embedding(tokens, table[0, 0]),
                 lambda: P.prsgd_embedding(tokens, table, out=dy.bfloat16()), lambda: P.prsgd_embedding(tokens, table, out=dy[:5]),
                 lambda: P.prsgd_embedding_backward(dy[:, :9], tokens, table), lambda: P.prsgd_embedding_backward(dy.bfloat16(), tokens, table),
                 lambda: P.prsgd_embedding_backward(dy, tokens, table, dtable=table[:1]), lambda: P.prsgd_embedding(tokens.view(2, 3), table)):
        with pytest.raises(ValueError):
            call()
