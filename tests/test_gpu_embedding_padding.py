"""Padding's rows of an embedding are +0 whatever the scale's sign, and workspaces of few rows stay as they were."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_padding_is_positive_zero(P, dtype):
    table = torch.randn(2, 9, 21, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    tokens = torch.tensor([3, -1, 9, 0, 8, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    y = P.prsgd_embedding(tokens, table, scale=-2.0)
    assert not y[[1, 2, 5]].any() and not y[[1, 2, 5]].signbit().any()
    assert torch.equal(y[0], -2 * table[0, 3]) and torch.equal(y[4], -2 * table[1, 8])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 255, 256])
def test_few_rows_write_no_workspace(P, rows, dtype):
    g = torch.Generator().manual_seed(rows)
    table, tokens = torch.empty(3, 40, 19, dtype=dtype, device="cuda"), torch.randint(-1, 41, (3 * rows,), generator=g).to(torch.int32).cuda()
    dy = torch.randn(3 * rows, 19, generator=g).to(dtype).cuda()
    ws = torch.full((P.prsgd_embedding_backward_workspace_bytes(tokens, table),), 0x5A, dtype=torch.uint8, device="cuda")
    got = P.prsgd_embedding_backward(dy, tokens, table, workspace=ws)
    assert ws.numel() == 256 and bool((ws == 0x5A).all()) and torch.equal(got, P.prsgd_embedding_backward(dy, tokens, table))
