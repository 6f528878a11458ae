"""What prsgd_rms_norm returns where the result takes the rows' own place."""
import pytest
import torch

import ops_oracle as O
from test_gpu_rms_norm import BF16, F32, P, _close, _rows, _weights     # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [7, 1000])
def test_no_sum_is_returned_once_the_rows_are_gone(P, width, dtype):                           # noqa: F811
    x, w, dy = _rows(6, width, dtype, 1), _weights(2, width), _rows(6, width, dtype, 2)
    want, rows = O.rms_norm(x, w), x.clone()
    y, s, rstd = P.prsgd_rms_norm(x, w, out=x)
    assert y is x and s is None
    _close(y, want[0], dtype)
    with pytest.raises(ValueError):                        # nothing to go back from
        P.prsgd_rms_norm_backward(dy, s, rstd, w)
    # another tensor on the same memory
    x.copy_(rows)
    assert P.prsgd_rms_norm(x, w, out=x.view(-1).view(6, width))[1] is None
    _close(x, want[0], dtype)
    # the rows kept elsewhere
    x.copy_(rows)
    kept = torch.empty_like(x)
    y, s, rstd = P.prsgd_rms_norm(x, w, out=x, sum_out=kept)
    assert s is kept and torch.equal(s, rows)
    grads = P.prsgd_rms_norm_backward(dy, s, rstd, w)
    again = P.prsgd_rms_norm_backward(dy, rows, rstd, w)
    assert torch.equal(grads[0], again[0]) and torch.equal(grads[1], again[1])
    # with a residual s is a tensor of its own
    x.copy_(rows)
    y, s, _ = P.prsgd_rms_norm(x, w, residual=rows, out=x)
    _close(s, O.rms_norm(rows, w, rows)[1], dtype)


def test_rows_left_alone_are_their_own_sum(P):                                                 # noqa: F811
    x, w = _rows(6, 40, F32, 1), _weights(2, 40)
    assert P.prsgd_rms_norm(x, w)[1] is x and P.prsgd_rms_norm(x, w, out=torch.empty_like(x))[1] is x
    assert P.prsgd_rms_norm_fp8(x, w)[2] is x
