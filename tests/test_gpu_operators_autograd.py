"""The operators and autograd: nothing is recorded, so tensors that require grad are refused while it records, and what is written in
place is seen by its check of saved tensors."""
import pytest
import torch

from test_gpu_rms_norm import F32, P, _rows, _weights                   # noqa: F401  (P: fixture)

pytestmark = pytest.mark.gpu


def _norm_operands():
    return {"x": _rows(6, 20, F32, 1), "residual": _rows(6, 20, F32, 2), "w": _weights(2, 20)}


def _back_operands():
    return {"dy": _rows(6, 20, F32, 3), "s": _rows(6, 20, F32, 1), "rstd": torch.ones(6, device="cuda"), "w": _weights(2, 20),
            "dsum": _rows(6, 20, F32, 4)}


def _matrices_of(*names):
    return {n: torch.randn(2, 70, 80, device="cuda") for n in names}


CASES = {
    "norm": (_norm_operands, lambda P, o: P.prsgd_rms_norm(**o)),
    "norm_fp8": (_norm_operands, lambda P, o: P.prsgd_rms_norm_fp8(**o)),
    "backward": (_back_operands, lambda P, o: P.prsgd_rms_norm_backward(**o)),
    "orthogonalize": (lambda: _matrices_of("g"), lambda P, o: P.prsgd_orthogonalize(**o)),
    "muon": (lambda: _matrices_of("x", "g", "m"), lambda P, o: P.prsgd_muon_step(lr=0.1, **o)),
}


@pytest.mark.parametrize("case", sorted(CASES))
def test_what_requires_grad_is_refused_while_autograd_records(P, case):                        # noqa: F811
    make, call = CASES[case]
    for name in make():
        o = make()
        o[name].requires_grad_()
        before = {k: v.detach().clone() for k, v in o.items()}
        with pytest.raises(ValueError, match="grad"):
            call(P, o)
        assert all(torch.equal(o[k].detach(), before[k]) for k in o)
        with pytest.raises(ValueError, match="grad"):      # ... and what was computed from it
            call(P, {k: v * 1.0 for k, v in o.items()})
        with torch.no_grad():
            call(P, o)
        with torch.inference_mode():
            call(P, make())


def test_shapes_alone_are_no_operands(P):                                                      # noqa: F811
    x, w = _rows(6, 20, F32, 1).requires_grad_(), _weights(2, 20).requires_grad_()
    assert P.prsgd_rms_norm_backward_workspace_bytes(x, w) > 0


def test_what_is_written_in_place_counts_as_changed(P):                                        # noqa: F811
    x, w, dy = _rows(6, 20, F32, 1), _weights(2, 20), _rows(6, 20, F32, 2)
    y, s, rstd, q = torch.empty_like(x), torch.empty_like(x), torch.empty(6, device="cuda"), torch.empty(6, 20, dtype=torch.float8_e4m3fn, device="cuda")
    dx, dw, scales = torch.empty_like(x), torch.empty_like(w), torch.empty(6, device="cuda")
    ws = torch.empty(P.prsgd_rms_norm_backward_workspace_bytes(x, w), dtype=torch.uint8, device="cuda")
    g, o, m, p = (torch.randn(2, 70, 80, device="cuda") for _ in range(4))

    def moved(call, written, read):
        before = [t._version for t in written + read]
        call()
        after = [t._version for t in written + read]
        assert all(a > b for a, b in zip(after, before[:len(written)]))
        assert after[len(written):] == before[len(written):]

    moved(lambda: P.prsgd_rms_norm(x, w, residual=dy, out=y, sum_out=s, rstd=rstd), [y, s, rstd], [x, w, dy])
    moved(lambda: P.prsgd_rms_norm_fp8(x, w, residual=dy, out=q, sum_out=s, scales=scales), [q, s, scales], [x, w, dy])
    moved(lambda: P.prsgd_rms_norm_backward(dy, s, rstd, w, dx=dx, dw=dw, workspace=ws), [dx, dw, ws], [dy, s, rstd, w])
    moved(lambda: P.prsgd_orthogonalize(g, out=o), [o], [g])
    moved(lambda: P.prsgd_muon_step(p, g, m, 0.1), [p, m], [g])

    leaf = torch.randn(2, 70, 80, device="cuda", requires_grad=True)
    for write in (lambda: P.prsgd_orthogonalize(g, out=p), lambda: P.prsgd_muon_step(p, g, m, 0.1), lambda: P.prsgd_muon_step(o, g, p, 0.1)):
        loss = (leaf * p).sum()                            # keeps p
        write()
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
