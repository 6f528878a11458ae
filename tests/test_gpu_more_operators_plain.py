"""The plain forms in perf/more_operators.py leave what they are given as it is and give the same twice, so that what they are compared with may run before or behind them."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def M():
    spec = importlib.util.spec_from_file_location("more_operators_cases", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _case(M, op, dtype):
    if op.startswith("embedding"):
        c = M._embedding("", op, dtype, 2, 60, 37, 20)
    elif op.startswith("scan"):
        c = M._scan("", op, dtype, 3, 20, 20, True)
    elif op == "dropout":
        c = M._dropout("", dtype, 2, 30, 20, True)
    else:
        c = M._xent("", op, dtype, 2, 30, 20, 37, True)
    del c["name"]
    return c


ADDS_TO_ITS_INPUT = pytest.mark.xfail(reason="adds dlast to the rows of dh that it is given: only its first pass over a state is the definition")


@pytest.mark.parametrize("op,dtype", [pytest.param(op, dtype, marks=ADDS_TO_ITS_INPUT if (op, dtype) == ("scan_backward", "f32") else ())
                                      for op in ("embedding", "embedding_backward", "scan", "scan_backward", "dropout", "xent", "xent_backward") for dtype in ("f32", "bf16")])
def test_plain_forms_leave_their_inputs(M, op, dtype):
    s = M.prepare(_case(M, op, dtype), 5)
    before = {k: v.clone() for k, v in vars(s).items() if isinstance(v, torch.Tensor)}
    first = {k: v.clone() for k, v in M.run(s).items()}
    again = M.run(s)
    # (sums that torch adds in any order, of a few terms)
    assert all(torch.allclose(first[k].float(), again[k].float(), rtol=1e-5, atol=1e-7) for k in first)
    assert all(torch.equal(getattr(s, k), v) for k, v in before.items())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_scans_gradients_are_those_of_a_first_pass(M, dtype):
    """The kernels' first and second pass over one state against a plain first pass over another of the same seed: fp32 roundings of some dozen steps, and the type's own."""
    case = _case(M, "scan_backward", dtype)
    want = M.run(M.prepare(case, 5))
    s = M.prepare(case, 5)
    M.own = True
    try:
        for _ in range(2):
            for k, v in M.run(s).items():
                step = 2.0 ** -8 if v.dtype == torch.bfloat16 else 1e-5
                assert bool(((v.float() - want[k].float()).abs() <= 2 * step * want[k].float().abs() + 1e-6 * want[k].float().abs().max()).all()), k
    finally:
        M.own = False
