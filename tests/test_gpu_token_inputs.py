"""Inputs of the token operators stay as they were, and a call gives the same again, also behind another one on other inputs."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _make(case, dtype, seed):
    """Operands by name, and the call."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*shape, dtype=dtype):
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    def ids(n, classes):
        return torch.randint(-1, classes + 1, (n,), generator=g, device="cuda").to(torch.int32)

    if case.startswith("embedding"):
        rows = 700 if case.endswith("many") else 90
        o = {"tokens": ids(2 * rows, 50), "table": rand(2, 50, 37), "dy": rand(2 * rows, 37)}
        if "backward" in case:
            return o, lambda P, o: (P.prsgd_embedding_backward(o["dy"], o["tokens"], o["table"], 1.5),)
        return o, lambda P, o: (P.prsgd_embedding(o["tokens"], o["table"], 1.5),)
    if case.startswith("scan"):
        rows, width = (3000, 20) if case.endswith("cut") else (150, 45)
        packed = torch.tensor([3, 40, 40, rows - 2], dtype=torch.int32, device="cuda") if "packed" in case else None
        n = 3
        o = {"v": rand(rows, width), "gate": rand(rows, width), "initial": rand(n, width, dtype=F32), "dh": rand(rows, width), "h": rand(rows, width),
             "dlast": rand(n, width, dtype=F32)}
        kw = {"sequences": n, "starts": packed}
        if packed is not None:
            o["starts"] = packed
        if "backward" in case:
            return o, lambda P, o: P.prsgd_gated_scan_backward(o["dh"], o["v"], o["gate"], o["h"], initial=o["initial"], dlast=o["dlast"], **kw)
        return o, lambda P, o: P.prsgd_gated_scan(o["v"], o["gate"], initial=o["initial"], **kw)
    if case == "dropout":
        o = {"x": rand(60, 45), "residual": rand(60, 45), "step": torch.tensor([seed], device="cuda")}
        return o, lambda P, o: (P.prsgd_dropout(o["x"], 0.3, 5, step=o["step"], residual=o["residual"]),)
    rows, width, classes, first = {"small": (8, 64, 10, False), "narrow": (30, 300, 3, False), "pair": (70, 96, 200, True), "copied": (300, 1001, 515, False),
                                   "large": (256, 512, 1024, True), "long": (40, 2100, 40, False)}[case.split("_")[-1]]
    o = {"h": rand(2 * rows, width), "w": rand(2, *((classes, width) if first else (width, classes))) * width ** -0.5, "labels": ids(2 * rows, classes),
         "dloss": rand(2 * rows, dtype=F32)}
    o["w"] = o["w"].contiguous()
    o["lse"] = torch.logsumexp(torch.bmm(o["h"].float().view(2, rows, width), (o["w"].float().transpose(1, 2) if first else o["w"].float()).contiguous()), 2).flatten()
    if "backward" in case:
        return o, lambda P, o: P.prsgd_linear_cross_entropy_backward(o["dloss"], o["h"], o["w"], o["labels"], o["lse"], first)
    return o, lambda P, o: P.prsgd_linear_cross_entropy(o["h"], o["w"], o["labels"], first)


CASES = (["embedding", "embedding_backward_few", "embedding_backward_many", "dropout"] +
         ["scan" + b + p + c for b in ("", "_backward") for p in ("", "_packed") for c in ("", "_cut")] +
         ["loss" + b + "_" + s for b in ("", "_backward") for s in ("small", "narrow", "pair", "copied", "large", "long")])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", CASES)
def test_inputs_stay_and_passes_repeat(P, case, dtype):
    o, call = _make(case, dtype, 1)
    other, _ = _make(case, dtype, 2)
    before = {k: v.clone() for k, v in o.items()}
    first = [t.clone() for t in call(P, o)]
    call(P, other)
    again = call(P, o)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert all(torch.equal(v, before[k]) for k, v in o.items())
