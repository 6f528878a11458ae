"""The operators of replicas over tokens, one after another: on other streams, captured and replayed, two captured runs over one workspace, autograd's view of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def P():
    from paper_1807_06629_amd import prsgd
    return prsgd


def _rand(seed, *shape, dtype=F32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


class Run:
    """A replica's pass and its gradients with everything given, so that a call allocates nothing."""

    def __init__(self, P, dtype, n, sequences, length, width, classes, workspace=None):
        self.P, self.n, self.sequences = P, n, n * sequences
        rows = n * sequences * length
        self.tokens = torch.empty(rows, dtype=torch.int32, device="cuda")
        self.labels = torch.empty_like(self.tokens)
        self.table = _rand(1, n, classes, width, dtype=dtype) * width ** -0.5
        self.gate, self.dloss = _rand(2, rows, width, dtype=dtype) + 1, _rand(3, rows)
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.x, self.h, self.s, self.ds, self.dh, self.dv, self.dgate = (torch.empty(rows, width, dtype=dtype, device="cuda") for _ in range(7))
        self.last, self.dinitial = (torch.empty(self.sequences, width, device="cuda") for _ in range(2))
        self.loss, self.lse = (torch.empty(rows, device="cuda") for _ in range(2))
        self.dw, self.dtable = torch.empty_like(self.table), torch.empty_like(self.table)
        need = max(P.prsgd_embedding_backward_workspace_bytes(self.tokens, self.table), P.prsgd_gated_scan_workspace_bytes(self.x, self.sequences),
                   P.prsgd_linear_cross_entropy_workspace_bytes(self.s, self.table, True),
                   P.prsgd_linear_cross_entropy_backward_workspace_bytes(self.s, self.table, True))
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if workspace is None else workspace[:need]
        self.fill(0)

    def fill(self, k):
        g = torch.Generator().manual_seed(k)
        classes = self.table.shape[1]
        self.tokens.copy_(torch.randint(-1, classes, self.tokens.shape, generator=g, dtype=torch.int32))
        self.labels.copy_(torch.randint(-1, classes, self.tokens.shape, generator=g, dtype=torch.int32))
        self.step.fill_(k)

    def __call__(self):
        P, ws = self.P, self.workspace
        P.prsgd_embedding(self.tokens, self.table, 2.0, out=self.x)
        P.prsgd_gated_scan(self.x, self.gate, sequences=self.sequences, out=self.h, last=self.last, workspace=ws)
        P.prsgd_dropout(self.h, 0.2, 9, step=self.step, layer=1, residual=self.x, out=self.s)
        P.prsgd_linear_cross_entropy(self.s, self.table, self.labels, True, loss=self.loss, lse=self.lse, workspace=ws)
        P.prsgd_linear_cross_entropy_backward(self.dloss, self.s, self.table, self.labels, self.lse, True, dh=self.ds, dw=self.dw, workspace=ws)
        P.prsgd_dropout(self.ds, 0.2, 9, step=self.step, layer=1, out=self.dh)
        P.prsgd_gated_scan_backward(self.dh, self.x, self.gate, self.h, sequences=self.sequences, dv=self.dv, dgate=self.dgate, dinitial=self.dinitial,
                                    workspace=ws)
        P.prsgd_embedding_backward(self.dv, self.tokens, self.table, 2.0, dtable=self.dtable, workspace=ws)

    def results(self):
        return [t.clone() for t in (self.x, self.h, self.last, self.s, self.loss, self.lse, self.ds, self.dw, self.dh, self.dv, self.dgate, self.dinitial, self.dtable)]

    def clear(self):
        for t in (self.x, self.h, self.last, self.s, self.loss, self.lse, self.ds, self.dw, self.dh, self.dv, self.dgate, self.dinitial, self.dtable):
            t.fill_(float("nan"))


# few rows with a small table; long sequences that are cut; unaligned bf16 that is copied; aligned bf16
SHAPES = [(F32, 3, 2, 9, 20, 33), (F32, 1, 2, 1300, 24, 40), (BF16, 2, 2, 500, 132, 2100), (BF16, 2, 4, 64, 128, 512), (F32, 2, 1, 2100, 16, 300)]


@pytest.mark.parametrize("shape", SHAPES)
def test_captured_and_replayed(P, shape):
    run = Run(P, *shape)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        run()
    for k in range(4):
        run.fill(10 + k)
        run.clear()
        graph.replay()
        torch.cuda.synchronize()
        got = run.results()
        run.clear()
        run()
        assert all(torch.equal(a, b) for a, b in zip(got, run.results())), k
        (run.dtable.float() ** 2).sum().item()


def test_two_captured_runs_over_one_workspace(P):
    """One after another on one stream, in either order."""
    big = torch.full((64 << 20,), 0xFF, dtype=torch.uint8, device="cuda")
    runs = [Run(P, *SHAPES[k], workspace=big) for k in (1, 2)]
    graphs = []
    for r in runs:
        r()
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=torch.cuda.Stream()):
            r()
    for k, order in enumerate(((0, 1), (1, 0), (0, 0, 1))):
        for r in runs:
            r.fill(20 + k)
            r.clear()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        got = [r.results() for r in runs]
        for r, g in zip(runs, got):
            r.clear()
            r()
            assert all(torch.equal(a, b) for a, b in zip(g, r.results())), k


def test_other_streams_at_once(P):
    """Two runs on streams of their own, with workspaces of their own."""
    runs = [Run(P, *SHAPES[k]) for k in (2, 2)]
    runs[1].fill(5)
    want = []
    for r in runs:
        r()
        want.append(r.results())
        r.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r()
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        assert all(torch.equal(a, b) for a, b in zip(w, r.results()))


def _operands(case):
    x, table = _rand(1, 12, 20), _rand(2, 2, 9, 20)
    ids = torch.arange(12, dtype=torch.int32, device="cuda") % 9
    if case == "embedding":
        return {"table": table}, lambda P, o: P.prsgd_embedding(ids, **o)
    if case == "embedding_backward":
        return {"dy": x, "table": table}, lambda P, o: P.prsgd_embedding_backward(o["dy"], ids, o["table"])
    if case == "scan":
        return {"v": x, "gate": _rand(3, 12, 20), "initial": _rand(4, 2, 20)}, lambda P, o: P.prsgd_gated_scan(**o)
    if case == "scan_backward":
        return ({"dh": x, "v": _rand(3, 12, 20), "gate": _rand(4, 12, 20), "h": _rand(5, 12, 20), "dlast": _rand(6, 2, 20)},
                lambda P, o: P.prsgd_gated_scan_backward(sequences=2, **o))
    if case == "dropout":
        return {"x": x, "residual": _rand(3, 12, 20)}, lambda P, o: P.prsgd_dropout(p=0.1, seed=1, **o)
    if case == "cross_entropy":
        return {"h": x, "w": table}, lambda P, o: P.prsgd_linear_cross_entropy(labels=ids, classes_first=True, **o)
    return ({"dloss": _rand(3, 12), "h": x, "w": table, "lse": _rand(4, 12).abs() + 9},
            lambda P, o: P.prsgd_linear_cross_entropy_backward(labels=ids, classes_first=True, **o))


@pytest.mark.parametrize("case", ["embedding", "embedding_backward", "scan", "scan_backward", "dropout", "cross_entropy", "cross_entropy_backward"])
def test_what_requires_grad_is_refused_while_autograd_records(P, case):
    for name in _operands(case)[0]:
        o, call = _operands(case)
        if case == "embedding_backward" and name == "table":
            continue                                        # of which nothing is read
        o[name].requires_grad_()
        with pytest.raises(ValueError, match="grad"):
            call(P, o)
        with torch.no_grad():
            call(P, o)


def test_what_is_written_in_place_counts_as_changed(P):
    x, state = _rand(1, 12, 20), _rand(2, 2, 20)
    before = x._version, state._version
    P.prsgd_dropout(x, 0.1, 1, out=x)
    P.prsgd_gated_scan(_rand(3, 12, 20), _rand(4, 12, 20), initial=state, last=state)
    assert x._version > before[0] and state._version > before[1]
