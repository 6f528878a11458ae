"""Operators of replicas of a model over tokens, as cases that can be timed and compared.

A case is one call: `embedding` / `embedding_backward` (rows of every worker's own table, and its gradient), `scan` /
`scan_backward` (gated linear recurrence over packed sequences), `dropout` (with the residual, mask from a counter), `xent` /
`xent_backward` (softmax cross entropy of rows through every worker's last matrix, logits never stored whole).

Rows of all workers stand one behind another, [workers * rows][width]; tables are [workers][classes][width], last matrices that
or [workers][width][classes].  Tokens and labels below zero are padding.
"""
import math

import numpy as np
import torch

own = False

PADDING = 0.03                       # share of a worker's rows, at their end, that is padding


def _embedding(name, op, dtype, workers, rows, classes, width):
    return {"name": name, "op": op, "dtype": dtype, "workers": workers, "rows": rows, "classes": classes, "width": width}


def _scan(name, op, dtype, sequences, length, width, ragged):
    return {"name": name, "op": op, "dtype": dtype, "sequences": sequences, "length": length, "width": width, "ragged": ragged}


def _dropout(name, dtype, workers, rows, width, residual):
    return {"name": name, "op": "dropout", "dtype": dtype, "workers": workers, "rows": rows, "width": width, "residual": residual}


def _xent(name, op, dtype, workers, rows, width, classes, classes_first):
    return {"name": name, "op": op, "dtype": dtype, "workers": workers, "rows": rows, "width": width, "classes": classes,
            "classes_first": classes_first}


def listed():
    return [
        # a minibatch of every one of eight workers: 2048 tokens each
        _embedding("embedding_bf16_8x2048_32768x1024", "embedding", "bf16", 8, 2048, 32768, 1024),
        # gradients of many small replicas; sizes that are multiples of nothing
        _embedding("embedding_back_f32_64x100_1001x250", "embedding_backward", "f32", 64, 100, 1001, 250),
        # gradients of large tables: most rows are zeros, the commonest token has hundreds
        _embedding("embedding_back_bf16_8x8192_32768x1024", "embedding_backward", "bf16", 8, 8192, 32768, 1024),
        # one token of each of 64 sequences that are being continued
        _scan("scan_f32_64x1x1000", "scan", "f32", 64, 1, 1000, False),
        # sequences of every length, packed
        _scan("scan_bf16_64x1024x2048", "scan", "bf16", 64, 1024, 2048, True),
        # gradients of few long ones
        _scan("scan_back_bf16_4x16384x2048", "scan_backward", "bf16", 4, 16384, 2048, False),
        # minibatches of many small replicas
        _dropout("dropout_f32_64x8x128", "f32", 64, 8, 128, False),
        # every row of eight workers' shards
        _dropout("dropout_bf16_8x8192x4096", "bf16", 8, 8192, 4096, True),
        # how likely one token is, through the averaged model
        _xent("xent_bf16_1x1x4096x65536", "xent", "bf16", 1, 1, 4096, 65536, False),
        # the logits layers of many small replicas: latency
        _xent("xent_back_f32_64x8x128x10", "xent_backward", "f32", 64, 8, 128, 10, False),
        # the wide last layer of eight large classifiers
        _xent("xent_back_bf16_8x128x4096x1000", "xent_backward", "bf16", 8, 128, 4096, 1000, False),
        # replicas whose last matrix is the embedding's table: matrix products alone
        _xent("xent_back_bf16_2x4096x2048x32768", "xent_backward", "bf16", 2, 4096, 2048, 32768, True),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """As often a round one as one that is a multiple of nothing."""
    d = _log_int(rng, low, high)
    return d // 64 * 64 if rng.random() < 0.5 and d >= 128 else d


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["embedding", "embedding_backward", "scan", "scan", "scan_backward", "dropout", "xent", "xent_backward",
                     "xent_backward"])
    dtype = rng.choice(["f32", "bf16"])
    es = 4 if dtype == "f32" else 2
    while True:
        if op in ("embedding", "embedding_backward"):
            case = _embedding("", op, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 16384), _log_int(rng, 8, 131072), _width(rng, 8, 4096))
            fits = case["workers"] * (case["rows"] + case["classes"]) * case["width"] * es <= 1 << 30
        elif op in ("scan", "scan_backward"):
            length = 1 if rng.random() < 0.2 else _log_int(rng, 2, 32768)
            case = _scan("", op, dtype, _log_int(rng, 1, 256), length, _width(rng, 8, 4096), rng.random() < 0.5)
            fits = case["sequences"] * length * case["width"] * es <= 1 << 28
        elif op == "dropout":
            case = _dropout("", dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 8192), _width(rng, 8, 16384), rng.random() < 0.5)
            fits = case["workers"] * case["rows"] * case["width"] * es <= 1 << 29
        else:
            case = _xent("", op, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 4096), _width(rng, 8, 4096), _log_int(rng, 2, 65536),
                         rng.random() < 0.5)
            rows, size = case["workers"] * case["rows"], float(case["width"] * case["classes"])
            fits = (rows * size <= 8192.0 * 2048 * 32768 / (8 if dtype == "f32" else 1) and case["workers"] * size * es <= 1 << 29 and
                    rows * case["classes"] <= 1 << 28)
        if fits:
            del case["name"]
            return case


class _State:
    pass


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda:0")


def _ids(g, case):
    """Tokens as text has them, the k-th commonest 1 / k as often as the commonest; the end of every worker's rows is padding."""
    n, rows, classes = case["workers"], case["rows"], case["classes"]
    u = torch.rand((n, rows), generator=g, device="cuda:0", dtype=torch.float64)
    ids = torch.exp(u * math.log(classes + 1.0)).long().sub_(1).clamp_(0, classes - 1).to(torch.int32)
    ids[:, rows - int(PADDING * rows):] = -1
    return ids.view(-1)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s, dtype = _State(), _dtype(case)
    s.op, s.dtype = case["op"], dtype
    if s.op in ("embedding", "embedding_backward"):
        n, width = case["workers"], case["width"]
        s.tokens = _ids(g, case)
        s.scale = math.sqrt(width)
        s.table = _normal(g, n, case["classes"], width).mul_(width ** -0.5).to(dtype)
        if s.op == "embedding_backward":
            s.dy = _normal(g, n * case["rows"], width).mul_(1e-2).to(dtype)
        return s
    if s.op in ("scan", "scan_backward"):
        n, length, width = case["sequences"], case["length"], case["width"]
        rows = n * length
        s.sequences, s.starts = n, None
        if case["ragged"]:
            cuts = torch.randint(0, rows + 1, (n - 1,), generator=g, device=dev).sort().values
            s.starts = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), rows)]).to(torch.int32)
        # gates that forget over one to some hundred steps, by channel
        s.gate = (_normal(g, rows, width) + 2.0 + 1.5 * _normal(g, 1, width)).to(dtype)
        s.v = _normal(g, rows, width).to(dtype)
        s.initial = _normal(g, n, width).mul_(0.5)
        if s.op == "scan_backward":
            s.h = _scan_plain(s)[0].to(dtype)
            s.dh = _normal(g, rows, width).mul_(1e-2).to(dtype)
            s.dlast = _normal(g, n, width).mul_(1e-2)
        return s
    if s.op == "dropout":
        rows, width = case["workers"] * case["rows"], case["width"]
        s.x = _normal(g, rows, width).to(dtype)
        s.residual = _normal(g, rows, width).to(dtype) if case["residual"] else None
        s.p, s.seed, s.step, s.layer = 0.1, seed, 1000 + seed % 1000, 3
        return s
    n, rows, width, classes = case["workers"], case["rows"], case["width"], case["classes"]
    s.workers, s.classes_first = n, case["classes_first"]
    s.h = _normal(g, n * rows, width).to(dtype)
    shape = (n, classes, width) if s.classes_first else (n, width, classes)
    s.w = _normal(g, *shape).mul_(2.0 * width ** -0.5).to(dtype)
    s.labels = _ids(g, case)
    if s.op == "xent_backward":
        s.lse = torch.logsumexp(_logits(s), 2).view(-1)
        s.dloss = torch.full((n * rows,), 1.0 / (rows - int(PADDING * rows)), device=dev)
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once at the end -------------------------------------

def _rows_of_tables(s):
    """Row of all workers' tables that every token names, and whether it names one."""
    n, classes, _ = s.table.shape
    worker = torch.arange(n, device=s.tokens.device).repeat_interleave(s.tokens.numel() // n)
    real = (s.tokens >= 0) & (s.tokens < classes)
    return worker * classes + torch.where(real, s.tokens.long(), 0), real


def _first_rows(s):
    """Rows at which sequences that have any begin, and which those are."""
    n, rows = s.sequences, s.v.shape[0]
    starts = torch.arange(n + 1, device=s.v.device) * (rows // n) if s.starts is None else s.starts.long()
    some = starts[1:] > starts[:-1]
    return starts, some


def _doubling(f, b):
    """x_t = f_t x_{t-1} + b_t over the first axis (x_{-1} is 0), joining neighbours, then pairs, then fours; f and b are used up."""
    k = 1
    while k < f.shape[0]:
        b[k:] += f[k:] * b[:-k]
        f[k:] = f[k:] * f[:-k]
        k *= 2
    return b


def _scan_plain(s):
    starts, some = _first_rows(s)
    gate = s.gate.float()
    f, b = torch.sigmoid(gate), torch.sigmoid(-gate) * s.v.float()
    first = starts[:-1][some]
    b[first] += f[first] * s.initial[some]
    f[first] = 0.0
    h = _doubling(f, b)
    last = s.initial.clone()
    last[some] = h[starts[1:][some] - 1]
    return h, last


def _scan_back_plain(s):
    starts, some = _first_rows(s)
    gate = s.gate.float()
    f = torch.sigmoid(gate)
    first, end = starts[:-1][some], starts[1:][some] - 1
    b = s.dh.float()
    b[end] += s.dlast[some]
    after = torch.zeros_like(f)
    after[:-1] = f[1:]
    after[end] = 0.0
    grad = _doubling(after.flip(0), b.flip(0)).flip(0)
    before = torch.zeros_like(f)
    before[1:] = s.h[:-1].float()
    before[first] = s.initial[some]
    rest = torch.sigmoid(-gate)
    dinitial = s.dlast.clone()
    dinitial[some] = f[first] * grad[first]
    return {"dv": (rest * grad).to(s.dtype), "dgate": (f * rest * (before - s.v.float()) * grad).to(s.dtype), "dinitial": dinitial}


def _philox(counter, key):
    """Philox4x32-10 (Salmon et al., SC'11) of int64 tensors that hold 32-bit words."""
    low = 0xFFFFFFFF
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # wraps at 64 bits as an unsigned product does
        c0, c1, c2, c3 = (p1 >> 32 & low) ^ c1 ^ k0, p1 & low, (p0 >> 32 & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _kept(s):
    """Which elements stay: blocks of eight of a row share four words, 16 bits each."""
    rows, width = s.x.shape
    per_row = (width + 7) // 8
    block = torch.arange(rows * per_row, device=s.x.device)
    zero = torch.zeros_like(block)
    top = 0x80000000 | s.layer << 16
    words = _philox((block & 0xFFFFFFFF, zero + (s.step & 0xFFFFFFFF), zero + (s.step >> 32), (block >> 32) + top),
                    (s.seed & 0xFFFFFFFF, s.seed >> 32))
    halves = torch.stack([w >> shift & 0xFFFF for w in words for shift in (0, 16)], 1)
    return (halves >= _dropped(s.p)).view(rows, per_row * 8)[:, :width]


def _dropped(p):
    """Of 65536 equally likely values, those that drop an element."""
    return int(math.floor(p * 65536.0 + 0.5))


def _logits(s):
    w = s.w.float()
    return torch.bmm(s.h.float().view(s.workers, -1, s.h.shape[1]), w.transpose(1, 2) if s.classes_first else w)


def _plain(s):
    if s.op == "embedding":
        at, real = _rows_of_tables(s)
        rows = s.table.view(-1, s.table.shape[2])[at].float() * s.scale
        return {"y": (rows * real[:, None]).to(s.dtype)}
    if s.op == "embedding_backward":
        at, real = _rows_of_tables(s)
        dtable = torch.zeros((s.table.shape[0] * s.table.shape[1], s.table.shape[2]), device=s.dy.device)
        dtable.index_add_(0, at, s.dy.float() * (s.scale * real.float())[:, None])
        return {"dtable": dtable.view(s.table.shape).to(s.dtype)}
    if s.op == "scan":
        h, last = _scan_plain(s)
        return {"h": h.to(s.dtype), "last": last}
    if s.op == "scan_backward":
        return _scan_back_plain(s)
    if s.op == "dropout":
        y = torch.where(_kept(s), s.x.float() * (65536.0 / (65536.0 - _dropped(s.p))), 0.0)
        return {"y": (y if s.residual is None else y + s.residual.float()).to(s.dtype)}
    z = _logits(s)
    real = s.labels >= 0
    label = torch.where(real, s.labels.long(), 0)[:, None]
    if s.op == "xent":
        top = z.amax(2, keepdim=True)
        lse = (z - top).exp_().sum(2).log().view(-1) + top.view(-1)
        return {"loss": torch.where(real, lse - z.view(label.shape[0], -1).gather(1, label)[:, 0], 0.0), "lse": lse}
    dz = (z.view(label.shape[0], -1) - s.lse[:, None]).exp_()
    dz.scatter_add_(1, label, -torch.ones_like(s.lse)[:, None])
    dz.mul_(torch.where(real, s.dloss, 0.0)[:, None])
    dz, h, w = dz.view(z.shape), s.h.float().view(s.workers, -1, s.h.shape[1]), s.w.float()
    dh = torch.bmm(dz, w if s.classes_first else w.transpose(1, 2))
    dw = torch.bmm(dz.transpose(1, 2), h) if s.classes_first else torch.bmm(h.transpose(1, 2), dz)
    return {"dh": dh.view(s.h.shape).to(s.dtype), "dw": dw.to(s.dtype)}


def _kernels(s):
    from paper_1807_06629_amd import prsgd
    if s.op == "embedding":
        return {"y": prsgd.prsgd_embedding(s.tokens, s.table, scale=s.scale)}
    if s.op == "embedding_backward":
        return {"dtable": prsgd.prsgd_embedding_backward(s.dy, s.tokens, s.table, scale=s.scale)}
    if s.op == "scan":
        h, last = prsgd.prsgd_gated_scan(s.v, s.gate, sequences=s.sequences, starts=s.starts, initial=s.initial)
        return {"h": h, "last": last}
    if s.op == "scan_backward":
        dv, dgate, dinitial = prsgd.prsgd_gated_scan_backward(s.dh, s.v, s.gate, s.h, sequences=s.sequences, starts=s.starts,
                                                              initial=s.initial, dlast=s.dlast)
        return {"dv": dv, "dgate": dgate, "dinitial": dinitial}
    if s.op == "dropout":
        return {"y": prsgd.prsgd_dropout(s.x, s.p, s.seed, step=s.step, layer=s.layer, residual=s.residual)}
    if s.op == "xent":
        loss, lse = prsgd.prsgd_linear_cross_entropy(s.h, s.w, s.labels, classes_first=s.classes_first)
        return {"loss": loss, "lse": lse}
    dh, dw = prsgd.prsgd_linear_cross_entropy_backward(s.dloss, s.h, s.w, s.labels, s.lse, classes_first=s.classes_first)
    return {"dh": dh, "dw": dw}


def run(state):
    return _kernels(state) if own else _plain(state)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    op, width = case["op"], float(case["width"])
    if op in ("embedding", "embedding_backward"):
        n, rows, classes = case["workers"], case["rows"], case["classes"]
        real = rows - int(PADDING * rows)
        if op == "embedding_backward":
            return {"bytes": n * (4.0 * rows + (real + classes) * width * es), "flops": n * 2.0 * real * width}
        k = np.arange(1, classes + 1)
        p = np.log1p(1.0 / k) / math.log(classes + 1.0)
        distinct = float(np.sum(1.0 - (1.0 - p) ** real))
        return {"bytes": n * (4.0 * rows + (distinct + rows) * width * es), "flops": n * real * width}
    if op in ("scan", "scan_backward"):
        elements, state = case["sequences"] * case["length"] * width, 4.0 * case["sequences"] * width
        if op == "scan":
            return {"bytes": 3 * es * elements + 2 * state, "flops": 8.0 * elements}
        return {"bytes": 6 * es * elements + 3 * state, "flops": 14.0 * elements}
    if op == "dropout":
        elements = case["workers"] * case["rows"] * width
        return {"bytes": (3 if case["residual"] else 2) * es * elements, "flops": 2.0 * elements}
    n, rows, classes = case["workers"], float(case["rows"]), float(case["classes"])
    product = 2.0 * n * rows * width * classes
    if op == "xent":
        return {"bytes": n * (es * width * (rows + classes) + 12.0 * rows), "flops": product}
    return {"bytes": n * (2 * es * width * (rows + classes) + 12.0 * rows), "flops": 3.0 * product}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _steps(s):
    """Rows of the sequences at each position, longest sequences first, so that those still running are the first ones."""
    rows, n = s.v.shape[0], s.sequences
    starts = torch.arange(n + 1, device=s.v.device) * (rows // n) if s.starts is None else s.starts.long()
    lengths, order = (starts[1:] - starts[:-1]).sort(descending=True)
    running = (lengths[None, :] > torch.arange(int(lengths[0]), device=s.v.device)[:, None]).sum(1).tolist()
    return starts[:-1][order], order, running


def _mulhilo16(a, m):
    """High and low words of a 32-bit product, by halves."""
    al, ah, ml, mh = a & 0xFFFF, a >> 16, m & 0xFFFF, m >> 16
    mid = (al * ml >> 16) + (ah * ml & 0xFFFF) + (al * mh & 0xFFFF)
    return ah * mh + (ah * ml >> 16) + (al * mh >> 16) + (mid >> 16), (mid & 0xFFFF) << 16 | (al * ml & 0xFFFF)


def _exact_dropout(s):
    rows, width = s.x.shape
    column = torch.arange(width, device=s.x.device)
    row = torch.arange(rows, device=s.x.device)[:, None]
    which = row * ((width + 7) // 8) + torch.arange((width + 7) // 8, device=s.x.device)
    a, b, c, d = (which % 2 ** 32, torch.full_like(which, s.step % 2 ** 32), torch.full_like(which, s.step // 2 ** 32),
                  which // 2 ** 32 + (2 ** 31 + 2 ** 16 * s.layer))
    for i in range(10):
        h0, l0 = _mulhilo16(a, 0xD2511F53)
        h1, l1 = _mulhilo16(c, 0xCD9E8D57)
        a, b, c, d = (h1 ^ b ^ ((s.seed % 2 ** 32 + i * 0x9E3779B9) % 2 ** 32), l1,
                      h0 ^ d ^ ((s.seed // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32), l0)
    word = torch.stack([a, b, c, d], 2)[:, column // 8, column % 8 // 2]
    half = torch.where(column % 2 == 0, word % 65536, word // 65536)
    q = round(s.p * 65536)
    y = s.x.double() / (1.0 - q / 65536.0) * (half >= q)
    return y if s.residual is None else s.residual.double() + y


def exact(case, seed):
    op = case["op"]
    if op in ("scan", "scan_backward") and case["length"] * (case["sequences"] if case["ragged"] else 1) > 100000:
        return None
    if op == "dropout" and case["workers"] * case["rows"] * case["width"] > 1 << 28:
        return None
    s = prepare(case, seed)
    if op == "dropout":
        return {"y": _exact_dropout(s)}
    if op in ("embedding", "embedding_backward"):
        n, rows = case["workers"], case["rows"]
        by_worker = s.tokens.view(n, rows).long()
        if op == "embedding":
            y = torch.zeros((n, rows, case["width"]), dtype=torch.float64, device=s.tokens.device)
            for i in range(n):
                real = by_worker[i] >= 0
                y[i, real] = s.table[i].double()[by_worker[i, real]] * s.scale
            return {"y": y.view(n * rows, -1)}
        dtable = torch.zeros(s.table.shape, dtype=torch.float64, device=s.tokens.device)
        for i in range(n):
            real = by_worker[i] >= 0
            dtable[i].index_add_(0, by_worker[i, real], s.dy.view(n, rows, -1)[i, real].double())
        return {"dtable": dtable * s.scale}
    if op in ("scan", "scan_backward"):
        first, order, running = _steps(s)
        state = s.initial.double()[order]
        if op == "scan":
            h = torch.empty(s.v.shape, dtype=torch.float64, device=s.v.device)
            for t, k in enumerate(running):
                at = first[:k] + t
                f = 1.0 / (1.0 + torch.exp(-s.gate[at].double()))
                state[:k] = f * state[:k] + (1.0 - f) * s.v[at].double()
                h[at] = state[:k]
            last = torch.empty_like(state)
            last[order] = state
            return {"h": h, "last": last}
        dv, dgate = (torch.empty(s.v.shape, dtype=torch.float64, device=s.v.device) for _ in range(2))
        grad = s.dlast.double()[order]
        for t in range(len(running) - 1, -1, -1):
            k = running[t]
            at = first[:k] + t
            f = 1.0 / (1.0 + torch.exp(-s.gate[at].double()))
            total = grad[:k] + s.dh[at].double()
            before = state[:k] if t == 0 else s.h[at - 1].double()
            dv[at] = (1.0 - f) * total
            dgate[at] = f * (1.0 - f) * (before - s.v[at].double()) * total
            grad[:k] = f * total
        dinitial = torch.empty_like(grad)
        dinitial[order] = grad
        return {"dv": dv, "dgate": dgate, "dinitial": dinitial}
    n, rows = case["workers"], case["rows"]
    out = []
    for i in range(n):
        at = slice(i * rows, (i + 1) * rows)
        h, label = s.h[at].double(), s.labels[at].long()
        w = s.w[i].double().t().contiguous() if s.classes_first else s.w[i].double()
        z = torch.mm(h, w)
        real = label >= 0
        if op == "xent":
            lse = torch.logsumexp(z, 1)
            picked = z[torch.arange(rows, device=z.device), label.clamp(min=0)]
            out.append((torch.where(real, lse - picked, 0.0), lse))
        else:
            dz = torch.exp(z - s.lse[at].double()[:, None])
            dz[real, label[real]] -= 1.0
            dz *= (s.dloss[at].double() * real)[:, None]
            dw = torch.mm(h.t().contiguous(), dz)
            out.append((torch.mm(dz, w.t().contiguous()), dw.t().contiguous() if s.classes_first else dw))
    if op == "xent":
        return {"loss": torch.cat([v[0] for v in out]), "lse": torch.cat([v[1] for v in out])}
    return {"dh": torch.cat([v[0] for v in out]), "dw": torch.stack([v[1] for v in out])}
