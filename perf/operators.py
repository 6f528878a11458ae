"""Orthogonalised updates and root-mean-square norms, as cases that can be timed and compared.

A case is one call: `orthogonalize` (Newton-Schulz products on a replica set's update), `muon_step` (momentum,
orthogonalisation and update of the replicas), `norm` / `norm_fp8` / `norm_backward` (residual addition and
root-mean-square norm of N workers' rows, each worker with a weight vector of its own).

Matrices are [count][rows][cols], one per worker; rows of the norm are [workers * rows][width].
"""
import math

import torch

own = False

COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
ORTH_EPS = 1e-7
MOMENTUM, DECAY, RATE = 0.95, 0.01, 0.01
NORM_EPS = 1e-6
FP8_MAX, FP8_LEAST = 448.0, 2.0 ** -100      # largest e4m3 value; least row maximum that a scale is made of


def _matrices(name, op, dtype, count, rows, cols):
    return {"name": name, "op": op, "dtype": dtype, "count": count, "rows": rows, "cols": cols}


def _rows(name, op, dtype, workers, rows, width):
    return {"name": name, "op": op, "dtype": dtype, "workers": workers, "rows": rows, "width": width}


def listed():
    return [
        # the logits layers of many small replicas: a short side of ten, latency alone
        _matrices("orth_f32_64x128x10", "orthogonalize", "f32", 64, 128, 10),
        # the first layer of eight one-hidden-layer classifiers on image-sized rows
        _matrices("orth_f32_8x784x256", "orthogonalize", "f32", 8, 784, 256),
        # widths and a worker count that are multiples of nothing
        _matrices("orth_bf16_6x1000x500", "orthogonalize", "bf16", 6, 1000, 500),
        # a hidden layer of eight large replicas: matrix products alone
        _matrices("orth_bf16_8x4096x4096", "orthogonalize", "bf16", 8, 4096, 4096),
        # the whole step on the first layer of many small replicas
        _matrices("muon_f32_64x256x128", "muon_step", "f32", 64, 256, 128),
        # ... on the hidden layer of sixteen mid-sized ones, fp32 masters
        _matrices("muon_f32_16x1024x1024", "muon_step", "f32", 16, 1024, 1024),
        # ... on the wide last layer of large ones whose parameters are held in bf16
        _matrices("muon_bf16_8x4096x1000", "muon_step", "bf16", 8, 4096, 1000),
        # one row through the averaged model
        _rows("norm_bf16_1x4096", "norm", "bf16", 1, 1, 4096),
        # every row of eight workers' shards
        _rows("norm_bf16_8x8192x4096", "norm", "bf16", 8, 8192, 4096),
        # a minibatch of every worker, for products in 8 bits; an odd width
        _rows("norm_fp8_bf16_8x100x1000", "norm_fp8", "bf16", 8, 100, 1000),
        # gradients of sixteen workers' minibatches in fp32 ...
        _rows("norm_back_f32_16x64x1024", "norm_backward", "f32", 16, 64, 1024),
        # ... and of large ones in bf16
        _rows("norm_back_bf16_8x4096x4096", "norm_backward", "bf16", 8, 4096, 4096),
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    """As often a round one as one that is a multiple of nothing."""
    d = _log_int(rng, low, high)
    return d // 64 * 64 if rng.random() < 0.5 and d >= 128 else d


def draw(rng):
    """One more case of the listed ones' ranges."""
    op = rng.choice(["orthogonalize", "orthogonalize", "muon_step", "muon_step", "norm", "norm_fp8", "norm_backward"])
    dtype = rng.choice(["f32", "bf16"])
    if op in ("orthogonalize", "muon_step"):
        most = 6.0 * STEPS * 8 * 4096.0 ** 3 / (4 if dtype == "f32" else 1)
        while True:
            case = _matrices("", op, dtype, _log_int(rng, 1, 64), _width(rng, 8, 4096), _width(rng, 8, 4096))
            r, l = sorted((case["rows"], case["cols"]))
            if case["count"] * STEPS * (4.0 * r * r * l + 2.0 * r ** 3) <= most:
                break
    else:
        while True:
            case = _rows("", op, dtype, _log_int(rng, 1, 64), _log_int(rng, 1, 8192), _width(rng, 8, 16384))
            if case["workers"] * case["rows"] * case["width"] * (4 if dtype == "f32" else 2) <= 8 * 4096 * 4096 * 2:
                break
    del case["name"]
    return case


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _update(g, count, rows, cols, directions, noise):
    """An update as minibatch gradients leave it: few strong directions that fall off, and a floor of noise."""
    k = max(1, min(rows, cols, directions))
    dev = torch.device("cuda:0")
    weight = torch.arange(1, k + 1, device=dev, dtype=torch.float32) ** -0.5
    left = torch.randn((count, rows, k), generator=g, device=dev) * weight
    right = torch.randn((count, k, cols), generator=g, device=dev)
    return (left @ right).add_(torch.randn((count, rows, cols), generator=g, device=dev), alpha=noise).mul_(1e-3)


class _State:
    pass


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    s, dtype = _State(), _dtype(case)
    s.op = case["op"]
    if s.op in ("orthogonalize", "muon_step"):
        n, rows, cols = case["count"], case["rows"], case["cols"]
        s.g = _update(g, n, rows, cols, 256, 0.1).to(dtype)
        if s.op == "muon_step":
            s.m = _update(g, n, rows, cols, 512, 0.2) * 4.0
            s.x = (torch.randn((n, rows, cols), generator=g, device=dev) * math.sqrt(2.0 / rows)).to(dtype)
            s.scale = 0.2 * math.sqrt(max(rows, cols))
        return s
    n, rows, width = case["workers"], case["workers"] * case["rows"], case["width"]
    # the stream's rows differ in size, as they do behind several blocks; weights near one
    size = torch.exp(0.5 * torch.randn((rows, 1), generator=g, device=dev))
    s.x = torch.randn((rows, width), generator=g, device=dev).mul_(size).to(dtype)
    s.w = 1.0 + 0.2 * torch.randn((n, width), generator=g, device=dev)
    if s.op == "norm_backward":
        s.dy = torch.randn((rows, width), generator=g, device=dev).mul_(1e-2).to(dtype)
        s.ds = torch.randn((rows, width), generator=g, device=dev).mul_(1e-2).to(dtype)
        x = s.x.float()
        s.rstd = torch.rsqrt(x.square().mean(1) + NORM_EPS)
    else:
        s.res = torch.randn((rows, width), generator=g, device=dev).mul_(0.5).to(dtype)
    return s


# ---- plain forms: elementary operations in 32 bits, rounded once at the end -------------------------------------

def _orthogonal(u):
    a, b, c = COEFFICIENTS
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + ORTH_EPS)
    for _ in range(STEPS):
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return x.transpose(1, 2).contiguous() if tall else x


def _plain(s):
    if s.op == "orthogonalize":
        return {"out": _orthogonal(s.g.float()).to(s.g.dtype)}
    if s.op == "muon_step":
        g = s.g.float()
        s.m.mul_(MOMENTUM).add_(g)
        o = _orthogonal(g + MOMENTUM * s.m)
        s.x.copy_((1.0 - RATE * DECAY) * s.x.float() - RATE * s.scale * o)
        return {"x": s.x, "m": s.m}
    rows, width = s.x.shape
    by_worker = (s.w.shape[0], rows // s.w.shape[0], width)
    if s.op == "norm_backward":
        x, dy = s.x.float() * s.rstd[:, None], s.dy.float()
        dw = (dy * x).view(by_worker).sum(1)
        wdy = (dy.view(by_worker) * s.w[:, None]).view(rows, width)
        dx = s.rstd[:, None] * (wdy - x * (wdy * x).mean(1, keepdim=True)) + s.ds.float()
        return {"dx": dx.to(s.x.dtype), "dw": dw}
    x = s.x.float() + s.res.float()
    rstd = torch.rsqrt(x.square().mean(1) + NORM_EPS)
    y = ((x * rstd[:, None]).view(by_worker) * s.w[:, None]).view(rows, width)
    if s.op == "norm":
        return {"y": y.to(s.x.dtype), "sum": x.to(s.x.dtype), "rstd": rstd}
    scale = y.abs().amax(1).clamp(min=FP8_LEAST) / FP8_MAX
    return {"q": (y / scale[:, None]).to(torch.float8_e4m3fn), "scale": scale, "sum": x.to(s.x.dtype)}


def _kernels(s):
    from paper_1807_06629_amd import prsgd
    if s.op == "orthogonalize":
        return {"out": prsgd.prsgd_orthogonalize(s.g, coefficients=COEFFICIENTS, steps=STEPS, eps=ORTH_EPS)}
    if s.op == "muon_step":
        prsgd.prsgd_muon_step(s.x, s.g, s.m, RATE, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY, scale=s.scale,
                              coefficients=COEFFICIENTS, steps=STEPS, eps=ORTH_EPS)
        return {"x": s.x, "m": s.m}
    if s.op == "norm_backward":
        dx, dw = prsgd.prsgd_rms_norm_backward(s.dy, s.x, s.rstd, s.w, dsum=s.ds)
        return {"dx": dx, "dw": dw}
    if s.op == "norm":
        y, total, rstd = prsgd.prsgd_rms_norm(s.x, s.w, residual=s.res, eps=NORM_EPS)
        return {"y": y, "sum": total, "rstd": rstd}
    q, scale, total = prsgd.prsgd_rms_norm_fp8(s.x, s.w, residual=s.res, eps=NORM_EPS)
    return {"q": q, "scale": scale, "sum": total}


def run(state):
    return _kernels(state) if own else _plain(state)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if "count" in case:
        n, (r, l) = case["count"], sorted((case["rows"], case["cols"]))
        # symmetric products count half; by products with X, or by the Gram matrix and its polynomial alone
        by_x = STEPS * (3.0 * r * r * l + 1.0 * r ** 3)
        by_gram = 3.0 * r * r * l + (4.0 * STEPS - 3.0) * r ** 3
        elements = float(n * r * l)
        moved = 2 * es if case["op"] == "orthogonalize" else 3 * es + 8
        return {"bytes": elements * moved, "flops": n * min(by_x, by_gram)}
    rows, width = float(case["workers"] * case["rows"]), case["width"]
    weights = 4.0 * case["workers"] * width
    if case["op"] == "norm_backward":
        return {"bytes": rows * (4 * es * width + 4) + 2 * weights, "flops": 12.0 * rows * width}
    if case["op"] == "norm":
        return {"bytes": rows * (4 * es * width + 4) + weights, "flops": 5.0 * rows * width}
    return {"bytes": rows * ((3 * es + 1) * width + 4) + weights, "flops": 7.0 * rows * width}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def _polar(u):
    """The same polynomial of the singular values, applied through the Gram matrix of the short side: every iterate is
    P X0 with P a polynomial of the first Gram matrix, so that only P and the current Gram matrix are carried."""
    a, b, c = COEFFICIENTS
    u = u.double()
    flip = u.shape[0] > u.shape[1]
    x0 = (u.t() if flip else u) / (torch.linalg.matrix_norm(u) + ORTH_EPS)
    x0 = x0.contiguous()
    gram = x0.mm(x0.t().contiguous())
    p = None
    for _ in range(STEPS):
        q = torch.addmm(b * gram, gram, gram, alpha=c)
        q.diagonal().add_(a)
        gram = q.mm(gram).mm(q)
        p = q if p is None else q.mm(p)
    o = p.mm(x0)
    return o.t() if flip else o


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "orthogonalize":
        return {"out": torch.stack([_polar(u) for u in s.g])}
    if s.op == "muon_step":
        g, m, x = s.g.double(), s.m.double(), s.x.double()
        m = MOMENTUM * m + g
        for i in range(x.shape[0]):
            x[i] = x[i] - RATE * (DECAY * x[i] + s.scale * _polar(g[i] + MOMENTUM * m[i]))
        return {"x": x, "m": m}
    owner = torch.arange(case["workers"], device=s.x.device).repeat_interleave(case["rows"])
    d = case["width"]
    if s.op == "norm_backward":
        dx = torch.empty(s.x.shape, dtype=torch.float64, device=s.x.device)
        dw = torch.zeros(s.w.shape, dtype=torch.float64, device=s.x.device)
        for i in range(case["workers"]):
            at = slice(i * case["rows"], (i + 1) * case["rows"])
            x, dy, k = s.x[at].double(), s.dy[at].double(), s.rstd[at].double()[:, None]
            dw[i] = torch.sum(dy * x * k, 0)
            t = dy * s.w[i].double()
            dx[at] = k * t - k ** 3 / d * x * torch.sum(t * x, 1, keepdim=True) + s.ds[at].double()
        return {"dx": dx, "dw": dw}
    x = s.x.double() + s.res.double()
    ms = torch.sum(x * x, 1) / d
    y = x / torch.sqrt(ms + NORM_EPS)[:, None] * s.w.double()[owner]
    if s.op == "norm":
        return {"y": y, "sum": x, "rstd": 1.0 / torch.sqrt(ms + NORM_EPS)}
    scale = torch.clamp(torch.max(torch.abs(y), 1).values, min=FP8_LEAST) / FP8_MAX
    return {"q": y / scale[:, None], "scale": scale, "sum": x}
