"""The operators of replicas of a model over tokens in 64 bits, from their formulas (shared by their tests)."""
from __future__ import annotations

import numpy as np
import torch

from oracle.philox import philox4x32_10


def _tables(t):
    return t if t.dim() == 3 else t[None]


def embedding(tokens, table, scale=1.0):
    t = _tables(table).double()
    n, classes, width = t.shape
    y = torch.zeros((tokens.numel(), width), dtype=torch.float64, device=table.device)
    for r, v in enumerate(tokens.tolist()):
        if 0 <= v < classes:
            y[r] = t[r * n // tokens.numel(), v] * float(torch.tensor(scale, dtype=torch.float32))
    return y


def embedding_backward(dy, tokens, table, scale=1.0):
    t = _tables(table)
    n, classes, width = t.shape
    d = torch.zeros(t.shape, dtype=torch.float64, device=dy.device)
    for r, v in enumerate(tokens.tolist()):
        if 0 <= v < classes:
            d[r * n // tokens.numel(), v] += dy[r].double()
    return (d * float(torch.tensor(scale, dtype=torch.float32))).reshape(table.shape)


def spans(rows, sequences, starts):
    if starts is None:
        n = rows // sequences
        return [(s * n, (s + 1) * n) for s in range(sequences)]
    s = starts.tolist()
    return list(zip(s[:-1], s[1:]))


def gated_scan(v, gate, sequences=1, starts=None, initial=None, unit=0.0):
    """(h, last), and how far fp32 may be from them: E_t = f E_{t-1} + unit (f |h_{t-1}| + (1 - f) |v|), unit the rounding of a step.
    Rows that no sequence has are zeros."""
    v, gate = v.double(), gate.double()
    f, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    h, off = torch.zeros_like(v), torch.zeros_like(v)
    last = torch.zeros((sequences, v.shape[1]), dtype=torch.float64, device=v.device) if initial is None else initial.double().clone()
    far = torch.zeros_like(last)
    for s, (a, b) in enumerate(spans(v.shape[0], sequences, starts)):
        for t in range(a, b):
            far[s] = f[t] * far[s] + unit * (f[t] * last[s].abs() + rest[t] * v[t].abs())
            last[s] = f[t] * last[s] + rest[t] * v[t]
            h[t], off[t] = last[s], far[s]
    return h, last, off, far


def gated_scan_backward(dh, v, gate, h, sequences=1, starts=None, initial=None, dlast=None, unit=0.0):
    """(dv, dgate, dinitial), and the same of their errors as above (E of c_t, which moves to the row before)."""
    dh, v, gate, h = dh.double(), v.double(), gate.double(), h.double()
    f, rest = torch.sigmoid(gate), torch.sigmoid(-gate)
    dv, dgate, dv_off, dgate_off = (torch.zeros_like(v) for _ in range(4))
    c = torch.zeros((sequences, v.shape[1]), dtype=torch.float64, device=v.device) if dlast is None else dlast.double().clone()
    far = torch.zeros_like(c)
    for s, (a, b) in enumerate(spans(v.shape[0], sequences, starts)):
        for t in range(b - 1, a - 1, -1):
            g, g_off = dh[t] + c[s], far[s] + unit * (dh[t].abs() + c[s].abs())
            before = h[t - 1] if t > a else initial[s].double() if initial is not None else torch.zeros_like(c[s])
            dv[t], dv_off[t] = rest[t] * g, rest[t] * (g_off + unit * g.abs())
            k = f[t] * rest[t]
            dgate[t] = k * (before - v[t]) * g
            dgate_off[t] = k * ((before - v[t]).abs() * (g_off + unit * g.abs()) + unit * (before.abs() + v[t].abs()) * g.abs())
            c[s], far[s] = f[t] * g, f[t] * (g_off + unit * g.abs())
    return (dv, dgate, c), (dv_off, dgate_off, far)


def kept(rows, width, p, seed, step=0, layer=0):
    """Which elements dropout keeps: bool [rows][width], and the share that it drops."""
    per_row = (width + 7) // 8
    block = np.arange(rows * per_row, dtype=np.uint64)
    counter = np.stack([block & np.uint64(0xFFFFFFFF), np.full_like(block, step & 0xFFFFFFFF), np.full_like(block, step >> 32),
                        (block >> np.uint64(32)) + np.uint64(0x80000000 + (layer << 16))], -1)
    words = philox4x32_10(counter, np.array([seed & 0xFFFFFFFF, seed >> 32], dtype=np.uint64))
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], -1).reshape(rows, per_row * 8)[:, :width]
    dropped = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    return torch.from_numpy(halves >= dropped), dropped / 65536.0


def dropout(x, p, seed, step=0, layer=0, residual=None):
    keep, q = kept(x.shape[0], x.shape[1], p, seed, step, layer)
    y = torch.where(keep.to(x.device), x.double() / (1.0 - q), 0.0)
    return y if residual is None else y + residual.double()


def _products(h, w, classes_first):
    w = _tables(w).double()
    h = h.double().view(w.shape[0], -1, h.shape[1])
    return h, (w.transpose(1, 2) if classes_first else w).contiguous()


def linear_cross_entropy(h, w, labels, classes_first=False):
    """(loss, lse, sum |h| |w| at its largest over the classes)"""
    h, m = _products(h, w, classes_first)
    z = torch.bmm(h, m).flatten(0, 1)
    lse = torch.logsumexp(z, 1)
    real = (labels >= 0) & (labels < z.shape[1])
    at = torch.where(real, labels.long(), 0)[:, None]
    return torch.where(real, lse - z.gather(1, at)[:, 0], 0.0), lse, torch.bmm(h.abs(), m.abs()).flatten(0, 1).amax(1)


def linear_cross_entropy_backward(dloss, h, w, labels, lse, classes_first=False):
    """(dh, dw), and the sums of the absolute values that make each up."""
    rows, shape = h, w.shape
    h, m = _products(h, w, classes_first)
    z = torch.bmm(h, m).flatten(0, 1)
    real = (labels >= 0) & (labels < z.shape[1])
    p = torch.exp(z - lse.double()[:, None])
    one = torch.zeros_like(p)
    one[real, labels[real].long()] = 1.0
    weight = torch.where(real, dloss.double(), 0.0)[:, None]
    dz, size = (torch.where(real[:, None], v, 0.0).view(h.shape[0], -1, z.shape[1]) for v in (weight * (p - one), weight.abs() * (p + one)))
    clean = torch.where(real.view(h.shape[0], -1)[:, :, None], h, 0.0)
    t = lambda a: a.transpose(1, 2).contiguous()                          # noqa: E731
    out = []
    for d, hh, mm in ((dz, clean, m), (size, clean.abs(), m.abs())):
        dw = torch.bmm(t(hh), d)
        out += [torch.where(real[:, None], torch.bmm(d, t(mm)).reshape(rows.shape), 0.0), (t(dw) if classes_first else dw).reshape(shape)]
    return out
