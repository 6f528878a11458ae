"""The operators on replica sets in 64 bits, from their formulas (shared by their tests)."""
from __future__ import annotations

import torch

NS = (3.4445, -4.7750, 2.0315)


def orthogonalize(g: torch.Tensor, coefficients=NS, steps=5, eps=1e-7) -> torch.Tensor:
    """[count][rows][cols], any type and device: the products as the definition has them."""
    a, b, c = (float(torch.tensor(v, dtype=torch.float32)) for v in coefficients)
    out = torch.empty(g.shape, dtype=torch.float64, device=g.device)
    for k in range(g.shape[0]):
        x = g[k].double()
        flip = x.shape[0] > x.shape[1]
        x = x.t().contiguous() if flip else x
        norm = x.norm() + float(torch.tensor(eps, dtype=torch.float32))
        x = x / norm if float(norm) != 0.0 else x
        for _ in range(steps):
            gram = x @ x.t().contiguous()
            x = a * x + (b * gram + c * (gram @ gram)) @ x
        out[k] = x.t() if flip else x
    return out


def muon_step(x, g, m, lr, mu, nesterov, weight_decay, scale, **kw):
    """(x, m) after the step."""
    x, g, m = x.double(), g.double(), m.double()
    m = mu * m + g
    o = orthogonalize(g + mu * m if nesterov else m, **kw)
    return (1.0 - lr * weight_decay) * x - lr * scale * o, m


def _weights(w, rows):
    w = w.double()
    if w.dim() == 1:
        return w.expand(rows, w.shape[0])
    return w.repeat_interleave(rows // w.shape[0], 0)


def rms_norm(x, w, residual=None, eps=1e-6):
    """(y, s, rstd)"""
    s = x.double() if residual is None else x.double() + residual.double()
    rstd = 1.0 / torch.sqrt((s * s).mean(1) + eps)
    return s * rstd[:, None] * _weights(w, x.shape[0]), s, rstd


def rms_norm_backward(dy, s, rstd, w, dsum=None):
    """(dx, dw)"""
    dy, s, rstd = dy.double(), s.double(), rstd.double()[:, None]
    sh, wdy = s * rstd, _weights(w, dy.shape[0]) * dy
    dx = rstd * (wdy - sh * (wdy * sh).mean(1, keepdim=True))
    if dsum is not None:
        dx = dx + dsum.double()
    per = (dy * sh).reshape(1 if w.dim() == 1 else w.shape[0], -1, dy.shape[1]).sum(1)
    return dx, per.reshape(w.shape)
