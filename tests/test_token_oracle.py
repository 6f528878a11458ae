"""The 64-bit forms of the token operators against autograd, differences and sampling statistics (no GPU)."""
import torch
import torch.nn.functional as F

import token_oracle as O


def _g(seed):
    return torch.Generator().manual_seed(seed)


def test_embedding_is_the_gather_and_its_gradient():
    table = torch.randn(2, 7, 5, generator=_g(1), dtype=torch.float64, requires_grad=True)
    tokens = torch.tensor([0, 6, -1, 6, 3, 7, 6, 0], dtype=torch.int32)
    dy = torch.randn(8, 5, generator=_g(2), dtype=torch.float64)
    y = O.embedding(tokens, table, 0.5)
    want = torch.cat([F.embedding(tokens[4 * i:4 * i + 4].long().clamp(0, 6), table[i]) for i in range(2)]) * 0.5
    want = want * ((tokens >= 0) & (tokens < 7))[:, None]
    assert torch.equal(y, want)
    (want * dy).sum().backward()
    assert torch.allclose(O.embedding_backward(dy, tokens, table.detach(), 0.5), table.grad, atol=1e-14)


def test_scan_is_the_recurrence_and_its_gradient():
    rows, width, starts = 11, 3, torch.tensor([1, 1, 6, 10], dtype=torch.int32)
    v, gate = (torch.randn(rows, width, generator=_g(k), dtype=torch.float64, requires_grad=True) for k in (1, 2))
    initial = torch.randn(3, width, generator=_g(3), dtype=torch.float64, requires_grad=True)
    dh, dlast = torch.randn(rows, width, generator=_g(4), dtype=torch.float64), torch.randn(3, width, generator=_g(5), dtype=torch.float64)
    out, ends = [], []
    for s in range(3):
        state = initial[s]
        for t in range(int(starts[s]), int(starts[s + 1])):
            f = 1.0 / (1.0 + torch.exp(-gate[t]))
            state = f * state + (1.0 - f) * v[t]
            out.append((state * dh[t]).sum())
        ends.append(state)
    (torch.stack(out).sum() + (torch.stack(ends) * dlast).sum()).backward()
    h, last, _, _ = O.gated_scan(v.detach(), gate.detach(), 3, starts, initial.detach())
    assert torch.allclose(last, torch.stack(ends).detach()) and not h[0].any() and not h[10].any()
    (dv, dgate, dinitial), _ = O.gated_scan_backward(dh, v.detach(), gate.detach(), h, 3, starts, initial.detach(), dlast)
    for got, want in ((dv, v.grad), (dgate, gate.grad), (dinitial, initial.grad)):
        assert torch.allclose(got, want, atol=1e-13)


def test_dropout_drops_its_share_and_masks_differ():
    masks = [O.kept(200, 333, 0.3, 5)[0], O.kept(200, 333, 0.3, 6)[0], O.kept(200, 333, 0.3, 5, step=1)[0], O.kept(200, 333, 0.3, 5, layer=1)[0],
             O.kept(200, 333, 0.3, 5, step=1 << 32)[0]]
    n = 200 * 333
    for i, m in enumerate(masks):
        assert abs(float((~m).float().mean()) - 0.3) < 5 * (0.21 / n) ** 0.5
        for o in masks[:i]:                                # two independent masks agree in 0.58 of the places
            assert abs(float((m == o).float().mean()) - 0.58) < 5 * (0.2436 / n) ** 0.5
    assert O.kept(3, 9, 0.0, 1)[0].all() and O.kept(1, 8, 0.5, 1)[1] == 0.5


def test_cross_entropy_is_torchs_and_its_gradient():
    for first in (False, True):
        h = torch.randn(6, 4, generator=_g(1), dtype=torch.float64, requires_grad=True)
        w = torch.randn(2, *((9, 4) if first else (4, 9)), generator=_g(2), dtype=torch.float64, requires_grad=True)
        labels = torch.tensor([3, -1, 8, 0, 9, 3], dtype=torch.int32)
        real = (labels >= 0) & (labels < 9)
        dloss = torch.randn(6, generator=_g(3), dtype=torch.float64)
        z = torch.cat([h[3 * i:3 * i + 3] @ (w[i].t() if first else w[i]) for i in range(2)])
        loss = F.cross_entropy(z, torch.where(real, labels, 0).long(), reduction="none") * real
        got, lse, _ = O.linear_cross_entropy(h.detach(), w.detach(), labels, first)
        assert torch.allclose(got, loss.detach()) and torch.allclose(lse, torch.logsumexp(z, 1).detach())
        (loss * dloss).sum().backward()
        dh, dw, _, _ = O.linear_cross_entropy_backward(dloss, h.detach(), w.detach(), labels, lse, first)
        assert torch.allclose(dh, h.grad, atol=1e-13) and torch.allclose(dw, w.grad, atol=1e-13)
