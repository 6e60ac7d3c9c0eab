"""Plain references of the operators in 64 bits, on the CPU, written from their
definitions: layer norm by rows, the gated delta rule token by token (its
gradients by torch's autograd over that loop), sampling from sorted shares."""
from __future__ import annotations

import math

import numpy as np
import torch


def rel(got, want) -> float:
    """2-norm of the difference over the 2-norm of the result."""
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape, (got.shape, want.shape)
    assert torch.isfinite(got).all() == torch.isfinite(want).all()
    if want.numel() == 0:
        return 0.0
    scale = want.norm().item()
    return (got - want).norm().item() / scale if scale else (got - want).norm().item()


def layer_norm(x, w, b, eps):
    x = x.double().cpu()
    mean = x.mean(-1, keepdim=True)
    var = (x - mean).square().mean(-1, keepdim=True)
    y = (x - mean) / torch.sqrt(var + eps)
    if w is not None:
        y = y * w.double().cpu()
    return y if b is None else y + b.double().cpu()


def delta(q, k, v, g, beta, off, state, scale):
    """(out, last memories) of packed sequences; differentiable in every float64 argument."""
    hv, hk = v.shape[1], q.shape[1]
    q, k = (x.repeat_interleave(hv // hk, 1) for x in (q, k))
    outs, finals = [], []
    for i in range(len(off) - 1):
        s = state[i]
        for t in range(off[i], off[i + 1]):
            s = s * torch.exp(g[t])[:, None, None]
            held = (k[t][:, :, None] * s).sum(1)
            s = s + beta[t][:, None, None] * k[t][:, :, None] * (v[t] - held)[:, None, :]
            outs.append(scale * (q[t][:, :, None] * s).sum(1))
        finals.append(s)
    out = torch.stack(outs) if outs else torch.zeros_like(v)
    return out, (torch.stack(finals) if finals else torch.zeros_like(state))


def stays(logits, temperature, top_k, top_p, min_p):
    """Shares of one row's choices after the filters, in float64, and the widths
    of the doubt about each cut: (shares, total share at which a cut may move)."""
    x = np.where(np.isnan(logits), -np.inf, logits.astype(np.float64))
    m = x.max()
    if m == np.inf:
        e = (x == np.inf).astype(np.float64)
    else:
        e = np.exp((x - m) / temperature)
    e[x == -np.inf] = 0.0
    order = np.lexsort((np.arange(len(x)), -x))
    keep = np.zeros(len(x), bool)
    keep[order[:top_k if top_k > 0 else len(x)]] = True
    keep &= e >= min_p * (1 - 1e-6)
    e = e * keep
    total = e.sum()
    before = np.cumsum(e[order]) - e[order]
    inside = before < top_p * total
    inside[0] = True
    keep2 = np.zeros(len(x), bool)
    keep2[order[inside]] = True
    return e * keep2, order


def log_softmax_of(shares, token) -> float:
    return math.log(shares[token] / shares.sum())
