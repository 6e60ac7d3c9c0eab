"""The selective scan by its definition in 64 bits on the CPU, token by token, differentiable; inputs for it."""
from __future__ import annotations

import math

import torch
import torch.nn.functional as F

NAMES = ("u", "dt", "a", "b", "c", "d", "z", "dt_bias", "state")
GRADS = ("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias", "dstate")


def inputs(tokens, channels, states, groups, n, dtype, seed=0, softplus=True):
    """u, dt, a, b, c, d, z, dt_bias, state and dJ/dout, dJ/dfinal: decays and step sizes as such layers have them."""
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    a = -torch.arange(1, states + 1).float() * torch.exp(0.3 * randn(channels, states))
    step = torch.exp(math.log(1e-3) + math.log(300.0) * torch.rand(channels, generator=gen))
    bias = torch.log(torch.expm1(step)) if softplus else step
    dt = 0.7 * randn(tokens, channels) if softplus else 0.05 * torch.rand(tokens, channels, generator=gen)
    x = dict(u=randn(tokens, channels).to(dtype), dt=dt.to(dtype), a=a, b=randn(tokens, groups, states).to(dtype),
             c=randn(tokens, groups, states).to(dtype), d=1 + 0.1 * randn(channels), z=randn(tokens, channels).to(dtype),
             dt_bias=bias, state=0.3 * randn(n, channels, states))
    return x, randn(tokens, channels).to(dtype), 0.3 * randn(n, channels, states)


def scan(x, off, softplus=True):
    """(out, last states) of float64 (differentiable) inputs; d, z, dt_bias and state may be None."""
    u, b, c = x["u"], x["b"], x["c"]
    channels = u.shape[1]
    per = channels // b.shape[1]
    b, c = b.repeat_interleave(per, 1), c.repeat_interleave(per, 1)
    s = x["dt"] if x["dt_bias"] is None else x["dt"] + x["dt_bias"]
    if softplus:
        s = F.softplus(s, threshold=1000.0)
    n = len(off) - 1
    h0 = torch.zeros(n, channels, b.shape[2], dtype=torch.float64) if x["state"] is None else x["state"]
    ys, finals = [], []
    for i in range(n):
        h = h0[i]
        for t in range(off[i], off[i + 1]):
            h = torch.exp(s[t][:, None] * x["a"]) * h + (s[t] * u[t])[:, None] * b[t]
            ys.append((h * c[t]).sum(-1))
        finals.append(h)
    y = torch.stack(ys) if ys else torch.zeros_like(u)
    if x["d"] is not None:
        y = y + x["d"] * u
    if x["z"] is not None:
        y = y * x["z"] * torch.sigmoid(x["z"])
    return y, torch.stack(finals)


def scan_even(x, n, softplus=True):
    """The same of n sequences of one length, all at once."""
    tokens, channels = x["u"].shape
    length, per = tokens // n, channels // x["b"].shape[1]
    cut = lambda t: t.reshape(n, length, *t.shape[1:])  # noqa: E731
    u, b, c = cut(x["u"]), cut(x["b"]).repeat_interleave(per, 2), cut(x["c"]).repeat_interleave(per, 2)
    s = cut(x["dt"] if x["dt_bias"] is None else x["dt"] + x["dt_bias"])
    if softplus:
        s = F.softplus(s, threshold=1000.0)
    h, ys = x["state"], []
    for t in range(length):
        h = torch.exp(s[:, t, :, None] * x["a"]) * h + (s[:, t] * u[:, t])[..., None] * b[:, t]
        ys.append((h * c[:, t]).sum(-1))
    y = (torch.stack(ys, 1) + x["d"] * u).reshape(tokens, channels)
    return y * x["z"] * torch.sigmoid(x["z"]), h
