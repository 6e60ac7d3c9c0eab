"""The operators together, as examples/recurrent_policy.py runs them: the frame
by frame calls against the whole episode's, and the gradients that reach the
features and the policy's weights against float64 automatic differentiation of
the definition on the CPU.

Tolerances.  Every quantity is a chain of float32 sums of at most 64 terms (2^-24
each) and products whose operands are split to 24 bits; T = 5 frames and six such
steps in a row stay below 5 * 6 * 64 * 2^-24 = 1.1e-4 of the largest magnitude
involved, whatever the order: 2e-4 of max(1, largest) is asked for.
"""
import numpy as np
import pytest

from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

TOL = 2e-4


def _reference(policy, rows, n, T):
    """(logits, leaves) of whole episodes from the definition, float64, differentiable."""
    import torch
    import torch.nn.functional as F
    x = rows.detach().cpu().double().requires_grad_()
    nw, nb, w_in, w_out = leaves = [p.detach().cpu().double().requires_grad_() for p in policy.params]
    mean, var = x.mean(1, keepdim=True), x.var(1, keepdim=True, unbiased=False)
    y = (x - mean) / torch.sqrt(var + 1e-5) * nw + nb
    q, k, v, g, b = (y @ w_in).split(policy.split, dim=1)
    H, dk, dv = policy.heads, policy.dk, policy.dv
    k = F.normalize(k.reshape(n, T, H, dk), dim=3)
    q, v = q.reshape(n, T, H, dk), v.reshape(n, T, H, dv)
    g, b = -F.softplus(g - 2.0).reshape(n, T, H), torch.sigmoid(b).reshape(n, T, H)
    S = torch.zeros((n, H, dk, dv), dtype=torch.float64)
    outs = []
    for t in range(T):
        S = S * torch.exp(g[:, t])[..., None, None]
        e = v[:, t] - (S * k[:, t][..., None]).sum(2)
        S = S + b[:, t][..., None, None] * k[:, t][..., None] * e[:, :, None, :]
        outs.append((S * q[:, t][..., None]).sum(2) * dk ** -0.5)
    return torch.stack(outs, 1).reshape(n * T, H * dv) @ w_out, [x] + leaves


def test_frames_and_episodes_agree():
    import torch
    import torch.nn.functional as F
    from examples import recurrent_policy as R
    n, T = 7, 5
    net, policy, frames = R.make(n, T)
    feats = torch.stack([net.step(frames[t]).clone() for t in range(T)], 1).reshape(n * T, -1)
    u = torch.rand((T, n), generator=torch.Generator().manual_seed(3)).cuda()
    memory = policy.memory(n)
    got = [policy.act(feats.view(n, T, -1)[:, t].contiguous(), memory, u[t]) for t in range(T)]
    actions = torch.stack([a for a, _ in got], 1).reshape(-1, 1).long()
    logp = torch.stack([p for _, p in got], 1).reshape(-1, 1)

    rows = feats.clone().requires_grad_()
    logits = policy.episode_logits(rows, n)
    want, leaves = _reference(policy, rows, n, T)
    scale = max(1.0, want.abs().max().item())
    assert (logits.detach().cpu() - want).abs().max().item() <= TOL * scale
    assert (F.log_softmax(want, 1).gather(1, actions.cpu()) - logp.cpu()).abs().max().item() <= 2 * TOL * scale

    dl = torch.randn(want.shape, generator=torch.Generator().manual_seed(4), dtype=torch.float64)
    grads = torch.autograd.grad(logits, [rows] + policy.params, dl.float().cuda())
    refs = torch.autograd.grad(want, leaves, dl.float().double())
    for i, (a, b) in enumerate(zip(grads, refs)):
        err = (a.cpu() - b).abs().max().item()
        assert err <= TOL * max(1.0, b.abs().max().item()), (i, err)
    net.close()


def test_training_raises_the_reward():
    import torch
    from examples import recurrent_policy as R
    n, T = 32, 8
    net, policy, frames = R.make(n, T)
    wanted = torch.zeros(n, device="cuda", dtype=torch.int32)
    gen = torch.Generator().manual_seed(5)
    rewards = [R.episode(net, policy, frames, torch.rand((T, n), generator=gen).cuda(), wanted, 1.0)[0].item()
               for _ in range(30)]
    assert np.mean(rewards[-5:]) > np.mean(rewards[:5]) + 0.1, rewards
    net.close()
