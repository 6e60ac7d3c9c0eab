"""A policy with a memory over many streams, trained with REINFORCE on the device.

Each frame of a stream goes through a reuse net, whose outputs serve as features;
they are normalised and projected to a query, a key, a value, a decay and a write
strength; the stream's memory is read and written by the gated delta rule; and an
action is drawn from logits formed of what was read.  After an episode the same
frames' features go through the operators as whole sequences, the gradients come
back through them to the features, and the frames are replayed through the net,
whose backward pass takes them over.

    python -m examples.recurrent_policy --streams 256 --frames 16 --episodes 5

The reward is synthetic: 1 where the action is a fixed function of the stream.
"""
from __future__ import annotations

import argparse
import time

import torch
import torch.nn.functional as F

from paper_1909_05632_amd import ReuseNet, ops
from synth import frames as synth


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        y, stats = ops.layer_norm(x, weight, bias, with_stats=True)
        ctx.save_for_backward(x, weight, stats)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        return ops.layer_norm_backward(dy.contiguous(), x, weight, stats)


class DeltaRule(torch.autograd.Function):
    """All tokens of n sequences of one length, from empty memories."""

    @staticmethod
    def forward(ctx, q, k, v, g, beta, n):
        out, _, saved = ops.delta_forward(q, k, v, g, beta, n=n, save=True)
        ctx.save_for_backward(q, k, v, g, beta, saved)
        ctx.n = n
        return out

    @staticmethod
    def backward(ctx, dout):
        *inputs, saved = ctx.saved_tensors
        grads = ops.delta_backward(dout.contiguous(), *inputs, n=ctx.n, saved=saved, want_dstate=False)
        return (*grads[:5], None)


class RecurrentPolicy:
    """Features [rows][width] to logits [rows][actions], a memory per stream between frames."""

    def __init__(self, width: int, actions: int, heads: int = 2, dk: int = 32, dv: int = 32, seed: int = 0):
        gen = torch.Generator().manual_seed(seed)

        def param(*shape, std=None):
            x = torch.zeros(shape) if std is None else torch.randn(shape, generator=gen) * std
            return x.cuda().requires_grad_()

        self.heads, self.dk, self.dv = heads, dk, dv
        self.split = [heads * dk, heads * dk, heads * dv, heads, heads]
        self.norm_w, self.norm_b = torch.ones(width).cuda().requires_grad_(), param(width)
        self.w_in = param(width, sum(self.split), std=width ** -0.5)
        self.w_out = param(heads * dv, actions, std=(heads * dv) ** -0.5)
        self.params = [self.norm_w, self.norm_b, self.w_in, self.w_out]

    def project(self, x):
        """q, k (of length 1), v, g, beta of each row of normalised features."""
        q, k, v, g, b = (x @ self.w_in).split(self.split, dim=1)
        k = F.normalize(k.reshape(-1, self.heads, self.dk), dim=2)
        return (q.reshape(k.shape).contiguous(), k.contiguous(), v.reshape(-1, self.heads, self.dv).contiguous(),
                -F.softplus(g - 2.0).contiguous(), torch.sigmoid(b).contiguous())

    @torch.no_grad()
    def act(self, features, memory, u, **filters):
        """One frame of every stream: (actions, their log-probabilities); the memory is updated."""
        x = ops.layer_norm(features, self.norm_w, self.norm_b)
        h = ops.delta_step(*self.project(x), memory)
        return ops.sample(h.flatten(1) @ self.w_out, u, **filters)

    def episode_logits(self, features, n: int):
        """[n frames' rows, stream by stream] logits of whole episodes, differentiable."""
        x = LayerNorm.apply(features, self.norm_w, self.norm_b)
        h = DeltaRule.apply(*self.project(x), n)
        return h.flatten(1) @ self.w_out

    def memory(self, n: int):
        return torch.zeros((n, self.heads, self.dk, self.dv), device="cuda")


def make(streams: int, frames: int, height: int = 40, width: int = 32, features: int = 32, actions: int = 6):
    """(net, policy, frames [T][streams][1][h][w])."""
    wl = synth.Workload(cid=71, streams=streams, frames=frames, h=height, w=width, convs=(40, 80), n_out=features)
    x = torch.from_numpy(synth.to_f32(synth.sprite_batch(wl))).cuda().unsqueeze(2).contiguous()
    net = ReuseNet(1, wl.h, wl.w, wl.convs, wl.n_out, streams, synth.net_weights(wl), fuse_first=False)
    return net, RecurrentPolicy(features, actions), x


def episode(net, policy, frames, u, wanted, lr: float = 0.05):
    """One episode and one update; returns (mean reward, actions, log-probabilities, loss)."""
    T, n = u.shape
    memory = policy.memory(n)
    feats = torch.empty((n, T, net.n_out), device="cuda")   # stream by stream, as sequences lie
    actions = torch.empty((T, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((T, n), device="cuda")
    for t in range(T):
        f = net.step(frames[t])
        feats[:, t] = f
        actions[t], logp[t] = policy.act(f, memory, u[t])
    reward = (actions == wanted).float()
    returns = reward - reward.mean()                        # of the frame's own action, against the mean

    rows = feats.reshape(n * T, -1).requires_grad_()
    taken = F.log_softmax(policy.episode_logits(rows, n), dim=1).gather(1, actions.t().reshape(-1, 1).long())
    loss = -(returns.t().reshape(-1, 1) * taken).sum() / (n * T)
    dparams = torch.autograd.grad(loss, [rows] + policy.params)

    dfeats = dparams[0].reshape(n, T, -1)
    grads = net.new_grads()
    for t in range(T):                                      # the caches of frame t again, for its gradient
        net.step(frames[t])
        net.backward(dfeats[:, t].contiguous(), grads, accumulate=t > 0)
    net.sgd_step(grads, lr)
    with torch.no_grad():
        for p, d in zip(policy.params, dparams[1:]):
            p -= lr * d
    return reward.mean(), actions, logp, loss.detach()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--streams", type=int, default=256)
    ap.add_argument("--frames", type=int, default=16)
    ap.add_argument("--episodes", type=int, default=5)
    ap.add_argument("--lr", type=float, default=2.0)
    args = ap.parse_args()
    net, policy, frames = make(args.streams, args.frames)
    gen = torch.Generator(device="cuda").manual_seed(1)
    wanted = torch.arange(args.streams, device="cuda", dtype=torch.int32) % 2
    for e in range(args.episodes):
        u = torch.rand((args.frames, args.streams), generator=gen, device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        reward, _, _, loss = episode(net, policy, frames, u, wanted, args.lr)
        torch.cuda.synchronize()
        ms = (time.perf_counter() - t0) * 1e3
        print(f"episode {e}: mean reward {reward.item():.3f}, {ms:.1f} ms, "
              f"{args.streams * args.frames / ms:.1f} K frames/s", flush=True)
    net.close()


if __name__ == "__main__":
    main()
