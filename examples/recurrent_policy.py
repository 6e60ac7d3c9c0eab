"""A policy with a memory over many streams, trained with REINFORCE on the device.

Each frame of a stream goes through a reuse net, whose outputs serve as features;
they are normalised and projected to a query, a key, a value, a decay and a write
strength; the stream's memory is read and written by the gated delta rule; and an
action is drawn from logits formed of what was read.  (With --memory scan, the memory
is a convolution's window and a selective scan's state instead, in a block beside the
features.)  After an episode the same
frames' features go through the operators as whole sequences, the gradients come
back through them to the features, and the frames are replayed through the net,
whose backward pass takes them over.

    python -m examples.recurrent_policy --streams 256 --frames 16 --episodes 5 --memory scan

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


class RmsNorm(torch.autograd.Function):
    """The norm of x, or of x + residual, which is then the second result."""

    @staticmethod
    def forward(ctx, x, weight, residual=None):
        got = ops.rms_norm(x, weight, residual, with_stats=True)
        ctx.save_for_backward(x if residual is None else got[1], weight, got[-1])
        ctx.sum = residual is not None
        return got[:2] if ctx.sum else got[0]

    @staticmethod
    def backward(ctx, dy, dtotal=None):
        total, weight, stats = ctx.saved_tensors
        if dtotal is not None:
            dtotal = dtotal.contiguous()
        dx, dweight = ops.rms_norm_backward(dy.contiguous(), total, weight, stats, dtotal)
        return dx, dweight, dx if ctx.sum else None


class CausalConv(torch.autograd.Function):
    """All tokens of sequences (seq_off, or n of one length), from empty windows."""

    @staticmethod
    def forward(ctx, x, weight, bias, seq_off, n):
        ctx.save_for_backward(x, weight, bias, seq_off)
        ctx.n = n
        return ops.causal_conv(x, weight, bias, seq_off, n)[0]

    @staticmethod
    def backward(ctx, dout):
        x, weight, bias, seq_off = ctx.saved_tensors
        grads = ops.causal_conv_backward(dout.contiguous(), x, weight, bias, seq_off, ctx.n, want_dstate=False)
        return (*grads[:3], None, None)


class Scan(torch.autograd.Function):
    """All tokens of sequences (seq_off, or n of one length), from empty states."""

    @staticmethod
    def forward(ctx, u, dt, a, b, c, d, z, dt_bias, seq_off, n):
        out, _, saved = ops.scan_forward(u, dt, a, b, c, d, z, dt_bias, seq_off=seq_off, n=n, save=True)
        ctx.save_for_backward(u, dt, a, b, c, d, z, dt_bias, seq_off, saved)
        ctx.n = n
        return out

    @staticmethod
    def backward(ctx, dout):
        *inputs, seq_off, saved = ctx.saved_tensors
        grads = ops.scan_backward(dout.contiguous(), *inputs, seq_off=seq_off, n=ctx.n, saved=saved, want_dstate=False)
        return (*grads[:8], None, None)


class LogProbs(torch.autograd.Function):
    """Log-probabilities of the actions that were taken, and the entropy of what they were drawn from."""

    @staticmethod
    def forward(ctx, logits, actions):
        taken, entropy, stats = ops.log_probs(logits, actions, with_stats=True)
        ctx.save_for_backward(logits, actions, stats)
        return taken, entropy

    @staticmethod
    def backward(ctx, dtaken, dentropy):
        logits, actions, stats = ctx.saved_tensors
        return ops.log_probs_backward(dtaken.contiguous(), dentropy.contiguous(), logits, actions, stats), None


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


class ScanPolicy:
    """Features [rows][width] to logits [rows][actions]; a stream keeps a window and a state between frames.

    A block: the features' norm, projected to an input, a gate, step sizes, b and c;
    the input through a short convolution and the scan; what that gives, projected
    back, beside the features."""

    def __init__(self, width: int, actions: int, channels: int = 64, states: int = 16, taps: int = 4, seed: int = 0):
        gen = torch.Generator().manual_seed(seed)

        def param(*shape, std=None):
            x = torch.zeros(shape) if std is None else torch.randn(shape, generator=gen) * std
            return x.cuda().requires_grad_()

        self.channels, self.states, self.taps = channels, states, taps
        self.split = [channels, channels, channels, states, states]
        self.norm_w, self.out_norm_w = (torch.ones(width).cuda().requires_grad_() for _ in range(2))
        self.w_in, self.w_mid = param(width, sum(self.split), std=width ** -0.5), param(channels, width, std=channels ** -0.5)
        self.conv_w, self.conv_b = param(channels, taps, std=taps ** -0.5), param(channels)
        self.a_log = torch.arange(1, states + 1).float().log().repeat(channels, 1).cuda().requires_grad_()
        self.d, self.dt_bias = torch.ones(channels).cuda().requires_grad_(), torch.full((channels,), -2.0).cuda().requires_grad_()
        self.w_out = param(width, actions, std=width ** -0.5)
        self.params = [self.norm_w, self.out_norm_w, self.w_in, self.w_mid, self.conv_w, self.conv_b, self.a_log, self.d,
                       self.dt_bias, self.w_out]

    def project(self, x):
        """u, z, dt, b, c of each row of normalised features: views of one product."""
        u, z, dt, b, c = (x @ self.w_in).split(self.split, dim=1)
        return u, z, dt, b.unsqueeze(1), c.unsqueeze(1)

    @torch.no_grad()
    def act(self, features, memory, u, **filters):
        """One frame of every stream: (actions, their log-probabilities); the memory is updated."""
        window, state = memory
        x, z, dt, b, c = self.project(ops.rms_norm(features, self.norm_w))
        x = ops.causal_conv_step(x, self.conv_w, window, self.conv_b)
        y = ops.scan_step(x, dt, -self.a_log.exp(), b, c, state, self.d, z, self.dt_bias)
        y, _ = ops.rms_norm(y @ self.w_mid, self.out_norm_w, features)
        return ops.sample(y @ self.w_out, u, **filters)

    def episode_logits(self, features, n=None, seq_off=None):
        """Logits of whole episodes' rows, stream by stream (n of one length, or as seq_off says), differentiable."""
        x, z, dt, b, c = self.project(RmsNorm.apply(features, self.norm_w))
        x = CausalConv.apply(x, self.conv_w, self.conv_b, seq_off, n)
        y = Scan.apply(x, dt, -self.a_log.exp(), b, c, self.d, z, self.dt_bias, seq_off, n)
        y, _ = RmsNorm.apply(y @ self.w_mid, self.out_norm_w, features)
        return y @ self.w_out

    def memory(self, n: int):
        return (torch.zeros((n, self.taps - 1, self.channels), device="cuda"),
                torch.zeros((n, self.channels, self.states), device="cuda"))


POLICIES = {"delta": RecurrentPolicy, "scan": ScanPolicy}


def make(streams: int, frames: int, height: int = 40, width: int = 32, features: int = 32, actions: int = 6,
         memory: str = "delta"):
    """(net, policy, frames [T][streams][1][h][w])."""
    wl = synth.Workload(cid=71, streams=streams, frames=frames, h=height, w=width, convs=(40, 80), n_out=features)
    x = torch.from_numpy(synth.to_f32(synth.sprite_batch(wl))).cuda().unsqueeze(2).contiguous()
    net = ReuseNet(1, wl.h, wl.w, wl.convs, wl.n_out, streams, synth.net_weights(wl), fuse_first=False)
    return net, POLICIES[memory](features, actions), x


def episode(net, policy, frames, u, wanted, lr: float = 0.05, entropy: float = 0.0):
    """One episode and one update, which `entropy` times the mean entropy is added to; returns (mean reward,
    actions, log-probabilities, loss)."""
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
    taken, spread = LogProbs.apply(policy.episode_logits(rows, n), actions.t().reshape(-1))
    loss = -(returns.t().reshape(-1) * taken + entropy * spread).sum() / (n * T)
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
    ap.add_argument("--memory", choices=sorted(POLICIES), default="delta")
    ap.add_argument("--entropy", type=float, default=0.0)
    args = ap.parse_args()
    net, policy, frames = make(args.streams, args.frames, memory=args.memory)
    gen = torch.Generator(device="cuda").manual_seed(1)
    wanted = torch.arange(args.streams, device="cuda", dtype=torch.int32) % 2
    for e in range(args.episodes):
        u = torch.rand((args.frames, args.streams), generator=gen, device="cuda")
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        reward, _, _, loss = episode(net, policy, frames, u, wanted, args.lr, args.entropy)
        torch.cuda.synchronize()
        ms = (time.perf_counter() - t0) * 1e3
        print(f"episode {e}: mean reward {reward.item():.3f}, {ms:.1f} ms, "
              f"{args.streams * args.frames / ms:.1f} K frames/s", flush=True)
    net.close()


if __name__ == "__main__":
    main()
