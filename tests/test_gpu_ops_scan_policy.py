"""The residual norm, the short convolution, the selective scan and the log-probabilities together, as
examples/recurrent_policy.py runs them: frames one by one against whole episodes, gradients against float64
automatic differentiation of the definition on the CPU, a run of the operators alone in a graph.

Tolerances.  Every quantity is a chain of float32 sums of at most 192 terms (2^-24 each): two norms, three
products, a convolution of 4 taps and a scan of T <= 12 tokens, each of them passed once forward and once
back.  Eight such steps of at most 192 terms stay below 8 * 192 * 2^-24 = 9.2e-5 of the largest magnitude
involved; the step sizes' exponentials multiply a scan's by at most 2: 2e-4 of max(1, largest) is asked for.
"""
import pytest
import torch
import torch.nn.functional as F

from tests import scan_ref as S
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

TOL = 2e-4


def _norm(x, w):
    return x / torch.sqrt(x.square().mean(1, keepdim=True) + 1e-5) * w


def _reference(policy, rows, off):
    """(logits, leaves) of whole episodes from the definition, float64, differentiable."""
    x = rows.detach().cpu().double().requires_grad_()
    leaves = [p.detach().cpu().double().requires_grad_() for p in policy.params]
    norm_w, out_w, w_in, w_mid, conv_w, conv_b, a_log, d, dt_bias, w_out = leaves
    u, z, dt, b, c = (_norm(x, norm_w) @ w_in).split(policy.split, dim=1)
    parts = []
    for lo, hi in zip(off, off[1:]):
        seq = F.pad(u[lo:hi], (0, 0, policy.taps - 1, 0))
        parts.append(conv_b + sum(seq[k:k + hi - lo] * conv_w[:, k] for k in range(policy.taps)))
    y, _ = S.scan(dict(u=F.silu(torch.cat(parts)), dt=dt, a=-a_log.exp(), b=b[:, None], c=c[:, None], d=d, z=z,
                       dt_bias=dt_bias, state=None), off)
    return _norm(x + y @ w_mid, out_w) @ w_out, [x] + leaves


def _check_gradients(policy, rows, off, logits, want, leaves):
    scale = max(1.0, want.abs().max().item())
    assert (logits.detach().cpu() - want).abs().max().item() <= TOL * scale
    dl = torch.randn(want.shape, generator=torch.Generator().manual_seed(4))
    grads = torch.autograd.grad(logits, [rows] + policy.params, dl.cuda())
    refs = torch.autograd.grad(want, leaves, dl.double())
    for i, (a, b) in enumerate(zip(grads, refs)):
        err = (a.cpu() - b).abs().max().item()
        assert err <= TOL * max(1.0, b.abs().max().item()), (i, err)
    return scale


def test_frames_and_episodes_agree():
    from examples import recurrent_policy as R
    n, T = 7, 5
    net, policy, frames = R.make(n, T, memory="scan")
    feats = torch.stack([net.step(frames[t]).clone() for t in range(T)], 1).reshape(n * T, -1)
    u = torch.rand((T, n), generator=torch.Generator().manual_seed(3)).cuda()
    memory = policy.memory(n)
    got = [policy.act(feats.view(n, T, -1)[:, t].contiguous(), memory, u[t]) for t in range(T)]
    actions = torch.stack([a for a, _ in got], 1).reshape(-1)
    logp = torch.stack([p for _, p in got], 1).reshape(-1)
    rows = feats.clone().requires_grad_()
    off = [i * T for i in range(n + 1)]
    logits = policy.episode_logits(rows, n)
    want, leaves = _reference(policy, rows, off)
    taken, entropy = R.LogProbs.apply(logits, actions)
    scale = _check_gradients(policy, rows, off, logits, want, leaves)
    logs = F.log_softmax(want, 1)
    for mine in (logp, taken.detach()):
        assert (logs.gather(1, actions.cpu().long()[:, None])[:, 0] - mine.cpu()).abs().max().item() <= 2 * TOL * scale
    assert (-(logs.exp() * logs).sum(1) - entropy.detach().cpu()).abs().max().item() <= 4 * TOL * scale
    net.close()


def test_episodes_of_any_length_and_their_gradients():
    from examples import recurrent_policy as R
    policy = R.ScanPolicy(32, 6)
    off = [0, 1, 1, 13, 15, 18]
    rows = torch.randn(18, 32, generator=torch.Generator().manual_seed(8)).cuda().requires_grad_()
    logits = policy.episode_logits(rows, seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    _check_gradients(policy, rows, off, logits, *_reference(policy, rows, off))


@pytest.mark.parametrize("memory", ["delta", "scan"])
def test_an_episode_runs(memory):
    from examples import recurrent_policy as R
    n, T = 8, 4
    net, policy, frames = R.make(n, T, memory=memory)
    before = [p.detach().clone() for p in policy.params]
    u = torch.rand((T, n), generator=torch.Generator().manual_seed(5)).cuda()
    reward, actions, logp, loss = R.episode(net, policy, frames, u, torch.zeros(n, device="cuda", dtype=torch.int32), 0.5, 0.01)
    assert actions.shape == (T, n) and (logp <= 0).all() and torch.isfinite(loss) and 0 <= reward <= 1
    assert all(torch.isfinite(p).all() for p in policy.params)
    assert sum(not torch.equal(p, q) for p, q in zip(policy.params, before)) >= len(before) - 1
    net.close()


def test_a_frame_in_a_graph():
    """A frame of every stream by the operators alone, captured once and replayed frame after frame."""
    from paper_1909_05632_amd import ops
    n, channels, states, T = 9, 32, 16, 6
    gen = torch.Generator().manual_seed(2)
    randn = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    frames, choices = randn(T, n, 3 * channels + 2 * states), torch.randint(0, channels, (T, n), generator=gen).int().cuda()
    w, w2, conv_w, conv_b, a = randn(frames.shape[2]), randn(channels), randn(channels, 4), randn(channels), -randn(channels, states).exp()

    def frame(x, choice, window, state):
        u, z, dt, b, c = ops.rms_norm(x, w).split([channels] * 3 + [states] * 2, dim=1)
        u = ops.causal_conv_step(u, conv_w, window, conv_b)
        y = ops.scan_step(u, dt, a, b.unsqueeze(1), c.unsqueeze(1), state, w2, z)
        y, total = ops.rms_norm(y, w2, x[:, :channels])
        return (*ops.log_probs(y, choice, top=3), total)

    memory = lambda: (torch.zeros(n, 3, channels, device="cuda"), torch.zeros(n, channels, states, device="cuda"))  # noqa: E731
    eager = memory()
    want = [[t.clone() for t in frame(frames[t], choices[t], *eager)] for t in range(T)]
    side = torch.cuda.Stream()
    held, x, choice = memory(), frames[0].clone(), choices[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = frame(x, choice, *held)
    for _ in range(2):                                   # two episodes from empty memories
        for t in held:
            t.zero_()
        for t in range(T):
            x.copy_(frames[t])
            choice.copy_(choices[t])
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want[t])), t
        assert all(torch.equal(p, q) for p, q in zip(held, eager))


def test_slots_past_32_bits():
    """Pools of more than 2^31 elements: the last slots are stepped as those of a small pool are."""
    from paper_1909_05632_amd import ops
    n, channels, states, slots = 3, 4096, 16, 34000
    gen = torch.Generator().manual_seed(6)
    randn = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    x, conv_w, a, b = randn(n, channels), randn(channels, 4), -randn(channels, states).exp(), randn(n, 1, states)
    far = torch.tensor([slots - 1, 0, slots - 2], dtype=torch.int32).cuda()
    state, window = randn(n, channels, states), randn(n, 3, channels)
    pool = torch.empty(slots, channels, states, device="cuda")
    windows = torch.empty(6 * slots, 3, channels, device="cuda")
    assert pool.numel() > 2 ** 31 and windows.numel() > 2 ** 31
    wide = torch.tensor([6 * slots - 1, 0, 6 * slots - 2], dtype=torch.int32).cuda()
    pool[far.long()], windows[wide.long()] = state, window
    want = ops.causal_conv_step(x, conv_w, window), ops.scan_step(x, x, a, b, b, state)
    got = ops.causal_conv_step(x, conv_w, windows, stream_ids=wide), ops.scan_step(x, x, a, b, b, pool, stream_ids=far)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(pool[far.long()], state) and torch.equal(windows[wide.long()], window)
    del pool, windows
    torch.cuda.empty_cache()
