"""The gated delta rule on the GPU against its recurrence in 64 bits.

Tolerances (2-norm, relative).  float32: a result passes through about five
products of up to 128 terms and the chunk's triangular solve; their roundings
of 2^-24 add up like sqrt(5 x 128) of them, 1.5e-6, and four times that is
allowed, 6e-6; the gradients of g and beta, differences of larger sums, get
2e-5.  bfloat16 inputs are exact, so float32 results keep those bounds, and
bfloat16 results are within their own rounding, 2^-9 each."""
import math

import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 6e-6, BF16: 2.0 ** -9 + 6e-6}
TOL_G = 2e-5


def _inputs(lengths, hk, hv, dk, dv, dtype, seed=0, near=0.5, decay=(1e-3, 1.0)):
    gen = torch.Generator().manual_seed(seed)
    n, tokens = len(lengths), sum(lengths)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    base = randn(1, hk, dk)
    k, q = near * base + randn(tokens, hk, dk), near * base + randn(tokens, hk, dk)
    x = dict(q=(q / q.norm(dim=-1, keepdim=True)).to(dtype), k=(k / k.norm(dim=-1, keepdim=True)).to(dtype),
             v=randn(tokens, hv, dv).to(dtype))
    lo, hi = (math.log(d) for d in decay)
    x["g"] = -torch.exp(lo + (hi - lo) * torch.rand(tokens, hv, generator=gen))
    x["beta"] = torch.sigmoid(randn(tokens, hv))
    x["state"] = 0.2 * randn(n, hv, dk, dv)
    x["dout"] = randn(tokens, hv, dv).to(dtype)
    x["dfinal"] = 0.2 * randn(n, hv, dk, dv)
    off = [0]
    for m in lengths:
        off.append(off[-1] + m)
    return x, off


NAMES = ("q", "k", "v", "g", "beta")


def _reference(x, off, scale, grads=True, state=True):
    a = {k: v.double().requires_grad_(grads) for k, v in x.items() if k in NAMES + ("state",)}
    s0 = a["state"] if state else torch.zeros_like(a["state"])
    out, final = R.delta(*(a[k] for k in NAMES), off, s0, scale)
    if not grads:
        return out, final, None
    ((out * x["dout"].double()).sum() + (final * x["dfinal"].double()).sum()).backward()
    return out.detach(), final.detach(), {k: (t.grad if t.grad is not None else torch.zeros_like(t)) for k, t in a.items()}


def _run(x, off, scale, **kw):
    from paper_1909_05632_amd import ops
    d = {k: v.cuda() for k, v in x.items()}
    so = torch.tensor(off, dtype=torch.int32).cuda()
    args = [d[k] for k in NAMES] + [so]
    out, final, saved = ops.delta_forward(*args, state=d["state"], scale=scale, save=True, **kw)
    grads = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=scale)
    return out, final, grads


def _compare(x, off, scale, label=""):
    out, final, grads = _run(x, off, scale)
    want, last, g = _reference(x, off, scale)
    dtype = x["q"].dtype
    bounds = (TOL[dtype],) * 3 + (TOL_G, TOL_G, TOL[F32])
    errors = {"out": (R.rel(out, want), TOL[dtype]), "final": (R.rel(final, last), TOL[F32])}
    for got, name, tol in zip(grads, NAMES + ("state",), bounds):
        errors["d" + name] = (R.rel(got, g[name]), tol)
    bad = {k: v for k, v in errors.items() if not v[0] <= v[1]}
    assert not bad, (label, bad)
    assert out.dtype == dtype and final.dtype == F32 and grads[0].dtype == dtype and grads[3].dtype == F32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths", [[1], [16, 16, 16], [64], [65], [0, 1, 63, 0, 64, 130, 2], [200, 5]])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 1, 64, 64), (2, 4, 32, 40), (1, 3, 128, 128), (2, 2, 100, 90)])
def test_sequences_and_gradients(lengths, hk, hv, dk, dv, dtype):
    x, off = _inputs(lengths, hk, hv, dk, dv, dtype)
    _compare(x, off, dk ** -0.5)


@pytest.mark.parametrize("dk,dv", [(1, 1), (1, 17), (3, 5), (16, 16), (17, 16), (33, 128), (72, 7), (128, 1), (127, 65)])
def test_odd_head_sizes(dk, dv):
    for dtype in (F32, BF16):
        x, off = _inputs([70, 3], 2, 2, dk, dv, dtype, seed=dk + dv)
        _compare(x, off, 0.3, (dk, dv, dtype))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 2, 128, 128), (2, 2, 64, 70), (1, 1, 20, 16)])
@pytest.mark.parametrize("lengths", [[3] * 11, [32, 33, 1, 0, 31, 2, 70, 5, 9, 4], [31, 1], [20]])
def test_short_and_long_sequences_in_one_call(lengths, hk, hv, dk, dv, dtype):
    """Sequences up to 32 tokens may go another way than longer ones; both in one batch."""
    x, off = _inputs(lengths, hk, hv, dk, dv, dtype, seed=len(lengths))
    _compare(x, off, dk ** -0.5, lengths)


def test_long_sequence_of_near_equal_keys():
    """Frames that hardly change: keys almost parallel, so the triangular systems are far from the identity."""
    x, off = _inputs([600], 1, 2, 64, 64, F32, near=8.0, decay=(1e-4, 1e-2))
    _compare(x, off, 0.125)


def test_strong_decay_keeps_far_differences():
    """Sums of g grow to thousands within a chunk; neighbours' decays stay exact."""
    x, off = _inputs([150], 1, 2, 32, 32, F32, decay=(20.0, 60.0))
    x["g"][::2] = -1e-3
    _compare(x, off, 0.2)


def test_memory_emptied_between_episodes():
    """g = -infinity at an episode's first token is a sequence of its own with a memory of zeros."""
    from paper_1909_05632_amd import ops
    for first in (30, 64):
        x, off = _inputs([150], 1, 2, 64, 48, F32)
        x["g"][first] = -math.inf
        out, final, grads = _run(x, off, 0.2)
        split = {k: v.clone() for k, v in x.items()}
        split["g"][first] = 0.0
        split["state"] = torch.cat([x["state"], torch.zeros_like(x["state"])])
        split["dfinal"] = torch.cat([torch.zeros_like(x["dfinal"]), x["dfinal"]])
        want, last, g = _reference(split, [0, first, 150], 0.2)
        assert R.rel(out, want) <= TOL[F32] and R.rel(final[0], last[1]) <= TOL[F32]
        for got, name, tol in zip(grads, NAMES, (TOL[F32],) * 3 + (TOL_G, TOL_G)):
            a, b = got.double().cpu(), g[name].clone()
            if name == "g":
                assert a[first].abs().max() <= TOL_G * b.norm() and torch.isfinite(a).all()
                a[first] = b[first] = 0.0
            assert R.rel(a, b) <= tol, (first, name)
        assert R.rel(grads[5][0], g["state"][0]) <= TOL[F32]
        step_state = x["state"].cuda()
        ops.delta_step(*(x[k][first:first + 1].cuda() for k in NAMES), step_state, scale=0.2)
        held = x["beta"][first].double()[:, None, None] * x["k"][first].double().repeat_interleave(2, 0)[:, :, None]
        assert R.rel(step_state[0], held * x["v"][first].double()[:, None, :]) <= TOL[F32]


def test_gradients_against_differences():
    x, off = _inputs([40, 70], 1, 2, 24, 20, F32, seed=9)
    scale = 0.2
    _, _, grads = _run(x, off, scale)
    gen = torch.Generator().manual_seed(1)
    names = NAMES + ("state",)
    h = 1e-6
    for _ in range(3):
        d = {k: torch.randn(x[k].shape, generator=gen).double() for k in names}
        val = []
        for s in (1, -1):
            y = {k: x[k].double() + s * h * d[k] for k in names}
            out, final = R.delta(*(y[k] for k in NAMES), off, y["state"], scale)
            val.append((out * x["dout"].double()).sum() + (final * x["dfinal"].double()).sum())
        mine = sum((g.double().cpu() * d[k]).sum() for g, k in zip(grads, names))
        size = sum(g.double().norm().item() * d[k].norm().item() for g, k in zip(grads, names))
        assert abs((val[0] - val[1]) / (2 * h) - mine) <= 2e-5 * size


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,hk,hv,dk,dv", [(1, 2, 4, 64, 64), (7, 1, 2, 128, 128), (5, 3, 3, 100, 90), (4, 1, 1, 1, 1),
                                           (3, 2, 2, 33, 127), (2, 1, 4, 16, 4)])
def test_step_is_a_sequence_of_one(n, hk, hv, dk, dv, dtype):
    from paper_1909_05632_amd import ops
    x, off = _inputs([1] * n, hk, hv, dk, dv, dtype, seed=n)
    want, last, _ = _reference(x, off, 0.3, grads=False)
    pool = torch.randn(n + 3, hv, dk, dv, generator=torch.Generator().manual_seed(2)).cuda()
    ids = torch.randperm(n + 3, generator=torch.Generator().manual_seed(3))[:n].int()
    before = pool.clone()
    pool[ids.long()] = x["state"].cuda()
    out = ops.delta_step(*(x[k].cuda() for k in NAMES), pool, stream_ids=ids.cuda(), scale=0.3)
    assert out.dtype == dtype and R.rel(out, want) <= TOL[dtype] and R.rel(pool[ids.long()], last) <= TOL[F32]
    rest = [i for i in range(n + 3) if i not in ids.tolist()]
    assert torch.equal(pool[rest], before[rest])


def test_steps_and_sequences_agree():
    """A stream taken frame by frame holds the memory that the whole sequence gives."""
    from paper_1909_05632_amd import ops
    x, off = _inputs([90], 2, 2, 64, 64, F32)
    d = {k: v.cuda() for k, v in x.items()}
    out, final, _ = _run(x, off, 0.125)
    state, outs = d["state"].clone(), []
    for t in range(90):
        outs.append(ops.delta_step(*(d[k][t:t + 1] for k in NAMES), state, scale=0.125))
    assert R.rel(torch.cat(outs), out) <= 2 * TOL[F32] and R.rel(state, final) <= 2 * TOL[F32]


def test_ids_outside_the_pool_are_left_out():
    from paper_1909_05632_amd import ops
    x, _ = _inputs([1] * 4, 1, 1, 32, 32, F32)
    d = {k: v.cuda() for k, v in x.items()}
    pool = d["state"].clone()
    out = ops.delta_step(*(d[k] for k in NAMES), pool, stream_ids=torch.tensor([1, -1, 9, 0], dtype=torch.int32).cuda())
    assert not out[1:3].any() and out[0].any() and out[3].any()
    assert torch.equal(pool[2:], d["state"][2:]) and not torch.equal(pool[:2], d["state"][:2])


def test_tokens_at_a_stride_and_even_sequences():
    """q, k and v as views of one projection; n sequences of the same length without offsets."""
    from paper_1909_05632_amd import ops
    for dtype in (F32, BF16):
        x, off = _inputs([20] * 6, 2, 4, 48, 32, dtype)
        want, last, grads = _run(x, off, 0.2)
        d = {k: v.cuda() for k, v in x.items()}
        for pad in (0, 3):                           # 3: rows off every alignment
            joint = torch.zeros(120, 2 * 48 * 2 + 4 * 32 + pad, dtype=dtype, device="cuda")
            q, k, v = joint[:, :96], joint[:, 96:192], joint[:, 192 + pad:]
            q, k, v = q.unflatten(1, (2, 48)), k.unflatten(1, (2, 48)), v.unflatten(1, (4, 32))
            q.copy_(d["q"]), k.copy_(d["k"]), v.copy_(d["v"])
            out, final, saved = ops.delta_forward(q, k, v, d["g"], d["beta"], n=6, state=d["state"], scale=0.2, save=True)
            got = ops.delta_backward(d["dout"], q, k, v, d["g"], d["beta"], n=6, saved=saved, dfinal=d["dfinal"], scale=0.2)
            tol = 2 * TOL[dtype]
            assert R.rel(out, want) <= tol and R.rel(final, last) <= 2 * TOL[F32]
            for a, b in zip(got, grads):
                assert R.rel(a, b) <= (tol if a.dtype == dtype else 2 * TOL_G)


def test_first_and_last_memories_are_optional():
    from paper_1909_05632_amd import ops
    x, off = _inputs([33, 0, 70], 1, 2, 64, 64, F32)
    x["state"].zero_()
    want, last, grads = _run(x, off, 0.125)
    d = {k: v.cuda() for k, v in x.items()}
    so = torch.tensor(off, dtype=torch.int32).cuda()
    args = [d[k] for k in NAMES] + [so]
    out, final = ops.delta_forward(*args, scale=0.125)                    # no state, nothing saved
    assert torch.equal(out, want) and torch.equal(final, last)
    mem = d["state"].clone()
    out, final = ops.delta_forward(*args, state=mem, final=mem, scale=0.125)
    assert final is mem and torch.equal(out, want) and torch.equal(mem, last)
    _, _, saved = ops.delta_forward(*args, scale=0.125, save=True)
    a = ops.delta_backward(d["dout"], *args, saved=saved, scale=0.125, want_dstate=False)
    b = ops.delta_backward(d["dout"], *args, saved=saved, scale=0.125, dfinal=torch.zeros_like(d["state"]))
    assert a[5] is None and all(torch.equal(u, w) for u, w in zip(a[:5], b[:5]))


def test_no_tokens():
    from paper_1909_05632_amd import ops
    x, _ = _inputs([], 1, 2, 16, 16, F32)
    d = {k: v.cuda() for k, v in x.items()}
    state = torch.randn(3, 2, 16, 16, device="cuda")
    args = [d[k] for k in NAMES] + [torch.zeros(4, dtype=torch.int32, device="cuda")]
    out, final, saved = ops.delta_forward(*args, state=state, save=True)
    assert out.shape == (0, 2, 16) and torch.equal(final, state)
    grads = ops.delta_backward(out, *args, saved=saved, dfinal=state)
    assert torch.equal(grads[5], state) and grads[0].shape == (0, 1, 16)
    args[5] = args[5][:1]
    out, final = ops.delta_forward(*args)
    assert final.shape == (0, 2, 16, 16)
    assert ops.delta_step(*(d[k] for k in NAMES), state).shape == (0, 2, 16)


def test_sequences_do_not_touch_each_other():
    """A sequence of NaN leaves the others' bits alone, also where chunks of both share a block of tokens."""
    x, off = _inputs([40, 30, 90], 1, 2, 64, 64, F32)
    out, final, grads = _run(x, off, 0.125)
    bad = {k: v.clone() for k, v in x.items()}
    for k in ("q", "k", "v", "g", "beta", "dout"):
        bad[k][40:70] = math.nan
    out2, final2, grads2 = _run(bad, off, 0.125)
    keep = list(range(40)) + list(range(70, 160))
    assert torch.equal(out2[keep], out[keep]) and torch.equal(final2[[0, 2]], final[[0, 2]])
    for a, b in zip(grads2[:5], grads[:5]):
        assert torch.equal(a[keep], b[keep])
    assert torch.equal(grads2[5][[0, 2]], grads[5][[0, 2]]) and out2[40:70].isnan().all()


def test_bits_repeat_on_another_stream_and_in_a_graph():
    from paper_1909_05632_amd import ops
    x, off = _inputs([100, 28], 2, 4, 64, 64, BF16)
    want, last, grads = _run(x, off, 0.125)
    d = {k: v.cuda() for k, v in x.items()}
    so = torch.tensor(off, dtype=torch.int32).cuda()
    args = [d[k] for k in NAMES] + [so]
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    out, final, saved = ops.delta_forward(*args, state=d["state"], scale=0.125, save=True, stream=st)
    got = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=0.125, stream=st)
    st.synchronize()
    assert torch.equal(out, want) and torch.equal(final, last) and all(torch.equal(a, b) for a, b in zip(got, grads))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        out, final, saved = ops.delta_forward(*args, state=d["state"], scale=0.125, save=True)
        got = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=0.125)
    for _ in range(3):
        for t in (out, final, *got):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(final, last)
        assert all(torch.equal(a, b) for a, b in zip(got, grads))
