"""The short causal convolution, by sequences and by single tokens, and its gradients on the GPU against 64-bit references.

Tolerances (2-norm, relative).  pre is a chain of at most 5 roundings, silu's
exponential and reciprocal are an ulp each: below 16 x 2^-24 = 1e-6; 4e-6 is
asked for.  Weight gradients add up to 64 tokens in a row and then a tree, of
terms of random sign: 4e-6 as well.  A result rounded once to bfloat16 is within
2^-8 of it (half a step).  Windows are copies."""
import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 4e-6, BF16: 2.0 ** -8 + 4e-6}


def _inputs(tokens, channels, taps, n, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    return (randn(tokens, channels).to(dtype), 0.6 * randn(channels, taps), 0.2 * randn(channels),
            randn(n, taps - 1, channels).to(dtype), randn(tokens, channels).to(dtype), randn(n, taps - 1, channels).to(dtype))


def _reference(x, w, b, off, window, silu):
    """(out, last windows), differentiable in float64 arguments."""
    outs, finals = [], []
    taps = w.shape[1]
    for i in range(len(off) - 1):
        rows = torch.cat([window[i], x[off[i]:off[i + 1]]])
        m = off[i + 1] - off[i]
        pre = b + sum(rows[k:k + m] * w[:, k] for k in range(taps))
        outs.append(pre * torch.sigmoid(pre) if silu else pre)
        finals.append(rows[m:])
    return torch.cat(outs), torch.stack(finals)


def _check(x, w, b, window, dout, dfinal, off, silu=True, even=None, with_window=True, with_bias=True, with_dfinal=True):
    from paper_1909_05632_amd import ops
    dtype = x.dtype
    c = lambda t: t.cuda()  # noqa: E731
    seqs = dict(n=even) if even else dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    kw = dict(state=c(window) if with_window else None, silu=silu, **seqs)
    bias = c(b) if with_bias else None
    out, final = ops.causal_conv(c(x), c(w), bias, **kw)
    grads = ops.causal_conv_backward(c(dout), c(x), c(w), bias, dfinal=c(dfinal) if with_dfinal else None, **kw)
    leaves = [t.double().requires_grad_() for t in (x, w, b if with_bias else torch.zeros_like(b),
                                                     window if with_window else torch.zeros_like(window))]
    y, last = _reference(*leaves[:3], off, leaves[3], silu)
    assert out.dtype == dtype and R.rel(out, y) <= TOL[dtype]
    assert torch.equal(final.cpu(), last.detach().to(dtype))
    loss = (y * dout.double()).sum() + ((last * dfinal.double()).sum() if with_dfinal else 0)
    want = torch.autograd.grad(loss, leaves, allow_unused=True)
    for got, ref, name, tol in zip(grads, want, ("dx", "dweight", "dbias", "dstate"), (TOL[dtype], 4e-6, 4e-6, TOL[dtype])):
        ref = torch.zeros_like(got, dtype=torch.float64, device="cpu") if ref is None else ref
        assert R.rel(got, ref) <= tol, name
    return out, final, grads


def _cuts(tokens, n, seed):
    gen = torch.Generator().manual_seed(seed)
    return [0] + sorted(torch.randint(0, tokens + 1, (n - 1,), generator=gen).tolist()) + [tokens]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("taps", [1, 2, 3, 4])
@pytest.mark.parametrize("tokens,channels,n", [(1, 8, 1), (5, 1, 3), (70, 7, 9), (64, 80, 2), (133, 33, 40), (97, 520, 5),
                                               (1000, 256, 12), (33, 1032, 1), (3, 2050, 5)])
def test_ragged_sequences_and_gradients(tokens, channels, n, taps, dtype):
    args = _inputs(tokens, channels, taps, n, dtype, seed=taps)
    _check(*args, _cuts(tokens, n, seed=n), silu=taps != 3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,length,channels", [(1, 33, 16), (256, 16, 256), (64, 1, 72), (300, 2, 24), (40, 3, 9), (2, 4096, 64)])
def test_even_sequences(n, length, channels, dtype):
    args = _inputs(n * length, channels, 4, n, dtype, seed=n)
    off = [i * length for i in range(n + 1)]
    out, final, grads = _check(*args, off, even=n)
    again, last, same = _check(*args, off)
    assert torch.equal(out, again) and torch.equal(final, last) and all(torch.equal(a, b) for a, b in zip(grads, same))


@pytest.mark.parametrize("what", ["window", "bias", "dfinal"])
def test_without(what):
    args = _inputs(150, 40, 4, 6, F32, seed=2)
    _check(*args, _cuts(150, 6, seed=1), **{"with_" + what: False})


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_short_length_at_every_place_of_a_run(dtype):
    """Sequences of 0 to 5 tokens one after another: they begin and end everywhere around the runs' ends."""
    lengths = [(7 * i) % 6 for i in range(200)]
    off = [0]
    for m in lengths:
        off.append(off[-1] + m)
    _check(*_inputs(off[-1], 24, 4, len(lengths), dtype, seed=3), off)


def test_views_at_a_stride_and_odd_addresses():
    from paper_1909_05632_amd import ops
    for dtype in (F32, BF16):
        x, w, b, window, dout, dfinal = _inputs(90, 64, 4, 3, dtype, seed=5)
        off = [0, 40, 41, 90]
        out, final, grads = _check(x, w, b, window, dout, dfinal, off)
        so = torch.tensor(off, dtype=torch.int32).cuda()
        for at in (8, 3):
            view = torch.full((90, 200), 9.0, dtype=dtype, device="cuda")[:, at:at + 64]
            view.copy_(x)
            o2, f2 = ops.causal_conv(view, w.cuda(), b.cuda(), so, state=window.cuda())
            g2 = ops.causal_conv_backward(dout.cuda(), view, w.cuda(), b.cuda(), so, state=window.cuda(), dfinal=dfinal.cuda())
            assert R.rel(o2, out) <= TOL[dtype] and torch.equal(f2, final)
            assert all(R.rel(p, q) <= TOL[dtype] for p, q in zip(g2, grads))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("taps", [1, 2, 3, 4])
@pytest.mark.parametrize("channels", [1, 30, 64, 520])
def test_single_tokens_are_the_sequence(channels, taps, dtype):
    """Frame by frame, streams in slots of any order, one of them left out: the whole sequences' values, to
    the roundings of each (a bfloat16 result may lie on either side of an edge)."""
    from paper_1909_05632_amd import ops
    n, length = 5, 6
    x, w, b, window, _, _ = (t.cuda() for t in _inputs(n * length, channels, taps, n, dtype, seed=7))
    out, final = ops.causal_conv(x, w, b, n=n, state=window)
    pool = torch.full((9, taps - 1, channels), 3.0, dtype=dtype, device="cuda")
    ids = torch.tensor([4, 0, 8, 2, 6], dtype=torch.int32, device="cuda")
    pool[ids.long()] = window
    frames = x.view(n, length, channels)
    for t in range(length):
        y = ops.causal_conv_step(frames[:, t], w, pool, b, stream_ids=ids)
        assert R.rel(y, out.view(n, length, channels)[:, t]) <= TOL[dtype]
    assert torch.equal(pool[ids.long()], final) and (pool[[1, 3, 5, 7]] == 3).all()
    before = pool.clone()
    away = torch.tensor([9, -1, 8, 2, 6], dtype=torch.int32, device="cuda")
    y = frames[:, 0].contiguous()
    got = ops.causal_conv_step(y, w, pool, b, stream_ids=away, out=y)          # over x itself
    assert got is y and not y[:2].any() and torch.equal(pool[[0, 1, 3, 4, 5, 7]], before[[0, 1, 3, 4, 5, 7]])


def test_gradient_against_differences():
    x, w, b, window, dout, dfinal = _inputs(30, 6, 4, 3, F32, seed=9)
    off = [0, 2, 17, 30]
    _, _, grads = _check(x, w, b, window, dout, dfinal, off)
    gen = torch.Generator().manual_seed(1)
    e = 1e-5
    leaves = [t.double() for t in (x, w, b, window)]
    for _ in range(4):
        d = [torch.randn(t.shape, generator=gen).double() for t in leaves]
        vals = []
        for s in (1, -1):
            p = [t + s * e * q for t, q in zip(leaves, d)]
            y, last = _reference(*p[:3], off, p[3], True)
            vals.append((y * dout.double()).sum() + (last * dfinal.double()).sum())
        mine = sum((g.double().cpu() * q).sum() for g, q in zip(grads, d))
        size = sum(g.double().norm().item() * q.norm().item() for g, q in zip(grads, d))
        assert abs((vals[0] - vals[1]) / (2 * e) - mine) <= 5e-6 * size


def test_values_that_are_not_finite_stay_in_their_channel_and_sequence():
    from paper_1909_05632_amd import ops
    x, w, b, window, dout, _ = _inputs(60, 16, 4, 2, F32, seed=11)
    off = torch.tensor([0, 25, 60], dtype=torch.int32).cuda()
    out, final = ops.causal_conv(x.cuda(), w.cuda(), b.cuda(), off, state=window.cuda())
    x[10, 3], x[58, 5] = float("nan"), float("inf")
    o2, f2 = ops.causal_conv(x.cuda(), w.cuda(), b.cuda(), off, state=window.cuda())
    hit = torch.zeros(60, 16, dtype=torch.bool)
    hit[10:14, 3], hit[58:, 5] = True, True
    assert torch.equal(o2.cpu()[~hit], out.cpu()[~hit]) and not torch.isfinite(o2.cpu()[hit]).any()
    assert torch.isfinite(f2[0]).all() and f2[1, 1, 5] == float("inf")


def test_no_tokens_and_empty_sequences():
    from paper_1909_05632_amd import ops
    w, b = torch.randn(8, 4, device="cuda"), torch.randn(8, device="cuda")
    x, window = torch.empty(0, 8, device="cuda"), torch.randn(3, 3, 8, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    for kw in (dict(seq_off=off), dict(n=3)):
        out, final = ops.causal_conv(x, w, b, state=window, **kw)
        assert out.shape == (0, 8) and torch.equal(final, window)
        dx, dw, db, ds = ops.causal_conv_backward(out, x, w, b, state=window, dfinal=window, **kw)
        assert dx.shape == (0, 8) and not dw.any() and not db.any() and torch.equal(ds, window)
    assert ops.causal_conv(x, w, b, seq_off=off[:1])[1].shape == (0, 3, 8)
    dx, dw, db, ds = ops.causal_conv_backward(x, x, w, b, seq_off=off[:1])
    assert not dw.any() and not db.any() and ds.shape == (0, 3, 8)
    assert ops.causal_conv_step(x, w, window, b).shape == (0, 8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("channels", [24, 7])
def test_tokens_behind_the_last_sequence(channels, dtype):
    """A padded batch: the rows behind are left as they were, whatever they hold, and reach no result."""
    from paper_1909_05632_amd import ops
    for held, off in ((5, [0, 3, 5]), (70, [0, 40, 40, 70]), (0, [0, 0])):
        n = len(off) - 1
        x, w, b, window, dout, dfinal = _inputs(held, channels, 4, n, dtype, seed=held)
        want = _check(x, w, b, window, dout, dfinal, off) if held else None
        pad = torch.full((100, channels), float("nan"), dtype=dtype)
        px, pd = torch.cat([x, pad]).cuda(), torch.cat([dout, pad]).cuda()
        kw = dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda(), state=window.cuda())
        out = torch.full_like(px, 7.0)
        _, final = ops.causal_conv(px, w.cuda(), b.cuda(), out=out, **kw)
        dx, dw, db, ds = ops.causal_conv_backward(pd, px, w.cuda(), b.cuda(), dfinal=dfinal.cuda(), **kw)
        assert (out[held:] == 7).all()
        if want is None:
            assert torch.equal(final.cpu(), window) and torch.equal(ds.cpu(), dfinal) and not dw.any() and not db.any()
            continue
        assert R.rel(out[:held], want[0]) <= TOL[dtype] and torch.equal(final, want[1])
        for got, ref, tol in zip((dx[:held], dw, db, ds), want[2], (TOL[dtype], 4e-6, 4e-6, TOL[dtype])):
            assert R.rel(got, ref) <= tol


def test_other_stream_same_bits_and_in_a_graph():
    from paper_1909_05632_amd import ops
    x, w, b, window, dout, dfinal = (t.cuda() for t in _inputs(2100, 136, 4, 7, BF16, seed=13))
    off = torch.tensor(_cuts(2100, 7, 5), dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def all_of(**kw):
        out, final = ops.causal_conv(x, w, b, off, state=window, **kw)
        return [out, final, *ops.causal_conv_backward(dout, x, w, b, off, state=window, dfinal=dfinal, **kw)]

    want = all_of()
    for _ in range(3):
        got = all_of(stream=side)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        got = all_of()
    for _ in range(3):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_offsets_past_32_bits():
    """300000 tokens of 8192 channels in bfloat16 are 2.4e9 elements: the last tokens are as they are alone."""
    from paper_1909_05632_amd import ops
    tokens, channels = 300000, 8192
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(tokens, channels, dtype=BF16, device="cuda").normal_(generator=gen)
    w, b = torch.randn(channels, 4, generator=gen, device="cuda"), torch.randn(channels, generator=gen, device="cuda")
    out, final = ops.causal_conv(x, w, b, n=1)
    tail, last = ops.causal_conv(x[-100:], w, b, n=1, state=x[None, -103:-100].contiguous())
    assert torch.equal(out[-100:], tail) and torch.equal(final, last)
    dx, dw, db, _ = ops.causal_conv_backward(out, x, w, b, n=1, want_dstate=False)
    dx2, _, _, _ = ops.causal_conv_backward(out[-100:].contiguous(), x[-100:], w, b, n=1, state=x[None, -103:-100].contiguous())
    assert torch.equal(dx[-100:], dx2) and torch.isfinite(dw).all()
    del x, out, dx
    torch.cuda.empty_cache()


def test_more_blocks_than_a_grid_axis_holds_and_no_windows():
    """One block more than 2^20, whose grid is rounded up, in calls that want no last windows and no gradient of
    the first ones: the tokens around the last blocks and the first ones are as they are alone."""
    from paper_1909_05632_amd import binding as B
    from paper_1909_05632_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(2)
    # single elements, 8 lanes: 32 runs of 32 tokens a block
    tokens, ref = (1 << 30) + 1, ops.ctypes.byref
    x = torch.empty(tokens, 1, dtype=BF16, device="cuda").normal_(generator=gen)
    w, b = torch.randn(1, 4, generator=gen, device="cuda"), torch.randn(1, generator=gen, device="cuda")
    out = torch.full_like(x, 7.0)
    shape = ops.rn_conv_shape(1, 1, 4, tokens, B.RN_BF16, 1, 1)
    assert ops.load_ops().reuse_ops_causal_conv(ref(shape), x.data_ptr(), w.data_ptr(), b.data_ptr(), None, None, None,
                                                out.data_ptr(), torch.cuda.current_stream().cuda_stream) == B.RN_OK
    assert torch.equal(out[:5000], ops.causal_conv(x[:5000], w, b, n=1)[0])
    assert torch.equal(out[-5000:], ops.causal_conv(x[-5000:], w, b, n=1, state=x[None, -5003:-5000].contiguous())[0])
    del x, out
    # 33 channels, single elements, 64 lanes: 4 runs of 64 tokens a block
    tokens, channels = (1 << 28) + 1, 33
    x = torch.empty(tokens, channels, dtype=BF16, device="cuda").normal_(generator=gen)
    w, b = torch.randn(channels, 4, generator=gen, device="cuda"), torch.randn(channels, generator=gen, device="cuda")
    dx, dw, _, none = ops.causal_conv_backward(x, x, w, b, n=1, want_dstate=False)
    assert none is None and torch.isfinite(dw).all()
    head, tail = x[:5003].contiguous(), x[-5000:].contiguous()
    assert torch.equal(dx[:5000], ops.causal_conv_backward(head, head, w, b, n=1)[0][:5000])
    window = x[None, -5003:-5000].contiguous()
    assert torch.equal(dx[-5000:], ops.causal_conv_backward(tail, tail, w, b, n=1, state=window)[0])
    del x, dx
    torch.cuda.empty_cache()
