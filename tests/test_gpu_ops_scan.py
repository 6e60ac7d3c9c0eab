"""The selective scan, by sequences and by single tokens, and its gradients on the GPU against 64-bit references.

Tolerances (2-norm, relative).  A token's decay is off by at most two roundings
of its exponent's product (0.37 2^-24 each of the result) and an ulp, and the
state by one more: below 2^-23.  Of T <= 1000 tokens' errors of random sign the
state keeps at most sqrt(T) = 32, 4e-6; a gradient passes through the states and
through the walk back, and sums over tokens and channels add a few roundings: 2e-5
is asked for.  A result rounded once to bfloat16 is within 2^-8 of it (half a
step)."""
import pytest
import torch

from tests import ops_ref as R
from tests import scan_ref as S
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 2e-5, BF16: 2.0 ** -8 + 2e-5}
WIDE = ("a", "d", "dt_bias", "state")          # float32 whatever the data


def _cuda(x):
    return {k: None if v is None else v.cuda() for k, v in x.items()}


def _run(x, dout, dfinal, softplus=True, **seqs):
    """(out, final, gradients by name) of the kernels."""
    from paper_1909_05632_amd import ops
    g = _cuda(x)
    state = g.pop("state")
    out, final, saved = ops.scan_forward(**g, softplus=softplus, state=state, save=True, **seqs)
    o2, f2 = ops.scan_forward(**g, softplus=softplus, state=state, **seqs)
    assert all(torch.equal(torch.nan_to_num(p), torch.nan_to_num(q)) for p, q in ((o2, out), (f2, final)))
    grads = ops.scan_backward(dout.cuda(), **g, softplus=softplus, saved=saved,
                              dfinal=None if dfinal is None else dfinal.cuda(), **seqs)
    return out, final, dict(zip(S.GRADS, grads))


def _check(x, dout, dfinal, off, softplus=True, even=None):
    seqs = dict(n=even) if even else dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    out, final, grads = _run(x, dout, dfinal, softplus, **seqs)
    dtype = x["u"].dtype
    leaves = {k: None if v is None else v.double().requires_grad_() for k, v in x.items()}
    y, last = S.scan(leaves, off, softplus)
    assert out.dtype == dtype and R.rel(out, y) <= TOL[dtype]
    assert R.rel(final, last) <= TOL[F32]
    loss = (y * dout.double()).sum() + (0 if dfinal is None else (last * dfinal.double()).sum())
    there = [k for k in S.NAMES if leaves[k] is not None]
    want = dict(zip(there, torch.autograd.grad(loss, [leaves[k] for k in there], allow_unused=True)))
    for k in S.NAMES:
        got = grads["d" + k]
        if k == "state":
            ref = torch.zeros_like(got, dtype=torch.float64, device="cpu") if want.get(k) is None and x[k] is not None else want.get(k)
            if ref is None:
                continue
        elif x[k] is None:
            assert got is None, k
            continue
        else:
            ref = torch.zeros_like(x[k], dtype=torch.float64) if want[k] is None else want[k]
        assert got.dtype == (F32 if k in WIDE else dtype)
        assert R.rel(got, ref) <= (TOL[F32] if k in WIDE else TOL[dtype]), k
    return out, final, grads


def _cuts(tokens, n, seed):
    gen = torch.Generator().manual_seed(seed)
    return [0] + sorted(torch.randint(0, tokens + 1, (n - 1,), generator=gen).tolist()) + [tokens]


# Around every change of lanes (4, 8, 16, 32, 64 states), blocks of channels that
# are not full, groups, sequences shorter and longer than a tile.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens,channels,states,groups,n", [
    (1, 1, 1, 1, 1), (7, 3, 2, 1, 2), (40, 260, 4, 1, 3), (33, 20, 5, 2, 4), (50, 130, 8, 1, 2), (64, 66, 9, 3, 3),
    (90, 70, 16, 1, 5), (35, 128, 16, 2, 1), (31, 7, 13, 1, 6), (45, 36, 17, 1, 2), (50, 40, 32, 2, 3), (37, 18, 33, 1, 2),
    (60, 40, 64, 1, 4), (20, 24, 64, 3, 1), (100, 1, 16, 1, 9)])
def test_ragged_sequences_and_gradients(tokens, channels, states, groups, n, dtype):
    x, dout, dfinal = S.inputs(tokens, channels, states, groups, n, dtype, seed=tokens)
    _check(x, dout, dfinal, _cuts(tokens, n, seed=n))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens,channels,states,n", [(700, 12, 16, 1), (900, 5, 4, 3), (600, 9, 40, 2), (1000, 6, 7, 4)])
def test_long_sequences_in_chunks(tokens, channels, states, n, dtype):
    """Few channels: sequences are cut into chunks, some ending inside a tile, some sequences within one."""
    x, dout, dfinal = S.inputs(tokens, channels, states, 1, n, dtype, seed=tokens)
    _check(x, dout, dfinal, _cuts(tokens, n, seed=3))


@pytest.mark.parametrize("n,length", [(3, 256), (2, 257), (2, 300), (1, 512), (1, 513)])
def test_lengths_around_a_chunk(n, length):
    x, dout, dfinal = S.inputs(n * length, 10, 16, 1, n, F32, seed=length)
    off = [i * length for i in range(n + 1)]
    out, final, grads = _check(x, dout, dfinal, off, even=n)
    again = _run(x, dout, dfinal, seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    assert R.rel(again[0], out) <= TOL[F32] and all(R.rel(again[2][k], grads[k]) <= TOL[F32] for k in S.GRADS)


@pytest.mark.parametrize("what", ["d", "z", "dt_bias", "state", "dfinal", "softplus"])
@pytest.mark.parametrize("tokens", [40, 600])
def test_without(what, tokens):
    softplus = what != "softplus"
    x, dout, dfinal = S.inputs(tokens, 24, 16, 2, 3, F32, seed=2, softplus=softplus)
    if what in x:
        x[what] = None
        if what == "dt_bias":
            x["dt"] = x["dt"] - 3
    _check(x, dout, None if what == "dfinal" else dfinal, _cuts(tokens, 3, seed=1), softplus)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_every_short_length(dtype):
    lengths = [(5 * i) % 19 for i in range(60)]
    off = [0]
    for m in lengths:
        off.append(off[-1] + m)
    x, dout, dfinal = S.inputs(off[-1], 12, 16, 1, len(lengths), dtype, seed=3)
    _check(x, dout, dfinal, off)


@pytest.mark.parametrize("n,length,channels,states", [(256, 16, 64, 16), (1200, 2, 128, 16), (300, 3, 1040, 60), (2500, 1, 260, 4)])
def test_many_sequences(n, length, channels, states):
    """More sequences than there are blocks to walk them: each block has several, and sums over them."""
    x, dout, dfinal = S.inputs(n * length, channels, states, 1, n, F32, seed=n)
    out, final, grads = _run(x, dout, dfinal, n=n)
    leaves = {k: v.double().requires_grad_() for k, v in x.items()}
    y, last = S.scan_even(leaves, n)
    assert R.rel(out, y) <= TOL[F32] and R.rel(final, last) <= TOL[F32]
    want = torch.autograd.grad((y * dout.double()).sum() + (last * dfinal.double()).sum(), [leaves[k] for k in S.NAMES])
    for k, ref in zip(S.NAMES, want):
        assert R.rel(grads["d" + k], ref) <= TOL[F32], k


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("channels,states,groups", [(1, 1, 1), (30, 4, 2), (64, 16, 1), (70, 13, 1), (40, 33, 1), (48, 64, 3)])
def test_single_tokens_are_the_sequence(channels, states, groups, dtype):
    """Frame by frame, streams in slots of any order, some left out: the bits of the whole sequences."""
    from paper_1909_05632_amd import ops
    n, length = 5, 6
    x, _, _ = S.inputs(n * length, channels, states, groups, n, dtype, seed=7)
    g = _cuda(x)
    state = g.pop("state")
    out, final = ops.scan_forward(**g, n=n, state=state)
    pool = torch.full((9, channels, states), 3.0, device="cuda")
    ids = torch.tensor([4, 0, 8, 2, 6], dtype=torch.int32, device="cuda")
    pool[ids.long()] = state

    def frame(t):
        at = torch.arange(n, device="cuda") * length + t
        return {k: v[at] if k in ("u", "dt", "b", "c", "z") else v for k, v in g.items()}

    for t in range(length):
        y = ops.scan_step(**frame(t), state=pool, stream_ids=ids)
        assert torch.equal(y, out.view(n, length, channels)[:, t])
    assert torch.equal(pool[ids.long()], final) and (pool[[1, 3, 5, 7]] == 3).all()
    before = pool.clone()
    away = torch.tensor([9, -1, 8, 2, 6], dtype=torch.int32, device="cuda")
    f = frame(0)
    got = ops.scan_step(**f, state=pool, stream_ids=away, out=f["u"])         # over u itself
    assert got is f["u"] and not got[:2].any() and torch.equal(pool[[0, 1, 3, 4, 5, 7]], before[[0, 1, 3, 4, 5, 7]])


def test_steps_of_many_streams():
    """More streams than the grid has rows for, without ids: against the sequences' kernel."""
    from paper_1909_05632_amd import ops
    for n, channels, states in ((3000, 96, 16), (70, 4100, 16)):
        x, _, _ = S.inputs(n, channels, states, 1, n, BF16, seed=n)
        g = _cuda(x)
        state = g.pop("state")
        out, final = ops.scan_forward(**g, n=n, state=state)
        y = ops.scan_step(**g, state=state)
        assert torch.equal(y, out) and torch.equal(state, final)


def test_steps_of_a_pool_without_slots():
    """No id is a slot then: every out is 0, and nothing is read or written through the pool's pointer."""
    from paper_1909_05632_amd import binding as B
    from paper_1909_05632_amd import ops
    L, ref = ops.load_ops(), ops.ctypes.byref
    for states, channels in ((16, 70), (5, 9)):
        x, a = torch.randn(3, channels, device="cuda"), torch.zeros(channels, states, device="cuda")
        b, pool = torch.randn(3, 1, states, device="cuda"), torch.full((1, channels, states), 3.0, device="cuda")
        ids, out = torch.tensor([0, -1, 7], dtype=torch.int32, device="cuda"), torch.ones(3, channels, device="cuda")
        shape = ops.rn_scan_shape(3, channels, 1, states, 3, B.RN_F32, 1, channels, channels, states, states, 0)
        given = ops.rn_scan_inputs(x.data_ptr(), x.data_ptr(), b.data_ptr(), b.data_ptr(), a.data_ptr(), None, None, None)
        stream = torch.cuda.current_stream().cuda_stream
        assert L.reuse_ops_scan_step(ref(shape), ref(given), ids.data_ptr(), 0, pool.data_ptr(), out.data_ptr(), stream) == B.RN_OK
        assert not out.any() and (pool == 3).all()


def test_views_odd_addresses_and_final_over_state():
    from paper_1909_05632_amd import ops
    for dtype, states in ((F32, 16), (BF16, 16), (BF16, 6)):
        x, dout, dfinal = S.inputs(300, 32, states, 2, 3, dtype, seed=5)
        off = [0, 280, 280, 300]
        out, final, grads = _check(x, dout, dfinal, off)
        so = torch.tensor(off, dtype=torch.int32).cuda()
        for at in (4, 3):
            g = _cuda(x)
            state = torch.zeros(1 + g["state"].numel(), device="cuda")[1:].view_as(g["state"]).copy_(g.pop("state"))
            one = torch.full((300, 4 * 64 + 2 * 2 * 80), 9.0, dtype=dtype, device="cuda")    # all of a token in one row
            p = at
            for k in ("u", "dt", "z", "b", "c"):
                w = g[k][0].numel()
                view = one[:, p:p + w]
                view.copy_(g[k].reshape(300, w))
                g[k], p = (view if g[k].dim() == 2 else view.unflatten(1, g[k].shape[1:])), p + w + at
            o2, f2, saved = ops.scan_forward(**g, seq_off=so, state=state, save=True)
            g2 = dict(zip(S.GRADS, ops.scan_backward(dout.cuda(), **g, seq_off=so, saved=saved, dfinal=dfinal.cuda())))
            assert R.rel(o2, out) <= TOL[dtype] and R.rel(f2, final) <= TOL[F32]
            assert all(R.rel(g2[k], grads[k]) <= TOL[dtype] for k in S.GRADS)
            o3, f3 = ops.scan_forward(**g, seq_off=so, state=state, final=state)
            assert f3 is state and torch.equal(o3, o2) and torch.equal(f3, f2)


def test_gradient_against_differences():
    x, dout, dfinal = S.inputs(30, 6, 5, 2, 3, F32, seed=9)
    off = [0, 2, 17, 30]
    _, _, grads = _check(x, dout, dfinal, off)
    gen = torch.Generator().manual_seed(1)
    e = 1e-5
    wide = {k: v.double() for k, v in x.items()}
    for _ in range(4):
        way = {k: torch.randn(v.shape, generator=gen).double() * (0.1 if k == "a" else 1) for k, v in wide.items()}
        vals = []
        for s in (1, -1):
            y, last = S.scan({k: wide[k] + s * e * way[k] for k in wide}, off)
            vals.append((y * dout.double()).sum() + (last * dfinal.double()).sum())
        mine = sum((grads["d" + k].double().cpu() * way[k]).sum() for k in wide)
        size = sum(grads["d" + k].double().norm().item() * way[k].norm().item() for k in wide)
        assert abs((vals[0] - vals[1]) / (2 * e) - mine) <= 2.5e-5 * size


def test_step_sizes_of_any_size():
    """softplus far out on both sides: -infinity leaves the state as it is, large steps empty it.  e^-|x| is
    off by the rounding of its exponent, |x| 2^-24 of itself, and all else by a few 2^-24: 4e-7."""
    from paper_1909_05632_amd import ops
    raw = torch.tensor([-float("inf"), -200.0, -90.0, -30.0, -12.0, -3.0, -1e-3, 0.0, 1e-3, 0.7, 3.0, 12.0, 20.0, 90.0, 1e4])
    T = len(raw)
    x = dict(u=torch.ones(1, T), dt=raw[None], a=torch.full((T, 1), -0.5), b=torch.ones(1, 1, 1), c=torch.ones(1, 1, 1),
             d=None, z=None, dt_bias=None, state=torch.full((1, T, 1), 2.0))
    g = _cuda(x)
    state = g.pop("state")
    out, final = ops.scan_forward(**g, n=1, state=state)
    s = torch.where(raw > 100, raw.double(), torch.log1p(torch.exp(raw.double())))
    want = torch.exp(-0.5 * s) * 2 + s
    tol = 4e-7 + raw.double().abs().clamp(max=200) * 2.0 ** -24
    assert ((out.cpu().double()[0] - want).abs() <= tol * want).all() and out[0, 0] == 2 and torch.equal(final[0, :, 0], out[0])
    # the step alone, from a state of 0: relative to itself also where it is tiny (below 1e-38 it is 0)
    small = ops.scan_forward(**g, n=1)[0].cpu().double()[0]
    fine = s > 1e-37
    assert ((small - s).abs()[fine] <= (tol * s)[fine]).all() and (small[~fine] <= 1e-37).all()


@pytest.mark.parametrize("tokens", [60, 700])
def test_values_that_are_not_finite_stay_in_their_channel_and_sequence(tokens):
    from paper_1909_05632_amd import ops
    x, dout, dfinal = S.inputs(tokens, 16, 16, 2, 3, F32, seed=11)
    cut = tokens // 2
    off = [0, 5, cut, tokens]
    out, final, grads = _run(x, dout, dfinal, seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    x["u"][10, 3], x["dt"][12, 5], x["z"][20, 7] = float("nan"), float("nan"), float("inf")
    x["b"][cut + 3, 1, 2] = float("nan")
    o2, f2, g2 = _run(x, dout, dfinal, seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    hit = torch.zeros(tokens, 16, dtype=torch.bool)
    hit[10:cut, 3], hit[12:cut, 5], hit[20, 7], hit[cut + 3:, 8:] = True, True, True, True
    assert torch.equal(o2.cpu()[~hit], out.cpu()[~hit]) and not torch.isfinite(o2.cpu()[hit]).any()
    away = torch.zeros(3, 16, dtype=torch.bool)
    away[1, 3], away[1, 5], away[2, 8:] = True, True, True
    assert torch.equal(f2.cpu()[~away], final.cpu()[~away])
    for k in ("du", "ddt", "db", "dc", "dz"):            # the first sequence knows nothing of it
        assert torch.equal(g2[k][:5], grads[k][:5]), k
    assert torch.equal(g2["dstate"][0], grads["dstate"][0])
    assert torch.equal(g2["da"][[0, 1, 2, 4, 6]], grads["da"][[0, 1, 2, 4, 6]])


def test_no_tokens_and_empty_sequences():
    from paper_1909_05632_amd import ops
    x, _, _ = S.inputs(0, 8, 5, 1, 3, F32)
    g = _cuda(x)
    state = g.pop("state")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    for kw in (dict(seq_off=off), dict(n=3)):
        out, final, saved = ops.scan_forward(**g, state=state, save=True, **kw)
        assert out.shape == (0, 8) and torch.equal(final, state)
        assert not ops.scan_forward(**g, **kw)[1].any()
        got = dict(zip(S.GRADS, ops.scan_backward(out, **g, saved=saved, dfinal=state, **kw)))
        assert torch.equal(got["dstate"], state) and got["du"].shape == (0, 8)
        assert not got["da"].any() and not got["dd"].any() and not got["ddt_bias"].any()
    none = dict(seq_off=off[:1])
    out, final, saved = ops.scan_forward(**g, save=True, **none)
    got = dict(zip(S.GRADS, ops.scan_backward(out, **g, saved=saved, **none)))
    assert final.shape == (0, 8, 5) and not got["da"].any() and not got["dd"].any() and not got["ddt_bias"].any()
    assert ops.scan_step(**g, state=state).shape == (0, 8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("states", [16, 6])
def test_tokens_behind_the_last_sequence(states, dtype):
    """A padded batch: the rows behind are left as they were, whatever they hold, and reach no result."""
    from paper_1909_05632_amd import ops
    for held, off in ((5, [0, 3, 5]), (300, [0, 40, 40, 300])):
        x, dout, dfinal = S.inputs(held, 12, states, 2, len(off) - 1, dtype, seed=held)
        out, final, grads = _check(x, dout, dfinal, off)
        pad = lambda t: torch.cat([t, torch.full((700, *t.shape[1:]), float("nan"), dtype=dtype)]).cuda()  # noqa: E731
        g = {k: pad(v) if k in ("u", "dt", "b", "c", "z") else v.cuda() for k, v in x.items()}
        state, seqs = g.pop("state"), dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())
        o2 = torch.full_like(g["u"], 7.0)
        _, f2, saved = ops.scan_forward(**g, state=state, save=True, out=o2, **seqs)
        assert (o2[held:] == 7).all() and R.rel(o2[:held], out) <= TOL[dtype] and R.rel(f2, final) <= TOL[F32]
        g2 = dict(zip(S.GRADS, ops.scan_backward(pad(dout), **g, saved=saved, dfinal=dfinal.cuda(), **seqs)))
        for k in S.GRADS:
            got = g2[k][:held] if k in ("du", "ddt", "db", "dc", "dz") else g2[k]
            assert R.rel(got, grads[k]) <= (TOL[F32] if k[1:] in WIDE else TOL[dtype]), k


def test_other_stream_same_bits_and_in_a_graph():
    from paper_1909_05632_amd import ops
    side = torch.cuda.Stream()
    for tokens, channels, n, dtype in ((2000, 24, 3, BF16), (500, 256, 30, F32)):
        x, dout, dfinal = S.inputs(tokens, channels, 16, 1, n, dtype, seed=13)
        g, dout, dfinal = _cuda(x), dout.cuda(), dfinal.cuda()
        state = g.pop("state")
        off = torch.tensor(_cuts(tokens, n, 5), dtype=torch.int32).cuda()

        def all_of(**kw):
            out, final, saved = ops.scan_forward(**g, seq_off=off, state=state, save=True, **kw)
            return [out, final, *ops.scan_backward(dout, **g, seq_off=off, saved=saved, dfinal=dfinal, **kw)]

        torch.cuda.synchronize()
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
    """600000 tokens of 4096 channels in bfloat16 are 2.4e9 elements: the last tokens go on from the state before."""
    from paper_1909_05632_amd import ops
    tokens, channels, states, tail = 600000, 4096, 2, 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    u, dt = (torch.empty(tokens, channels, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    b, c = (torch.empty(tokens, 1, states, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    a = -torch.rand(channels, states, generator=gen, device="cuda") - 0.05
    out, final = ops.scan_forward(u, dt, a, b, c, n=1)
    cut = tokens - tail
    # a state of 2000 tokens before the tail has forgotten what lies further back: decays are e^-0.02 a token at most
    warm = [t[cut - 2000:cut] for t in (u, dt)] + [a] + [t[cut - 2000:cut] for t in (b, c)]
    state = ops.scan_forward(*warm, n=1)[1]
    end, last = ops.scan_forward(u[cut:], dt[cut:], a, b[cut:], c[cut:], n=1, state=state)
    assert R.rel(out[cut:], end) <= TOL[BF16] and R.rel(final, last) <= TOL[F32]
    del u, dt, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("states", [2, 5, 16, 40])
@pytest.mark.parametrize("tokens", [1, 2, 3, 7, 16, 19, 130])
def test_states_that_are_emptied_by_every_token(tokens, states, dtype):
    """a of -infinity: exp(s a) is 0 for every s above 0, whatever the sequence's length.  (The gradients are those
    of a very low finite a, whose da is 0 and whose part in ds is too.)"""
    from paper_1909_05632_amd import ops
    x, dout, dfinal = S.inputs(tokens, 6, states, 2, 1, dtype, seed=tokens)
    some = torch.rand(6, states, generator=torch.Generator().manual_seed(1)) < 0.4
    some[0, 0], x["a"][some] = True, -1e30
    lowest = _check(x, dout, dfinal, [0, tokens])
    x["a"][some] = -float("inf")
    out, final, grads = _run(x, dout, dfinal, n=1)
    assert torch.equal(out, lowest[0]) and torch.equal(final, lowest[1])
    assert all(torch.equal(grads[k], lowest[2][k]) for k in S.GRADS)
    g = _cuda(x)
    pool = g.pop("state")
    for t in range(min(tokens, 3)):
        y = ops.scan_step(**{k: v[t:t + 1] if k in ("u", "dt", "b", "c", "z") else v for k, v in g.items()}, state=pool)
        assert torch.equal(y, out[t:t + 1])


def test_a_step_of_zero_leaves_the_state_whatever_a_is():
    from paper_1909_05632_amd import ops
    a = torch.tensor([[-3.4e38, -2.5e38, -1.0, 2.5e38, 3.4e38]], device="cuda")
    for tokens in (1, 5, 100):
        u, dt = torch.ones(tokens, 1, device="cuda"), torch.zeros(tokens, 1, device="cuda")
        b = torch.ones(tokens, 1, 5, device="cuda")
        state = torch.tensor([[[1.0, -2.0, 3.0, 4.0, -5.0]]], device="cuda")
        out, final, saved = ops.scan_forward(u, dt, a, b, b, softplus=False, n=1, state=state, save=True)
        assert (out == 1).all() and torch.equal(final, state)
        dstate = ops.scan_backward(out, u, dt, a, b, b, softplus=False, n=1, saved=saved)[-1]
        assert (dstate == tokens).all()
        assert (ops.scan_step(u[:1], dt[:1], a, b[:1], b[:1], state, softplus=False) == 1).all()
        assert torch.equal(final, state)


def test_states_that_grow_across_chunks():
    """a above 0: over a chunk exp(sum of s a) may be past float32 while the state is 0, or so small that the
    product is not.  (Exponents of up to 140 are off by 140 2^-24 of the result at each of two roundings: 2e-5.)"""
    from paper_1909_05632_amd import ops
    gen = torch.Generator().manual_seed(4)
    tokens, channels = 200, 3
    for states in (2, 6):
        a = 6 - 2 * torch.arange(states).float().remainder(2).expand(channels, states)
        u, dout = torch.zeros(tokens, channels), torch.zeros(tokens, channels)
        u[-5:], dout[:5] = torch.randn(5, channels, generator=gen), torch.randn(5, channels, generator=gen)
        x = dict(u=u, dt=torch.ones(tokens, channels), a=a.contiguous(), b=torch.randn(tokens, 1, states, generator=gen),
                 c=torch.randn(tokens, 1, states, generator=gen), d=None, z=None, dt_bias=None, state=None)
        out, _, grads = _check(x, dout, None, [0, tokens], softplus=False)
        assert out[-5:].all() and not out[:-5].any() and grads["du"][:5].all() and not grads["du"][5:].any()
        # a state of 1e-30, over 16 tokens of growth, then held
        x["dt"][16:], x["u"], x["state"] = 0, torch.zeros_like(u), torch.full((1, channels, states), 1e-30)
        g = _cuda(x)
        out, final = ops.scan_forward(**g, softplus=False, n=1)
        y, last = S.scan({k: None if v is None else v.double() for k, v in x.items()}, [0, tokens], False)
        assert R.rel(final, last) <= 4e-5 and R.rel(out, y) <= 4e-5


# Chunks of `chunk` tokens in the gradients: the least power of two, 32 or more, that
# leaves no more than 4096 for all blocks of channels (64 of a group, or what it has).
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens,channels,states,groups,n,chunk", [
    (1100, 130, 16, 130, 2, 64), (1200, 140, 64, 140, 3, 64), (1200, 300, 32, 150, 2, 64), (1000, 270, 4, 270, 1, 128),
    (1300, 230, 7, 230, 3, 128), (1400, 390, 16, 390, 2, 256), (900, 600, 33, 600, 1, 256), (2100, 4160, 16, 1, 3, 64),
    (2200, 4100, 8, 2, 2, 64), (1500, 6200, 4, 1, 2, 64)])
def test_gradients_in_chunks_of_several_tiles(tokens, channels, states, groups, n, chunk, dtype):
    blocks = groups * -(-(channels // groups) // 64)
    assert max(32, 1 << (-(-tokens * blocks // 4096) - 1).bit_length()) == chunk and tokens / n > 2 * chunk
    x, dout, dfinal = S.inputs(tokens, channels, states, groups, n, dtype, seed=tokens)
    off = _cuts(tokens, n, seed=groups)
    assert max(q - p for p, q in zip(off, off[1:])) > 2 * chunk
    out, final, grads = _run(x, dout, dfinal, seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    leaves = {k: v.cuda().double().requires_grad_() for k, v in x.items()}
    y, last = S.scan(leaves, off)
    assert R.rel(out, y) <= TOL[dtype] and R.rel(final, last) <= TOL[F32]
    loss = (y * dout.cuda().double()).sum() + (last * dfinal.cuda().double()).sum()
    for k, want in zip(S.NAMES, torch.autograd.grad(loss, [leaves[k] for k in S.NAMES])):
        assert R.rel(grads["d" + k], want) <= (TOL[F32] if k in WIDE else TOL[dtype]), k


def test_gradients_past_32_bits():
    """600000 tokens of 4096 channels in bfloat16 are 2.4e9 elements: the gradients of the last tokens, and of the
    first, are those of calls of their own (decays are e^-0.02 a token at most: 2000 tokens on, nothing is left)."""
    from paper_1909_05632_amd import ops
    tokens, channels, states, part, far = 600000, 4096, 2, 512, 2000
    gen = torch.Generator(device="cuda").manual_seed(1)
    u, dt = (torch.empty(tokens, channels, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    b, c = (torch.empty(tokens, 1, states, dtype=BF16, device="cuda").normal_(generator=gen) for _ in range(2))
    a = -torch.rand(channels, states, generator=gen, device="cuda") - 0.05
    saved = ops.scan_forward(u, dt, a, b, c, n=1, save=True)[2]
    grads = dict(zip(S.GRADS, ops.scan_backward(u, u, dt, a, b, c, n=1, saved=saved)))
    del saved
    for lo, hi, keep in ((0, part + far, slice(0, part)), (tokens - part - far, tokens, slice(far, part + far))):
        x = [t[lo:hi] for t in (u, dt)] + [a] + [t[lo:hi] for t in (b, c)]
        kept = ops.scan_forward(*x, n=1, save=True)[2]
        alone = dict(zip(S.GRADS, ops.scan_backward(x[0].contiguous(), *x, n=1, saved=kept)))
        for k in ("du", "ddt", "db", "dc"):
            assert R.rel(grads[k][lo:hi][keep], alone[k][keep]) <= TOL[BF16], k
        if lo == 0:
            assert R.rel(grads["dstate"], alone["dstate"]) <= TOL[F32]
    assert torch.isfinite(grads["da"]).all()
    del u, dt, grads
    torch.cuda.empty_cache()
