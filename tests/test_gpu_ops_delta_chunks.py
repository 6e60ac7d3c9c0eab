"""Chunks of the gated delta rule where their triangular systems, their batches or
their values are hard, on the GPU against the recurrence in 64 bits.  Inputs and
tolerances are those of test_gpu_ops_delta.py unless a test derives its own."""
import math
import random

import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available
from tests.test_gpu_ops_delta import BF16, F32, NAMES, TOL, TOL_G, _compare, _inputs, _reference, _run

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("length", [33, 48, 49, 64, 65, 600])
def test_write_strengths_up_to_two(length, dtype):
    """Near-equal keys and beta up to 2, where the inverse's entries stay at 2 from the diagonal
    to the corner: (I + A)^-1_ij = -beta (1 - beta)^(i-j-1).

    Its 64 entries a row, each off by some 2^-24 of their size, no longer shrink: 64 x 2^-24 of a
    chunk's errors E, four times that allowed, 1.5e-5, and as the memory hardly decays the chunks'
    errors add up like their square root.  The gradients pass through two such systems, twice
    that; those of g and beta are allowed more in the proportion of TOL_G to TOL."""
    x, off = _inputs([length], 1, 2, 64, 64, dtype, near=8.0, decay=(1e-4, 1e-2), seed=length)
    u = torch.rand(x["beta"].shape, generator=torch.Generator().manual_seed(5))
    x["beta"] = 2.0 - 0.05 * u
    x["beta"][:, 1] = 2.0
    out, final, grads = _run(x, off, 0.125)
    want, last, g = _reference(x, off, 0.125)
    tol = 4 * 64 * 2.0 ** -24 * math.sqrt((length + 63) // 64)
    own = 2.0 ** -9 if dtype is BF16 else 0.0
    assert R.rel(out, want) <= tol + own and R.rel(final, last) <= tol
    for got, name in zip(grads, NAMES + ("state",)):
        more = TOL_G / TOL[F32] if name in ("g", "beta") else 1.0
        assert R.rel(got, g[name]) <= 2 * tol * more + (own if got.dtype is BF16 else 0.0), name


@pytest.mark.parametrize("what", ["memory", "written", "scores"])
def test_bfloat16_outputs_are_sums_in_float32(what):
    """Outputs that cancel to 2^-14 of their terms show what the terms were rounded to: the memory
    read, the values written, and the scores, none of them a bfloat16 input.

    Two keys, the axes 0 and 1, and queries of their difference: out = x0 - x1.  Rounded once to
    bfloat16 it is within 2^-8 of its own size; x0 and x1, of size 1 at most, and their sums carry
    eight roundings of 2^-24, where exponentials enter two more of 2^-23 and their arguments'."""
    from paper_1909_05632_amd import ops
    hv, dk, dv, tokens = 32, 64, 48, 70
    gen = torch.Generator().manual_seed(1)
    q, k = torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dk)
    k[0, 0, 0] = k[1:, 0, 1] = 1.0
    q[2:, 0, 0], q[2:, 0, 1] = 1.0, -1.0
    v, g, beta = torch.zeros(tokens, hv, dv), torch.zeros(tokens, hv), torch.zeros(tokens, hv)
    state = torch.zeros(1, hv, dk, dv)
    x0 = 0.5 + 0.5 * torch.rand(hv, dv, generator=gen)
    near = 1 - 2.0 ** -14 * torch.rand(hv, dv, generator=gen)
    bound = 2.0 ** -21
    if what == "memory":
        state[0, :, 0], state[0, :, 1] = x0, x0 * near
    else:
        v[:2] = 1.0
        if what == "written":
            beta[0], beta[1] = x0[:, 0], x0[:, 0] * near[:, 0]
        else:
            beta[:2] = 1.0
            g[1], g[2] = torch.log(near[:, 0]), torch.log(x0[:, 0])
            bound = 2.0 ** -20
    x = dict(q=q.bfloat16(), k=k.bfloat16(), v=v.bfloat16(), g=g, beta=beta)
    out, _ = ops.delta_forward(*(x[n].cuda() for n in NAMES), n=1, state=state.cuda(), scale=1.0)
    want, _ = R.delta(*(x[n].double() for n in NAMES), [0, tokens], state.double(), 1.0)
    largest = want[2:].abs().max().item()
    off = ((out.double().cpu() - want)[2:].abs() - 2.0 ** -8 * want[2:].abs()).max().item()
    assert largest < 2.0 ** -13 and off <= bound


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [3, 40, 64, 65, 300])
def test_long_ones_among_short_share_no_slot(n, dtype):
    """32 tokens a sequence or fewer on average, so that short ones go token by token: the others lie
    at every distance from the places where slots begin, some next to each other."""
    rng = random.Random(n)
    lengths = [rng.choice((0, 1, 2, 5, 16, 31, 32)) for _ in range(n)]
    for at in range(0, n, 9):
        lengths[at:at + 2] = [rng.choice((33, 34, 64, 65, 95, 96, 97, 129)), rng.choice((0, 33, 64))][:len(lengths[at:at + 2])]
    while sum(lengths) > 32 * n:
        lengths[lengths.index(max(lengths))] -= 7
    assert any(m > 32 for m in lengths)
    x, off = _inputs(lengths, 1, 2, 16, 24, dtype, seed=n)
    _compare(x, off, 0.25, lengths)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("lengths,even", [([150], False), ([40, 70], False), ([64, 64], True), ([20], False),
                                          ([16] * 4, True), ([5, 32, 70, 1, 0, 9], False)])
def test_values_that_are_not_finite_reach_later_tokens_only(lengths, even, dtype):
    """NaN or infinity in a token leaves the bits of the tokens before it alone, of the other
    columns (v), of the other tokens (q), of the other heads (g, beta) and of the other sequences."""
    from paper_1909_05632_amd import ops
    hk, hv, dk, dv = 2, 4, 64, 70
    x, off = _inputs(lengths, hk, hv, dk, dv, dtype, seed=sum(lengths))
    d = {k: v.cuda() for k, v in x.items()}
    how = dict(n=len(lengths)) if even else dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())

    def run(y, save):
        got = ops.delta_forward(*(y[k] for k in NAMES), state=y["state"], scale=0.125, save=save, **how)
        return got[0], got[1]

    want, last = run(d, False)
    longest = max(range(len(lengths)), key=lambda i: lengths[i])
    begin, end = off[longest], off[longest + 1]
    for step in (0, 1, 15, 17, 40, 63, 64, 100):
        t = begin + step
        if t >= end:
            continue
        for name in NAMES:
            for value in (math.nan, math.inf, -math.inf):
                if name == "g" and value == -math.inf:
                    continue                         # that empties the memory
                y = {k: v.clone() for k, v in d.items()}
                head = 1 if name in ("q", "k") else 2
                if name in ("g", "beta"):
                    y[name][t, head] = value
                else:
                    y[name][t, head, 7] = value
                for save in (False, True):
                    out, final = run(y, save)
                    reached, memory = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(final, dtype=torch.bool)
                    heads = slice(2, 4) if name in ("q", "k") else slice(2, 3)
                    cols = slice(7, 8) if name == "v" else slice(0, dv)
                    reached[t:t + 1 if name == "q" else end, heads, cols] = True
                    if name != "q":
                        memory[longest, heads, :, cols] = True
                    case = (step, name, value, save)
                    assert torch.equal(out[~reached], want[~reached]), case
                    assert torch.equal(final[~memory], last[~memory]), case
                    assert not out[reached].isfinite().any() and not final[memory].isfinite().any(), case


@pytest.mark.parametrize("length", [20, 150])
def test_a_memory_that_is_not_finite_stays_in_its_column(length):
    from paper_1909_05632_amd import ops
    for dtype in (F32, BF16):
        x, off = _inputs([length, length], 1, 2, 40, 33, dtype)
        d = {k: v.cuda() for k, v in x.items()}
        want, last = ops.delta_forward(*(d[k] for k in NAMES), n=2, state=d["state"], scale=0.125)
        for value in (math.nan, math.inf):
            bad = d["state"].clone()
            bad[1, 0, 3, 20] = value
            out, final = ops.delta_forward(*(d[k] for k in NAMES), n=2, state=bad, scale=0.125)
            reached, memory = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(final, dtype=torch.bool)
            reached[length:, 0, 20] = True
            memory[1, 0, :, 20] = True
            assert torch.equal(out[~reached], want[~reached]) and torch.equal(final[~memory], last[~memory])
            assert not out[reached].isfinite().any() and not final[memory].isfinite().any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dk", [64, 100])
@pytest.mark.parametrize("lengths,even", [([70] * 9, True), ([40, 97, 0, 64, 33] + [50] * 12, False)])
def test_batches_that_take_two_column_tiles_a_block(lengths, even, dk, dtype):
    """More than 256 (ragged: 512) sequences x heads x 32s of columns: a walk's block then has two
    tiles of 16 columns, the second one here in part past dv, for every size of keys."""
    from paper_1909_05632_amd import ops
    x, off = _inputs(lengths, 2, 16, dk, 33, dtype, seed=dk)
    d = {k: v.cuda() for k, v in x.items()}
    args = [d[k] for k in NAMES]
    how = dict(n=len(lengths)) if even else dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    want, last, g = _reference(x, off, 0.125)
    tol = TOL[F32] if dtype is F32 else 2.0 ** -9 + TOL[F32]
    out, final = ops.delta_forward(*args, state=d["state"], scale=0.125, **how)
    assert R.rel(out, want) <= tol and R.rel(final, last) <= TOL[F32]
    out2, final2, saved = ops.delta_forward(*args, state=d["state"], scale=0.125, save=True, **how)
    assert torch.equal(out2, out) and torch.equal(final2, final)
    grads = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=0.125, **how)
    for got, name, bound in zip(grads, NAMES + ("state",), (tol,) * 3 + (TOL_G, TOL_G, TOL[F32])):
        assert R.rel(got, g[name]) <= bound, name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_training_batch_of_episodes(dtype):
    """256 streams of 64 frames, 4 heads of 64 x 64: some of the episodes against the recurrence."""
    from paper_1909_05632_amd import ops
    x, off = _inputs([64] * 256, 4, 4, 64, 64, dtype, seed=7)
    d = {k: v.cuda() for k, v in x.items()}
    args = [d[k] for k in NAMES]
    out, final, saved = ops.delta_forward(*args, n=256, state=d["state"], scale=0.125, save=True)
    grads = ops.delta_backward(d["dout"], *args, n=256, saved=saved, dfinal=d["dfinal"], scale=0.125)
    tol = TOL[F32] if dtype is F32 else 2.0 ** -9 + TOL[F32]
    for i in (0, 1, 63, 64, 130, 255):
        a, b = off[i], off[i + 1]
        part = {k: v[i:i + 1] if k in ("state", "dfinal") else v[a:b] for k, v in x.items()}
        want, last, g = _reference(part, [0, b - a], 0.125)
        assert R.rel(out[a:b], want) <= tol and R.rel(final[i:i + 1], last) <= TOL[F32], i
        for got, name, bound in zip(grads, NAMES, (tol,) * 3 + (TOL_G, TOL_G)):
            assert R.rel(got[a:b], g[name]) <= bound, (i, name)
        assert R.rel(grads[5][i:i + 1], g["state"]) <= TOL[F32], i


@pytest.mark.parametrize("lengths,even", [([20], False), ([16] * 4, True), ([16] * 4, False), ([5, 32, 70, 1, 0, 9], False)])
def test_memory_emptied_in_short_sequences(lengths, even):
    """g = -infinity at a token of sequences that go token by token: what follows is a sequence of its own."""
    from paper_1909_05632_amd import ops
    x, off = _inputs(lengths, 1, 2, 64, 48, F32, seed=3)
    cut = {i: m // 2 for i, m in enumerate(lengths) if m > 1}
    x["g"][[off[i] + c for i, c in cut.items()]] = -math.inf
    d = {k: v.cuda() for k, v in x.items()}
    args = [d[k] for k in NAMES]
    how = dict(n=len(lengths)) if even else dict(seq_off=torch.tensor(off, dtype=torch.int32).cuda())
    out, final, saved = ops.delta_forward(*args, state=d["state"], scale=0.2, save=True, **how)
    grads = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=0.2, **how)
    parts, firsts = [0], []                          # each sequence as the two it falls into
    split = {k: v.clone() for k, v in x.items()}
    state, dfinal = [], []
    for i, m in enumerate(lengths):
        c = cut.get(i, 0)
        if c:
            parts.append(off[i] + c)
            firsts.append(off[i] + c)
            state += [x["state"][i], torch.zeros_like(x["state"][i])]
            dfinal += [torch.zeros_like(x["dfinal"][i]), x["dfinal"][i]]
        else:
            state.append(x["state"][i]), dfinal.append(x["dfinal"][i])
        parts.append(off[i] + m)
    split["g"][firsts] = 0.0
    split["state"], split["dfinal"] = torch.stack(state), torch.stack(dfinal)
    want, last, g = _reference(split, parts, 0.2)
    ends = [parts.index(off[i + 1], 1) - 1 if lengths[i] else None for i in range(len(lengths))]
    assert R.rel(out, want) <= TOL[F32]
    for i, e in enumerate(ends):
        assert R.rel(final[i], last[e] if e is not None else x["state"][i]) <= TOL[F32], i
    for got, name, tol in zip(grads, NAMES, (TOL[F32],) * 3 + (TOL_G, TOL_G)):
        a, b = got.double().cpu(), g[name].clone()
        if name == "g":
            assert a[firsts].abs().max() <= TOL_G * b.norm() and torch.isfinite(a).all()
            a[firsts] = b[firsts] = 0.0
        assert R.rel(a, b) <= tol, name


@pytest.mark.parametrize("lengths", [[20, 16, 9], [5, 32, 70, 1, 0, 9], [16] * 4])
def test_a_sequence_of_nan_stays_alone_token_by_token(lengths):
    x, off = _inputs(lengths, 1, 2, 64, 64, F32)
    out, final, grads = _run(x, off, 0.125)
    at = 1
    bad = {k: v.clone() for k, v in x.items()}
    for k in ("q", "k", "v", "g", "beta", "dout"):
        bad[k][off[at]:off[at + 1]] = math.nan
    out2, final2, grads2 = _run(bad, off, 0.125)
    keep = [t for t in range(off[-1]) if not off[at] <= t < off[at + 1]]
    rest = [i for i in range(len(lengths)) if i != at]
    assert torch.equal(out2[keep], out[keep]) and torch.equal(final2[rest], final[rest])
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(grads2[:5], grads[:5]))
    assert torch.equal(grads2[5][rest], grads[5][rest]) and out2[off[at]:off[at + 1]].isnan().all()
