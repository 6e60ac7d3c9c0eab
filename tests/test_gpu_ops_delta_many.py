"""The gated delta rule over many sequences at once, and gradients of even short
ones, on the GPU against the recurrence in 64 bits.  Inputs, comparison and
tolerances are those of test_gpu_ops_delta.py; a bfloat16 result of a few
elements is within the worst case of one rounding, 2^-8, where the 2-norm of
many is within 2^-9."""
import random

import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available
from tests.test_gpu_ops_delta import BF16, F32, TOL, TOL_G, _compare, _inputs, _reference

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]


def _lengths(n, longest, seed):
    """n lengths, many of them 0, 1 and a chunk's, more long ones than an average of 32 allows or fewer."""
    rng = random.Random(seed)
    return [rng.choice((0, 1, 2, 31, 32, 33, 63, 64, 65, rng.randint(1, longest))) for _ in range(n)]


# 64 sequences are ordered by length, 65 are not; a slot's sequence is searched 64
# places at once, twice from 66 sequences on.
@pytest.mark.parametrize("n", [2, 63, 64, 65, 66, 130])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_ragged_sequences(n, dtype):
    x, off = _inputs(_lengths(n, 200, n), 1, 2, 16, 24, dtype, seed=n)
    _compare(x, off, 0.25, n)


@pytest.mark.parametrize("hv", [1, 3, 8])
def test_sequences_of_one_length_and_empty_ones(hv):
    """Ties in the order by length, and lengths that differ by all there is."""
    for lengths in ([70] * 9, [0] * 5 + [150] + [0] * 5, [100, 0, 100, 0, 100], list(range(0, 130, 13))):
        x, off = _inputs(lengths, 1, hv, 32, 48, F32, seed=hv)
        _compare(x, off, 0.2, lengths)


def test_few_long_among_thousands_of_short():
    """5000 sequences, most of a token or none: the search for a slot's sequence takes three turns."""
    from paper_1909_05632_amd import ops
    lengths = [i % 3 % 2 for i in range(5000)]
    longs = {0: 70, 2499: 40, 4160: 130, 4999: 65}
    for i, m in longs.items():
        lengths[i] = m
    x, off = _inputs(lengths, 1, 1, 8, 8, F32, seed=1)
    d = {k: v.cuda() for k, v in x.items()}
    args = [d[k] for k in ("q", "k", "v", "g", "beta")] + [torch.tensor(off, dtype=torch.int32).cuda()]
    out, final, saved = ops.delta_forward(*args, state=d["state"], scale=0.3, save=True)
    grads = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=d["dfinal"], scale=0.3)
    for i in list(longs) + [1, 3, 2500, 4998]:
        a, b = off[i], off[i + 1]
        part = {k: v[i:i + 1] if k in ("state", "dfinal") else v[a:b] for k, v in x.items()}
        want, last, g = _reference(part, [0, b - a], 0.3)
        assert R.rel(final[i:i + 1], last) <= TOL[F32] and R.rel(grads[5][i:i + 1], g["state"]) <= TOL[F32], i
        if b > a:
            assert R.rel(out[a:b], want) <= TOL[F32], i
            for got, name in zip(grads, ("q", "k", "v", "g", "beta")):
                assert R.rel(got[a:b], g[name]) <= TOL_G, (i, name)


@pytest.mark.parametrize("length", [1, 3, 16, 17, 32])
@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 3, 64, 64), (2, 2, 128, 128), (1, 2, 65, 33), (2, 4, 30, 100), (1, 1, 1, 1)])
def test_gradients_of_even_short_sequences(length, hk, hv, dk, dv):
    """Without offsets the lengths are known before the call: one tile of tokens or two."""
    from paper_1909_05632_amd import ops
    n = 5
    for dtype in (F32, BF16):
        x, off = _inputs([length] * n, hk, hv, dk, dv, dtype, seed=length)
        d = {k: v.cuda() for k, v in x.items()}
        args = [d[k] for k in ("q", "k", "v", "g", "beta")]
        want, last, g = _reference(x, off, 0.3)
        out, final, saved = ops.delta_forward(*args, n=n, state=d["state"], scale=0.3, save=True)
        grads = ops.delta_backward(d["dout"], *args, n=n, saved=saved, dfinal=d["dfinal"], scale=0.3)
        tol = TOL[F32] if dtype is F32 else 2.0 ** -8 + TOL[F32]
        assert R.rel(out, want) <= tol and R.rel(final, last) <= TOL[F32]
        for got, name, tol in zip(grads, ("q", "k", "v", "g", "beta", "state"), (tol,) * 3 + (TOL_G, TOL_G, TOL[F32])):
            assert R.rel(got, g[name]) <= tol, (dtype, name)


def test_short_gradients_without_a_last_gradient_or_off_alignment():
    from paper_1909_05632_amd import ops
    for lengths in ([16] * 4, [5, 32, 0, 17]):
        x, off = _inputs(lengths, 1, 2, 64, 64, F32, seed=9)
        d = {k: v.cuda() for k, v in x.items()}
        off_ = torch.tensor(off, dtype=torch.int32).cuda()
        args = [d[k] for k in ("q", "k", "v", "g", "beta")] + [off_]
        out, final, saved = ops.delta_forward(*args, state=d["state"], scale=0.125, save=True)
        none = ops.delta_backward(d["dout"], *args, saved=saved, scale=0.125)
        zero = ops.delta_backward(d["dout"], *args, saved=saved, dfinal=torch.zeros_like(d["dfinal"]), scale=0.125)
        assert all(torch.equal(a, b) for a, b in zip(none, zero))

        def off_by_one(t):                           # the same values, one element off every alignment
            r = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape)
            return r.copy_(t)
        odd = [off_by_one(t) for t in args[:5]] + [off_]
        out2, final2, saved2 = ops.delta_forward(*odd, state=off_by_one(d["state"]), scale=0.125, save=True)
        got = ops.delta_backward(off_by_one(d["dout"]), *odd, saved=saved2, dfinal=off_by_one(d["dfinal"]), scale=0.125)
        _, _, g = _reference(x, off, 0.125)
        assert R.rel(out2, out) <= TOL[F32] and R.rel(final2, final) <= TOL[F32]
        for a, name, tol in zip(got, ("q", "k", "v", "g", "beta", "state"), (TOL[F32],) * 3 + (TOL_G, TOL_G, TOL[F32])):
            assert R.rel(a, g[name]) <= tol, name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,hv", [(60, 9), (70, 8)])
def test_more_blocks_than_fit_at_once(n, hv, dtype):
    """A walk's block then takes two column tiles, the second one in part past dv."""
    x, off = _inputs(_lengths(n, 150, 3), 1, hv, 16, 20, dtype, seed=2)
    _compare(x, off, 0.25, (n, hv))
