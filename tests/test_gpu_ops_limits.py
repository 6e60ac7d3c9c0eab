"""The operators at the ends of the sizes that their checks let through."""
import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]


@pytest.fixture(autouse=True)
def _free():
    yield
    torch.cuda.empty_cache()


def test_more_heads_of_streams_than_a_grid_axis_holds():
    """65535 streams of 320 heads: 21 million blocks of 256 threads.  A memory is one number, so
    that a token and its gradients are a line each; a dozen roundings of 2^-24 of terms that
    cancel no more than random ones do stay below 4e-6 of the norm."""
    from paper_1909_05632_amd import ops
    n, heads, scale = 65535, 320, 0.7
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v, g, beta, s, do, ds = (torch.randn(n, heads, generator=gen, device="cuda") for _ in range(8))
    g, beta, k = -g.abs(), torch.sigmoid(beta), torch.tanh(k)
    shape = lambda t: t.unsqueeze(-1)  # noqa: E731
    args = [shape(q), shape(k), shape(v), g, beta]
    Q, K, V, G, B, S, DO, DS = (t.double() for t in (q, k, v, g, beta, s, do, ds))
    mid = torch.exp(G) * S
    err = V - K * mid
    new = mid + B * K * err
    tol = 4e-6
    state = s.clone().view(n, heads, 1, 1)
    out = ops.delta_step(*args, state, scale=scale)
    assert R.rel(out[..., 0], scale * Q * new) <= tol and R.rel(state[..., 0, 0], new) <= tol
    out, final, saved = ops.delta_forward(*args, n=n, state=s.view(n, heads, 1, 1), scale=scale, save=True)
    assert R.rel(out[..., 0], scale * Q * new) <= tol and R.rel(final[..., 0, 0], new) <= tol
    grads = ops.delta_backward(shape(do), *args, n=n, saved=saved, dfinal=ds.view(n, heads, 1, 1), scale=scale)
    D = DS + scale * Q * DO
    x = K * D
    after = D - K * B * x
    want = (scale * DO * new, D * B * err - B * x * mid, B * x, after * mid, x * err, torch.exp(G) * after)
    for a, b, name in zip(grads, want, ("q", "k", "v", "g", "beta", "state")):
        assert R.rel(a.reshape(n, heads), b) <= tol, name


@pytest.mark.parametrize("rows,vocab", [((1 << 26) + 100, 2), ((1 << 24) + 50, 65), ((1 << 22) + 50, 4097)])
def test_more_rows_of_choices_than_a_grid_axis_holds(rows, vocab):
    """One wave, 256 threads and 1024 threads a row: each row's draw is the one it has in a small batch."""
    from paper_1909_05632_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(rows, vocab, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    u = torch.rand(rows, generator=gen, device="cuda")
    tokens, logprobs = torch.full((rows,), -5, dtype=torch.int32, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    ops.sample(x, u, 0.8, 30, 0.9, tokens=tokens, logprobs=logprobs)
    for lo in (0, rows // 2 - 1000, rows - 5000, rows - 1):
        t, p = ops.sample(x[lo:lo + 5000], u[lo:lo + 5000], 0.8, 30, 0.9)
        assert bool((t == tokens[lo:lo + 5000]).all()) and bool((p == logprobs[lo:lo + 5000]).all()), lo
    assert int(tokens.min()) >= 0 and int(tokens.max()) < vocab and float(logprobs.max()) <= 0


def test_weight_gradients_wider_than_a_grid_axis_holds():
    """2^25 + 6 columns in 16s, 1024 threads each: with one row dweight is dy xh and dbias dy."""
    from paper_1909_05632_amd import ops
    width = (1 << 25) + 6
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(1, width, generator=gen, device="cuda") for _ in range(2))
    stats = torch.tensor([[0.25, 1.5]], device="cuda")
    dw, db = torch.full((width,), 7.0, device="cuda"), torch.full((width,), 7.0, device="cuda")
    dx, _, _ = ops.layer_norm_backward(dy, x, None, stats, dweight=dw, dbias=db)
    assert bool((db == dy[0]).all())
    xh = (x.double() - 0.25) * 1.5
    assert R.rel(dw, (dy.double() * xh)[0]) <= 4e-6
    # a thread adds 2^17 terms of random sign in a row: 2^8.5 roundings of their sum's size, which dx shares through two means
    d = dy.double()
    assert R.rel(dx, 1.5 * (d - d.mean() - xh * (d * xh).mean())) <= 2.0 ** -24 * 2 ** 8.5


def test_steps_of_an_empty_pool():
    """No id is a slot of a pool of 0 slots: every out is 0."""
    from paper_1909_05632_amd import ops
    ids = torch.tensor([0, -1, 7], dtype=torch.int32, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        for channels, states in ((70, 16), (9, 5)):
            x, a = torch.randn(3, channels, device="cuda").to(dtype), torch.zeros(channels, states, device="cuda")
            b, pool = torch.randn(3, 1, states, device="cuda").to(dtype), torch.empty(0, channels, states, device="cuda")
            out = torch.ones(3, channels, dtype=dtype, device="cuda")
            assert ops.scan_step(x, x, a, b, b, pool, stream_ids=ids, out=out) is out and not out.any()
            for taps in (1, 4):
                w, pool = torch.randn(channels, taps, device="cuda"), torch.empty(0, taps - 1, channels, dtype=dtype, device="cuda")
                out = torch.ones(3, channels, dtype=dtype, device="cuda")
                assert ops.causal_conv_step(x, w, pool, stream_ids=ids, out=out) is out and not out.any()
        q, v = torch.randn(3, 2, 8, device="cuda").to(dtype), torch.randn(3, 4, 5, device="cuda").to(dtype)
        g, pool, out = torch.zeros(3, 4, device="cuda"), torch.empty(0, 4, 8, 5, device="cuda"), torch.ones_like(v)
        assert ops.delta_step(q, q, v, g, g, pool, stream_ids=ids, out=out) is out and not out.any()
