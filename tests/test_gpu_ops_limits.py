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
