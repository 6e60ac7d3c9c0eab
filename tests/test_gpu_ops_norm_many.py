"""Layer norm over more rows than its grids have blocks, and gradients written
over their inputs where a block walks several rows.  Tolerances are those of
test_gpu_ops_norm.py."""
import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

EPS = 1e-5


def _inputs(rows, width, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x = ((randn(rows, width) + 0.7) * torch.exp(randn(rows, 1))).to(dtype)
    return x, randn(rows, width).to(dtype), 1 + 0.1 * randn(width), 0.1 * randn(width)


@pytest.mark.parametrize("rows,width,dtype", [(16400, 2050, torch.float32), (16390, 16388, torch.bfloat16),
                                              (16384 * 32 + 77, 40, torch.bfloat16), (16384 * 4 + 9, 200, torch.float32)])
def test_rows_past_the_grids_first_turn(rows, width, dtype):
    """One block a row and many rows a block, in registers and too wide for them."""
    from paper_1909_05632_amd import ops
    x, dy, w, b = _inputs(rows, width, dtype, rows)
    y, stats = ops.layer_norm(x, w, b, EPS, with_stats=True)
    dx, dw, db = ops.layer_norm_backward(dy, x, w, stats)
    tol = 4e-6 if dtype is torch.float32 else 2.0 ** -8
    some = sorted({0, 1, 100, rows // 2, 16383, *range(16384, 16390), rows - 2, rows - 1})
    want = R.layer_norm(x[some], w, b, EPS)
    mean = x[some].double().mean(-1, keepdim=True)
    sd = torch.sqrt((x[some].double() - mean).square().mean(-1, keepdim=True) + EPS)
    xh, t = (x[some].double() - mean) / sd, dy[some].double() * w.double()
    gx = (t - t.mean(-1, keepdim=True) - xh * (t * xh).mean(-1, keepdim=True)) / sd
    for i in range(len(some)):
        assert R.rel(y[some[i]], want[i]) <= tol and R.rel(dx[some[i]], gx[i]) <= tol, some[i]
    gw, gb = torch.zeros(width, dtype=torch.float64, device="cuda"), torch.zeros(width, dtype=torch.float64, device="cuda")
    for lo in range(0, rows, 2048):
        p, d = x[lo:lo + 2048].double(), dy[lo:lo + 2048].double()
        var, mean = torch.var_mean(p, dim=-1, correction=0, keepdim=True)
        gw += (d * (p - mean) / torch.sqrt(var + EPS)).sum(0)
        gb += d.sum(0)
    assert R.rel(dw, gw) <= 4e-6 and R.rel(db, gb) <= 4e-6


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,width", [(3000, 96), (40, 2050), (700, 8192), (41, 20000)])
def test_gradients_over_their_inputs(rows, width, dtype):
    """dx over x and over dy, a block's next row being on its way while this one is written."""
    from paper_1909_05632_amd import ops
    x, dy, w, b = _inputs(rows, width, dtype, width)
    stats = ops.layer_norm(x, w, b, EPS, with_stats=True)[1]
    dx, dw, db = ops.layer_norm_backward(dy, x, w, stats)
    for over in ("x", "dy"):
        x2, dy2 = x.clone(), dy.clone()
        got = ops.layer_norm_backward(dy2, x2, w, stats, dx=x2 if over == "x" else dy2)
        assert got[0] is (x2 if over == "x" else dy2)
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db), over
