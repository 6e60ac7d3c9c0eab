"""Layer norm and its gradients on the GPU against 64-bit references.

Tolerances (2-norm, relative): float32 results carry a few roundings of 2^-24
and sums over a row's W elements (lane sums and a tree: below 32 roundings in a
row), so 64 x 2^-24 = 4e-6; a result rounded once to bfloat16 (8 significant
bits, to nearest) is within 2^-8 of it each.  Weight gradients add `rows` terms in at most 512 strips: 4e-6 as well,
their terms being of random sign."""
import numpy as np
import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

TOL = {torch.float32: 4e-6, torch.bfloat16: 2.0 ** -8}
EPS = 1e-5


def _inputs(rows, width, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = ((torch.randn(rows, width, generator=gen) + 0.7) * torch.exp(torch.randn(rows, 1, generator=gen))).to(dtype)
    dy = torch.randn(rows, width, generator=gen).to(dtype)
    w = 1 + 0.1 * torch.randn(width, generator=gen)
    b = 0.1 * torch.randn(width, generator=gen)
    return x, dy, w, b


def _grads(x, dy, w, b):
    x64 = x.double().requires_grad_(True)
    w64 = w.double().requires_grad_(True)
    b64 = b.double().requires_grad_(True)
    (R.layer_norm(x64, w64, b64, EPS) * dy.double()).sum().backward()
    return x64.grad, w64.grad, b64.grad


# Widths around every change of lanes, registers and vectors, odd ones and the
# ones beyond the registers; one row to many.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,width", [
    (1, 1), (3, 2), (5, 7), (1, 64), (33, 80), (130, 18), (17, 255), (9, 257), (1, 512), (40, 1000), (7, 1024),
    (5, 2050), (3, 4096), (3, 5789), (2, 8192), (2, 8193), (2, 16384), (1, 20001), (2, 40000), (5000, 24)])
def test_forward_and_gradients(rows, width, dtype):
    from paper_1909_05632_amd import ops
    x, dy, w, b = _inputs(rows, width, dtype)
    xd, dyd, wd, bd = (t.cuda() for t in (x, dy, w, b))
    y, stats = ops.layer_norm(xd, wd, bd, EPS, with_stats=True)
    assert y.dtype == dtype and torch.equal(y, ops.layer_norm(xd, wd, bd, EPS))
    dx, dw, db = ops.layer_norm_backward(dyd, xd, wd, stats)
    gx, gw, gb = _grads(x, dy, w, b)
    tol = TOL[dtype]
    assert R.rel(y, R.layer_norm(x, w, b, EPS)) <= tol
    if width == 1:                                   # x - mean is 0: so are dx and dweight
        assert dx.abs().max() == 0 and dw.abs().max() == 0
    elif width == 2:                                 # xh is +-1: dx is what rounding and eps leave of a difference of equals
        assert (dx.double().cpu() - gx).abs().max() <= tol * (stats[:, 1].max().item() * dy.double().abs().max())
    else:
        assert R.rel(dx, gx) <= tol
    if width > 1:
        assert R.rel(dw, gw) <= TOL[torch.float32]
    assert R.rel(db, gb) <= TOL[torch.float32]


def test_gradient_against_differences():
    from paper_1909_05632_amd import ops
    x, dy, w, b = _inputs(6, 50, torch.float32, seed=3)
    _, stats = ops.layer_norm(x.cuda(), w.cuda(), b.cuda(), EPS, with_stats=True)
    dx, dw, db = ops.layer_norm_backward(dy.cuda(), x.cuda(), w.cuda(), stats)
    gen = torch.Generator().manual_seed(4)
    h = 1e-5
    for _ in range(4):
        d = [torch.randn(t.shape, generator=gen).double() for t in (x, w, b)]
        up, down = ((R.layer_norm(x.double() + s * h * d[0], w.double() + s * h * d[1], b.double() + s * h * d[2], EPS)
                     * dy.double()).sum() for s in (1, -1))
        mine = sum((g.double().cpu() * e).sum() for g, e in zip((dx, dw, db), d))
        # the difference's own error is of h^2 = 1e-10, the gradient's of 4e-6 of its norm times that of d
        size = sum(g.double().norm().item() * e.norm().item() for g, e in zip((dx, dw, db), d))
        assert abs((up - down) / (2 * h) - mine) <= 5e-6 * size


def test_rows_at_a_stride_and_odd_addresses():
    from paper_1909_05632_amd import ops
    x, dy, w, b = (t.cuda() for t in _inputs(20, 128, torch.bfloat16))
    y, stats = ops.layer_norm(x, w, b, EPS, with_stats=True)
    wide = torch.zeros(20, 300, dtype=torch.bfloat16, device="cuda")
    for at in (8, 3):                                # rows that keep, and that break, 16-byte alignment
        view = wide[:, at:at + 128]
        view.copy_(x)
        y2, st2 = ops.layer_norm(view, w, b, EPS, with_stats=True)
        assert R.rel(y2, y) <= 2.0 ** -9 and R.rel(st2, stats) <= 4e-6
        dyw = torch.zeros(20, 300, dtype=torch.bfloat16, device="cuda")[:, at:at + 128]
        dyw.copy_(dy)
        a = ops.layer_norm_backward(dy, x, w, stats)
        c = ops.layer_norm_backward(dyw, view, w, stats)
        assert R.rel(c[0], a[0]) <= 2.0 ** -8 and R.rel(c[1], a[1]) <= 4e-6 and R.rel(c[2], a[2]) <= 4e-6
    y3 = ops.layer_norm(x.view(4, 5, 128), w, b, EPS)
    assert torch.equal(y3.view(20, 128), y)


def test_in_place_no_affine_accumulate_and_dx_alone():
    from paper_1909_05632_amd import ops
    for width in (96, 20000):
        x, dy, w, b = (t.cuda() for t in _inputs(12, width, torch.float32))
        y, stats = ops.layer_norm(x, None, None, EPS, with_stats=True)
        assert R.rel(y, R.layer_norm(x, None, None, EPS)) <= 4e-6
        dx, dw, db = ops.layer_norm_backward(dy, x, None, stats)
        one = torch.ones(width, device="cuda")
        dx1, _, _ = ops.layer_norm_backward(dy, x, one, stats)
        assert torch.equal(dx, dx1)
        dw2, db2 = dw.clone(), db.clone()
        only, none1, none2 = ops.layer_norm_backward(dy, x, None, stats, want_params=False)
        assert torch.equal(only, dx) and none1 is None and none2 is None
        ops.layer_norm_backward(dy, x, None, stats, dweight=dw2, dbias=db2, accumulate=True)
        assert torch.equal(dw2, dw + dw) and torch.equal(db2, db + db)
        z = dy.clone()
        got, dw3, db3 = ops.layer_norm_backward(z, x, None, stats, dx=z)     # over dy itself
        assert got is z and torch.equal(z, dx) and torch.equal(dw3, dw) and torch.equal(db3, db)
        ops.layer_norm(x, None, None, EPS, out=x)
        assert torch.equal(x, y)


def test_rows_apart_and_values_that_are_not_finite():
    """A row of NaN or infinity stays alone; constant rows give the bias."""
    from paper_1909_05632_amd import ops
    x, dy, w, b = (t.cuda() for t in _inputs(9, 160, torch.float32))
    y = ops.layer_norm(x, w, b, EPS)
    x2 = x.clone()
    x2[3, 5] = float("nan")
    x2[7, 0] = float("inf")
    x2[8] = 4.0
    y2 = ops.layer_norm(x2, w, b, EPS)
    rest = [0, 1, 2, 4, 5, 6]
    assert torch.equal(y2[rest], y[rest])
    assert y2[3].isnan().all() and y2[7].isnan().any() and torch.equal(y2[8], b)


def test_empty_batch_and_other_stream():
    from paper_1909_05632_amd import ops
    w, b = torch.ones(40, device="cuda"), torch.zeros(40, device="cuda")
    x = torch.empty(0, 40, device="cuda")
    y, stats = ops.layer_norm(x, w, b, EPS, with_stats=True)
    assert y.shape == (0, 40) and stats.shape == (0, 2)
    dx, dw, db = ops.layer_norm_backward(x, x, w, stats)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    x = torch.randn(64, 40, device="cuda")
    want = ops.layer_norm(x, w, b, EPS)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = ops.layer_norm(x, w, b, EPS, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_same_bits_every_time_and_in_a_graph():
    from paper_1909_05632_amd import ops
    x, dy, w, b = (t.cuda() for t in _inputs(3000, 136, torch.bfloat16))
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        y, stats = ops.layer_norm(x, w, b, EPS, with_stats=True)
        want = ops.layer_norm_backward(dy, x, w, stats)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            gy, gstats = ops.layer_norm(x, w, b, EPS, with_stats=True)
            got = ops.layer_norm_backward(dy, x, w, gstats)
    for _ in range(3):
        for t in (gy, *got):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gy, y) and all(torch.equal(a, c) for a, c in zip(got, want))


def test_strips_do_not_meet():
    """Each weight gradient is the sum of its own column, whatever the others hold."""
    from paper_1909_05632_amd import ops
    x, dy, w, b = (t.cuda() for t in _inputs(777, 48, torch.float32))
    _, stats = ops.layer_norm(x, w, b, EPS, with_stats=True)
    _, dw, db = ops.layer_norm_backward(dy, x, w, stats)
    dy2 = dy.clone()
    dy2[:, 10] = 0
    _, dw2, db2 = ops.layer_norm_backward(dy2, x, w, stats)
    assert db2[10] == 0 and dw2[10] == 0
    other = np.r_[0:10, 11:48]
    assert torch.equal(dw2[other], dw[other]) and torch.equal(db2[other], db[other])
