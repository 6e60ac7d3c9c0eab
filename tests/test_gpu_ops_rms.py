"""The residual norm, its 8-bit output and its gradients on the GPU against 64-bit references.

Tolerances (2-norm, relative): float32 results carry a few roundings of 2^-24
and sums over a row's W elements (lane sums and a tree: below 32 roundings in a
row), so 64 x 2^-24 = 4e-6; a result rounded once to bfloat16 is within 2^-8 of
it each (half a step).  Weight gradients add `rows` terms in at most 512 strips:
4e-6 as well, their terms being of random sign.  The sum of x and the residual
is one float32 addition rounded to the type, and q follows from it by two
float32 products, a quotient and a rounding to e4m3: both are compared bit by
bit."""
import pytest
import torch

from tests import ops_ref as R
from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]

TOL = {torch.float32: 4e-6, torch.bfloat16: 2.0 ** -8 + 4e-6}
EPS = 1e-5
F32, BF16 = torch.float32, torch.bfloat16


def _inputs(rows, width, dtype, seed=0):
    gen = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x, r = randn(rows, width).to(dtype), (2 * randn(rows, width) * torch.exp(randn(rows, 1))).to(dtype)
    return x, r, randn(rows, width).to(dtype), randn(rows, width).to(dtype), 1 + 0.1 * randn(width)


def _sum(x, r):
    return (x.float() + r.float()).to(x.dtype)


def _norm(h, w):
    h = h.double()
    return h / torch.sqrt(h.square().mean(-1, keepdim=True) + EPS) * w.double()


def _grads(h, w, dy, dh):
    h, w = h.double().requires_grad_(), w.double().requires_grad_()
    (_norm(h, w) * dy.double()).sum().backward()
    return h.grad + (0 if dh is None else dh.double()), w.grad


def _q(h, w):
    """The 8-bit output and its scales by the definition, in float32 (the scales in 64 bits)."""
    t = h.float() * w
    m = t.abs().amax(-1, keepdim=True)
    q = (t * torch.where(m > 0, 448.0 / m, torch.zeros(()))).to(torch.float8_e4m3fn)
    rms = torch.sqrt(h.double().square().mean(-1, keepdim=True) + EPS)
    return q, (m.double() / rms / 448)[:, 0]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", [
    (1, 1), (3, 2), (5, 7), (1, 64), (33, 80), (130, 18), (17, 255), (9, 257), (1, 512), (40, 1000), (7, 1024),
    (5, 2050), (3, 4096), (3, 5789), (2, 8192), (2, 8193), (2, 16384), (1, 20001), (2, 40000), (5000, 24)])
def test_forward_8bit_and_gradients(rows, width, dtype):
    from paper_1909_05632_amd import ops
    x, r, dy, dh, w = _inputs(rows, width, dtype)
    xd, rd, dyd, dhd, wd = (t.cuda() for t in (x, r, dy, dh, w))
    y, total, rstd = ops.rms_norm(xd, wd, rd, EPS, with_stats=True)
    h = _sum(x, r)
    assert y.dtype == dtype and torch.equal(total.cpu(), h)
    assert R.rel(y, _norm(h, w)) <= TOL[dtype]
    alone = ops.rms_norm(total, wd, eps=EPS)                       # without the residual: the same of its sum
    assert torch.equal(alone, y)
    q, scales, total2, rstd2 = ops.rms_norm(xd, wd, rd, EPS, with_stats=True, quantize=True)
    assert torch.equal(total2, total) and torch.equal(rstd2, rstd)
    q64, s64 = _q(h, w)
    assert torch.equal(q.cpu().view(torch.uint8), q64.view(torch.uint8)) and R.rel(scales, s64) <= 4e-6
    far = (q.cpu().double() * s64[:, None] - _norm(h, w)).abs()
    assert (far <= 2.0 ** -4 * 1.001 * _norm(h, w).abs() + 2.0 ** -10 * 1.001 * s64[:, None]).all()
    for extra, extra64 in ((dhd, dh), (None, None)):
        dx, dw = ops.rms_norm_backward(dyd, total, wd, rstd, dtotal=extra)
        gx, gw = _grads(h, w, dy, extra64)
        if width > 2 or extra is not None:
            assert R.rel(dx, gx) <= TOL[dtype]
        else:                       # one or two elements: what is left of a difference of near equals
            assert (dx.double().cpu() - gx).abs().max() <= TOL[dtype] * (rstd.max().item() * dy.double().abs().max()) * 2
        assert R.rel(dw, gw) <= TOL[F32]


def test_gradient_against_differences():
    from paper_1909_05632_amd import ops
    x, r, dy, dh, w = _inputs(6, 50, F32, seed=3)
    _, total, rstd = ops.rms_norm(x.cuda(), w.cuda(), r.cuda(), EPS, with_stats=True)
    dx, dw = ops.rms_norm_backward(dy.cuda(), total, w.cuda(), rstd, dtotal=dh.cuda())
    h = total.cpu().double()
    gen = torch.Generator().manual_seed(4)
    e = 1e-5
    for _ in range(4):
        a, b = (torch.randn(t.shape, generator=gen).double() for t in (h, w))
        up, down = ((_norm(h + s * e * a, w.double() + s * e * b) * dy.double()).sum() + ((h + s * e * a) * dh.double()).sum()
                    for s in (1, -1))
        mine = (dx.double().cpu() * a).sum() + (dw.double().cpu() * b).sum()
        # the difference's own error is of e^2 = 1e-10, the gradient's of 4e-6 of its norm times that of the direction
        size = dx.double().norm().item() * a.norm().item() + dw.double().norm().item() * b.norm().item()
        assert abs((up - down) / (2 * e) - mine) <= 5e-6 * size


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_at_a_stride_odd_addresses_and_more_axes(dtype):
    from paper_1909_05632_amd import ops
    x, r, dy, dh, w = (t.cuda() for t in _inputs(20, 128, dtype))
    y, total, rstd = ops.rms_norm(x, w, r, EPS, with_stats=True)
    q, scales, _ = ops.rms_norm(x, w, r, EPS, quantize=True)
    dx, dw = ops.rms_norm_backward(dy, total, w, rstd, dtotal=dh)
    odd = torch.zeros(129, device="cuda")[1:].copy_(w)

    def wide(t, at):
        return torch.zeros(20, 300, dtype=dtype, device="cuda")[:, at:at + 128].copy_(t)

    for at in (8, 3):                                # rows that keep, and that break, 16-byte alignment
        for weight in (w, odd):
            y2, total2, rstd2 = ops.rms_norm(wide(x, at), weight, wide(r, 8), EPS, with_stats=True)
            assert torch.equal(total2, total) and R.rel(y2, y) <= TOL[dtype] and R.rel(rstd2, rstd) <= 4e-6
            q2, scales2, _ = ops.rms_norm(wide(x, at), weight, wide(r, 8), EPS, quantize=True)
            assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and R.rel(scales2, scales) <= 4e-6
            dx2, dw2 = ops.rms_norm_backward(wide(dy, 8), wide(total, at), weight, rstd, dtotal=wide(dh, at))
            assert R.rel(dx2, dx) <= 2 * TOL[dtype] and R.rel(dw2, dw) <= 4e-6
    y3, t3 = ops.rms_norm(x.view(4, 5, 128), w, r.view(4, 5, 128), EPS)
    assert torch.equal(y3.view(20, 128), y) and torch.equal(t3.view(20, 128), total)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [96, 333, 20000])
def test_results_over_the_inputs(width, dtype):
    from paper_1909_05632_amd import ops
    x, r, dy, dh, w = (t.cuda() for t in _inputs(12, width, dtype))
    y, total, rstd = ops.rms_norm(x, w, r, EPS, with_stats=True)
    a, b = x.clone(), r.clone()
    got = ops.rms_norm(a, w, b, EPS, out=a, total=b)                 # y over x, the sum over the residual
    assert got[0] is a and got[1] is b and torch.equal(a, y) and torch.equal(b, total)
    a, b = x.clone(), r.clone()
    ops.rms_norm(a, w, b, EPS, out=b, total=a)                       # and the other way
    assert torch.equal(b, y) and torch.equal(a, total)
    dx, dw = ops.rms_norm_backward(dy, total, w, rstd, dtotal=dh)
    for i in range(3):
        t = [dy.clone(), total.clone(), dh.clone()]
        got, dw2 = ops.rms_norm_backward(t[0], t[1], w, rstd, dtotal=t[2], dx=t[i])
        assert got is t[i] and torch.equal(got, dx) and torch.equal(dw2, dw)
    dw3 = dw.clone()
    ops.rms_norm_backward(dy, total, w, rstd, dtotal=dh, dweight=dw3, accumulate=True)
    assert torch.equal(dw3, dw + dw)
    only, none = ops.rms_norm_backward(dy, total, w, rstd, dtotal=dh, want_params=False)
    assert torch.equal(only, dx) and none is None
    one = torch.ones(width, device="cuda")
    assert torch.equal(ops.rms_norm(x, None, eps=EPS), ops.rms_norm(x, one, eps=EPS))


def test_rows_apart_zeros_and_values_that_are_not_finite():
    """A row of NaN or infinity stays alone; a row of zeros gives zeros and a scale of 0."""
    from paper_1909_05632_amd import ops
    for width in (160, 9001):
        x, _, _, _, w = (t.cuda() for t in _inputs(9, width, F32))
        y, (q, scales) = ops.rms_norm(x, w, eps=EPS), ops.rms_norm(x, w, eps=EPS, quantize=True)
        x2 = x.clone()
        x2[3, 5], x2[7, 0], x2[8] = float("nan"), float("inf"), 0
        y2, (q2, scales2) = ops.rms_norm(x2, w, eps=EPS), ops.rms_norm(x2, w, eps=EPS, quantize=True)
        rest = [0, 1, 2, 4, 5, 6]
        assert torch.equal(y2[rest], y[rest]) and torch.equal(scales2[rest], scales[rest])
        assert torch.equal(q2.view(torch.uint8)[rest], q.view(torch.uint8)[rest])
        assert y2[3].isnan().all() and y2[7, 0].isnan() and scales2[[3, 7]].isnan().all()
        assert not y2[8].any() and not q2[8].float().any() and scales2[8] == 0


def test_empty_batch_other_stream_and_same_bits_in_a_graph():
    from paper_1909_05632_amd import ops
    w = torch.ones(40, device="cuda")
    e = torch.empty(0, 40, device="cuda")
    y, total, rstd = ops.rms_norm(e, w, e, EPS, with_stats=True)
    assert y.shape == total.shape == (0, 40) and rstd.shape == (0,)
    dx, dw = ops.rms_norm_backward(e, e, w, rstd)
    assert dx.shape == (0, 40) and not dw.any()
    x, r, dy, dh, w = (t.cuda() for t in _inputs(3000, 136, BF16))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    y, total, rstd = ops.rms_norm(x, w, r, EPS, with_stats=True, stream=st)
    want = [y, total, *ops.rms_norm_backward(dy, total, w, rstd, dtotal=dh, stream=st)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st), torch.cuda.graph(graph, stream=st):
        gy, gt, gr = ops.rms_norm(x, w, r, EPS, with_stats=True)
        got = [gy, gt, *ops.rms_norm_backward(dy, gt, w, gr, dtotal=dh)]
    for _ in range(3):
        for t in got:
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_more_rows_than_a_grid_takes_at_once():
    """Blocks walk the rows: each row of a long batch is the one it is in a short one."""
    from paper_1909_05632_amd import ops
    x, r, _, _, w = (t.cuda() for t in _inputs(70001, 520, BF16))
    y, total = ops.rms_norm(x, w, r, EPS)
    for lo in (0, 16380, 65530, 70000):
        a, b = ops.rms_norm(x[lo:lo + 9], w, r[lo:lo + 9], EPS)
        assert torch.equal(a, y[lo:lo + 9]) and torch.equal(b, total[lo:lo + 9])


def test_rows_of_tiny_values_in_8_bits():
    """448 / m is infinite where m is below 1.3e-36; q and the scales are as they are for any other row.
    (y is q scale to half a step of e4m3, 2^-4 of it or 2^-10 of 448, and a few 2^-24.)"""
    from paper_1909_05632_amd import ops
    for width in (96, 9000):
        for size in (3e-36, 1e-36, 2.0 ** -121, 1e-37):
            x = (size * torch.linspace(-1, 1, width)).expand(3, width).contiguous()
            q, scales = ops.rms_norm(x.cuda(), eps=EPS, quantize=True)
            y = x.double() / EPS ** 0.5
            got = q.cpu().double() * scales.cpu().double()[:, None]
            largest = y.abs().max()
            assert ((got - y).abs() <= (y.abs() * 2.0 ** -4).clamp(min=largest / 448 * 2.0 ** -10) + 1e-5 * largest).all()
            assert q.float().abs().max() == 448


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_whose_squares_overflow(dtype):
    """Finite values above 2^64 have an infinite sum of squares: y is 0 by its formula, and the scale NaN, so that
    such a row is not taken for one of zeros.  The rows beside it are as they were."""
    from paper_1909_05632_amd import ops
    for width in (160, 9001):
        x, r, _, _, w = (t.cuda() for t in _inputs(6, width, dtype))
        y, total, q, scales = *ops.rms_norm(x, w, r, EPS), *ops.rms_norm(x, w, r, EPS, quantize=True)[:2]
        x2 = x.clone()
        x2[1], x2[3, width // 2], x2[4] = 2e19, -1e30, 3e38
        y2, total2, q2, scales2 = *ops.rms_norm(x2, w, r, EPS), *ops.rms_norm(x2, w, r, EPS, quantize=True)[:2]
        rest, over = [0, 2, 5], [1, 3, 4]
        assert torch.equal(y2[rest], y[rest]) and torch.equal(scales2[rest], scales[rest])
        assert torch.equal(q2.view(torch.uint8)[rest], q.view(torch.uint8)[rest])
        assert torch.isfinite(total2).all() and not y2[over].any() and scales2[over].isnan().all()
