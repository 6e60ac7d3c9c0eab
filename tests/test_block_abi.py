"""The C ABI and the torch functions of a recurrent block's operators: bad
arguments are refused with a status and a text before any launch.  None of it
needs a GPU: every call below ends in the checks (or has nothing to do)."""
import pytest
import torch

from paper_1909_05632_amd import binding as B
from paper_1909_05632_amd import ops

P = 256          # a pointer that is not NULL; no call below gets as far as using it


def _err(status, want, text):
    assert status == want, (status, ops.reuse_ops_last_error())
    assert text in ops.reuse_ops_last_error(), ops.reuse_ops_last_error()


def _caller(call, **base):
    return lambda **kw: call(*{**base, **kw}.values())


@pytest.fixture
def calls(monkeypatch):
    """The functions on CPU tensors; every call that would have been launched."""
    seen = []
    monkeypatch.setattr(ops, "_data", lambda x, what: ops._CODES[x.dtype])
    monkeypatch.setattr(ops, "_launch", lambda device, *call: seen.append(call))
    return seen


# ------------------------------------------------------------------ residual norm

def test_rms_norm_arguments():
    L = ops.load_ops()
    call = _caller(L.reuse_ops_rms_norm, rows=4, width=8, x=P, xs=8, dtype=B.RN_F32, residual=2 * P, rs=8, w=P, eps=1e-5,
                   y=3 * P, q=None, scales=None, total=4 * P, rstd=None, stream=None)
    _err(call(rows=-1), B.RN_EINVAL, "rows")
    _err(call(width=0), B.RN_EINVAL, "width")
    _err(call(dtype=B.RN_U8), B.RN_EINVAL, "dtype")
    _err(call(x=None), B.RN_EINVAL, "NULL")
    _err(call(y=None), B.RN_EINVAL, "NULL")
    _err(call(q=P), B.RN_EINVAL, "go together")
    _err(call(scales=P), B.RN_EINVAL, "go together")
    _err(call(residual=None), B.RN_EINVAL, "no total")
    _err(call(xs=7), B.RN_EINVAL, "stride")
    _err(call(rs=7), B.RN_EINVAL, "stride")
    _err(call(total=3 * P), B.RN_EINVAL, "two arrays")
    _err(call(y=P, xs=9), B.RN_EINVAL, "not contiguous")
    _err(call(total=2 * P, rs=9), B.RN_EINVAL, "not contiguous")
    _err(call(eps=-1.0), B.RN_EINVAL, "eps")
    _err(call(eps=float("nan")), B.RN_EINVAL, "eps")
    assert call(rows=0, x=None, y=None) == B.RN_OK
    need = L.reuse_ops_rms_norm_backward_scratch_bytes(4, 8)
    assert need > 0 and need % 256 == 0
    assert L.reuse_ops_rms_norm_backward_scratch_bytes(-1, 8) == L.reuse_ops_rms_norm_backward_scratch_bytes(4, 0) == 0
    back = _caller(L.reuse_ops_rms_norm_backward, rows=4, width=8, dy=P, dys=8, total=2 * P, ts=8, dtype=B.RN_F32, w=None,
                   rstd=P, dtotal=3 * P, dts=8, dx=4 * P, dw=P, acc=0, scratch=P, bytes=need, stream=None)
    _err(back(rows=1 << 50), B.RN_EINVAL, "rows")
    _err(back(dtype=9), B.RN_EINVAL, "dtype")
    for name in ("dy", "total", "rstd", "dx"):
        _err(back(**{name: None}), B.RN_EINVAL, "NULL")
    for name in ("dys", "ts", "dts"):
        _err(back(**{name: 7}), B.RN_EINVAL, "stride")
    for name, p in (("dys", P), ("ts", 2 * P), ("dts", 3 * P)):
        _err(back(**{name: 9, "dx": p}), B.RN_EINVAL, "not contiguous")
    _err(back(scratch=None), B.RN_EINVAL, "scratch")
    _err(back(scratch=P + 4), B.RN_EINVAL, "aligned")
    _err(back(bytes=need - 1), B.RN_ENOSPACE, "need")
    assert back(rows=0, dw=None) == B.RN_OK


def test_rms_norm_tensors(calls):
    x, w, f8 = torch.zeros(3, 8), torch.ones(8), torch.zeros(3, 8, dtype=torch.float8_e4m3fn)
    stats = torch.zeros(3)
    assert ops.rms_norm(x, w).shape == (3, 8)
    assert [t.dtype for t in ops.rms_norm(x, w, x, with_stats=True, quantize=True)] == [
        torch.float8_e4m3fn, torch.float32, torch.float32, torch.float32]
    calls.clear()
    for bad, kw in ((ValueError, dict(residual=x[:2])), (ValueError, dict(residual=x.bfloat16())), (TypeError, dict(residual=1.0)),
                    (ValueError, dict(weight=w[:7])), (TypeError, dict(weight=w.double())), (ValueError, dict(total=x)),
                    (ValueError, dict(scales=stats)), (TypeError, dict(out=f8)), (TypeError, dict(out=x, quantize=True)),
                    (ValueError, dict(quantize=True, scales=stats[:2])), (ValueError, dict(out=torch.zeros(8, 3).t()))):
        with pytest.raises(bad):
            ops.rms_norm(x, **kw)
    for bad, args, kw in ((ValueError, (x[:2], x, w, stats), {}), (ValueError, (x, x, w, stats[:2]), {}),
                          (TypeError, (x, x, w, None), {}), (ValueError, (x, x, w, stats), dict(dtotal=x[:1])),
                          (ValueError, (x, x, w, stats), dict(accumulate=True)), (TypeError, (x, x, w, stats), dict(dx=x.bfloat16()))):
        with pytest.raises(bad):
            ops.rms_norm_backward(*args, **kw)
    with pytest.raises(ValueError, match="width"):
        ops.rms_norm(torch.empty(1, (1 << 32) + 8, device="meta"))
    for i in range(3):
        some = [x, w, x]
        some[i] = some[i].clone().requires_grad_()
        with pytest.raises(ValueError, match="requires grad"):
            ops.rms_norm(*some)
    for i in range(5):
        some = [x, x, w, stats, x]
        some[i] = some[i].clone().requires_grad_()
        with pytest.raises(ValueError, match="requires grad"):
            ops.rms_norm_backward(*some)
    assert not calls


# ------------------------------------------------------------------ log-probabilities

def test_log_probs_arguments():
    L = ops.load_ops()
    base = dict(n=2, vocab=6, logits=P, stride=6, dtype=B.RN_F32, tokens=P, temperature=1.0, top=2, lp=P, h=P, ids=P, tlp=P,
                stats=None, scratch=P, bytes=256, stream=None)
    call = _caller(L.reuse_ops_log_probs, **base)
    for kw, text in ((dict(n=-1), "n must"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 20) + 1), "vocab"), (dict(top=-1), "top"),
                     (dict(top=7), "top"), (dict(vocab=1000, top=65), "top"), (dict(dtype=B.RN_U8), "dtype"),
                     (dict(temperature=0.0), "temperature"), (dict(temperature=-1.0), "temperature"),
                     (dict(temperature=float("nan")), "temperature"), (dict(temperature=float("inf")), "temperature"),
                     (dict(temperature=1e-39), "temperature"), (dict(logits=None), "NULL"), (dict(tokens=None), "NULL"),
                     (dict(ids=None), "NULL"), (dict(tlp=None), "NULL"), (dict(stride=5), "stride"), (dict(scratch=None), "scratch"),
                     (dict(scratch=P + 8), "aligned")):
        _err(call(**kw), B.RN_EINVAL, text)
    _err(call(bytes=255), B.RN_ENOSPACE, "need")
    assert call(n=0, logits=None, tokens=None) == B.RN_OK
    size = L.reuse_ops_log_probs_scratch_bytes
    assert size(-1, 6, 0) == size(2, 0, 0) == size(2, 6, 7) == size(2, 1000, 65) == 0
    assert size(2, 6, 2) == 256 == size(1 << 20, 1 << 20, 64) == size((1 << 31) - 1, 1 << 20, 0)
    assert size(1, 1 << 20, 64) >= 32 * 12 and size(1, 1 << 20, 64) % 256 == 0
    _err(_caller(L.reuse_ops_log_probs, **{**base, "vocab": 1 << 20, "stride": 1 << 20, "n": 1})(), B.RN_ENOSPACE, "need")
    back = _caller(L.reuse_ops_log_probs_backward, n=2, vocab=6, logits=P, stride=6, dtype=B.RN_F32, tokens=P, temperature=1.0,
                   stats=P, dlp=P, dh=P, dl=2 * P, ds=6, stream=None)
    for kw, text in ((dict(n=-1), "n must"), (dict(vocab=0), "vocab"), (dict(dtype=7), "dtype"), (dict(temperature=0.0), "temperature"),
                     (dict(logits=None), "NULL"), (dict(tokens=None), "NULL"), (dict(stats=None), "NULL"), (dict(dl=None), "NULL"),
                     (dict(stride=5), "stride"), (dict(ds=5), "stride"), (dict(dl=P, ds=7), "same stride")):
        _err(back(**kw), B.RN_EINVAL, text)
    assert back(n=0, logits=None) == B.RN_OK


def test_log_probs_tensors(calls):
    x, t, one, st = torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), torch.ones(3), torch.zeros(3, 4)
    assert [tuple(g.shape) for g in ops.log_probs(x, t, top=2, with_stats=True)] == [(3,), (3,), (3, 2), (3, 2), (3, 4)]
    assert ops.log_probs_backward(one, None, x, t, st).shape == (3, 8)
    calls.clear()
    for bad, args, kw in ((ValueError, (x[0], t), {}), (ValueError, (x, t[:2]), {}), (TypeError, (x, t.long()), {}),
                          (ValueError, (x, t), dict(top=9)), (ValueError, (x, t), dict(top=-1)), (TypeError, (x, t), dict(top=1.5)),
                          (ValueError, (torch.zeros(8, 3).t(), t), {}), (ValueError, (torch.zeros(3, 0), t), {}),
                          (ValueError, (torch.empty((1 << 32) + 2, 4, device="meta"), t), {})):
        with pytest.raises(bad):
            ops.log_probs(*args, **kw)
    for bad, args, kw in ((ValueError, (one[:2], None, x, t, st), {}), (TypeError, (one, one.double(), x, t, st), {}),
                          (ValueError, (one, one, x, t, st[:, :3]), {}), (TypeError, (one, one, x, t, None), {}),
                          (ValueError, (one, one, x, t, st), dict(dlogits=x.bfloat16())),
                          (ValueError, (one, one, x, t, st), dict(dlogits=torch.zeros(8, 3).t()))):
        with pytest.raises(bad):
            ops.log_probs_backward(*args, **kw)
    with pytest.raises(ValueError, match="requires grad"):
        ops.log_probs(x.clone().requires_grad_(), t)
    for i in (0, 1, 2, 4):
        some = [one, one, x, t, st]
        some[i] = some[i].clone().requires_grad_()
        with pytest.raises(ValueError, match="requires grad"):
            ops.log_probs_backward(*some)
    assert not calls


# ------------------------------------------------------------------ short convolution

def _conv(n=2, channels=8, taps=4, tokens=10, dtype=B.RN_F32, silu=1, stride=8):
    return ops.rn_conv_shape(n, channels, taps, tokens, dtype, silu, stride)


def test_causal_conv_arguments():
    L, ref = ops.load_ops(), ops.ctypes.byref
    bad = ((dict(n=-1), "n must"), (dict(n=65536), "n must"), (dict(channels=0), "channels"), (dict(channels=65537), "channels"),
           (dict(taps=0), "taps"), (dict(taps=5), "taps"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"),
           (dict(n=0), "without sequences"), (dict(dtype=B.RN_U8), "dtype"), (dict(stride=7), "stride"), (dict(stride=1 << 23), "2^23"))
    s = _conv()
    need = L.reuse_ops_causal_conv_backward_scratch_bytes(ref(s))
    assert need >= 8 * 5 * 4 and need % 256 == 0
    fwd = _caller(L.reuse_ops_causal_conv, shape=ref(s), x=P, w=P, b=None, off=P, window=2 * P, final=3 * P, out=4 * P, stream=None)
    back = _caller(L.reuse_ops_causal_conv_backward, shape=ref(s), x=P, w=P, b=None, off=P, window=2 * P, dout=3 * P, dfinal=4 * P,
                   dx=5 * P, dw=P, db=P, dwindow=6 * P, scratch=P, bytes=need, stream=None)
    one = _conv(tokens=2)
    step = _caller(L.reuse_ops_causal_conv_step, shape=ref(one), x=P, w=P, b=None, ids=None, slots=2, window=2 * P, out=3 * P,
                   stream=None)
    for kw, text in bad:
        t = _conv(**kw)
        assert L.reuse_ops_causal_conv_backward_scratch_bytes(ref(t)) == 0
        for call in (fwd, back, step):
            _err(call(shape=ref(t)), B.RN_EINVAL, text)
    assert L.reuse_ops_causal_conv_backward_scratch_bytes(ref(_conv(tokens=(1 << 31) - 64))) > 0
    most = _conv(tokens=(1 << 31) - 63)
    assert L.reuse_ops_causal_conv_backward_scratch_bytes(ref(most)) == 0
    for call in (fwd, back, step):
        _err(call(shape=ref(most)), B.RN_EINVAL, "2^31 - 64")
        _err(call(shape=None), B.RN_EINVAL, "shape")
    for call in (fwd, back):
        t = _conv(n=3)
        _err(call(shape=ref(t), off=None), B.RN_EINVAL, "multiple")
    for name in ("x", "w", "out"):
        _err(fwd(**{name: None}), B.RN_EINVAL, "NULL")
    _err(fwd(out=P), B.RN_EINVAL, "out must not be x")
    _err(fwd(final=2 * P), B.RN_EINVAL, "first ones")
    for name in ("x", "w", "dout", "dx", "dw", "db", "scratch"):
        _err(back(**{name: None}), B.RN_EINVAL, "NULL")
    _err(back(dx=P), B.RN_EINVAL, "neither")
    _err(back(dx=3 * P), B.RN_EINVAL, "neither")
    _err(back(dwindow=4 * P), B.RN_EINVAL, "neither")
    _err(back(scratch=P + 8), B.RN_EINVAL, "aligned")
    _err(back(bytes=need - 1), B.RN_ENOSPACE, "need")
    _err(step(shape=ref(s)), B.RN_EINVAL, "one token a stream")
    _err(step(slots=1), B.RN_EINVAL, "slots")
    _err(step(slots=-1, ids=P), B.RN_EINVAL, "slots")
    for name in ("x", "w", "window", "out"):
        _err(step(**{name: None}), B.RN_EINVAL, "NULL")
    wide = _conv(tokens=2, stride=9)
    _err(step(shape=ref(wide), out=P), B.RN_EINVAL, "not contiguous")
    _err(step(out=2 * P), B.RN_EINVAL, "two arrays")
    none = _conv(n=0, tokens=0)
    assert fwd(shape=ref(none)) == step(shape=ref(none), slots=0) == B.RN_OK


def test_causal_conv_tensors(calls):
    x, w, b, s = torch.zeros(6, 8), torch.zeros(8, 4), torch.zeros(8), torch.zeros(2, 3, 8)
    off = torch.tensor([0, 2, 6], dtype=torch.int32)
    out, final = ops.causal_conv(x, w, b, off, state=s)
    assert out.shape == (6, 8) and final.shape == (2, 3, 8)
    assert [tuple(g.shape) for g in ops.causal_conv_backward(out, x, w, b, off, state=s)] == [(6, 8), (8, 4), (8,), (2, 3, 8)]
    assert ops.causal_conv_step(x[:2], w, s, b).shape == (2, 8)
    calls.clear()
    for bad, args, kw in ((ValueError, (x[0], w), dict(n=1)), (ValueError, (x, w[:7]), dict(n=1)), (ValueError, (x, b), dict(n=1)),
                          (ValueError, (x, torch.zeros(8, 5)), dict(n=1)), (TypeError, (x, w.double()), dict(n=1)),
                          (ValueError, (x, w, b[:3]), dict(n=1)), (ValueError, (x, w), {}), (ValueError, (x, w), dict(n=4)),
                          (ValueError, (x, w, b, off), dict(state=s[:1])), (TypeError, (x, w, b, off), dict(state=s.bfloat16())),
                          (ValueError, (x, w, b, off), dict(final=s[:, :2])), (ValueError, (x, w, b, off), dict(out=x[:5])),
                          (TypeError, (x, w, b, off.long()), {}), (ValueError, (torch.zeros(8, 6).t(), w), dict(n=1))):
        with pytest.raises(bad):
            ops.causal_conv(*args, **kw)
    for bad, kw in ((ValueError, dict(state=s[:1])), (ValueError, dict(state=s[:, :2].contiguous())),
                    (TypeError, dict(state=s, stream_ids=off.long())), (ValueError, dict(state=s, out=x))):
        with pytest.raises(bad):
            ops.causal_conv_step(x[:2], w, **kw)
    with pytest.raises(ValueError, match="dout|shape"):
        ops.causal_conv_backward(out[:3], x, w, b, off)
    with pytest.raises(TypeError, match="dfinal"):
        ops.causal_conv_backward(out, x, w, b, off, dfinal=s.bfloat16())
    for call, args in ((ops.causal_conv, [x, w, b, off, None, s]), (ops.causal_conv_backward, [out, x, w, b, off, None, s, s]),
                       (ops.causal_conv_step, [x[:2], w, s, b])):
        for i, t in enumerate(args):
            if isinstance(t, torch.Tensor) and t.is_floating_point():
                some = list(args)
                some[i] = t.clone().requires_grad_()
                with pytest.raises(ValueError, match="requires grad"):
                    call(*some)
    assert not calls


# ------------------------------------------------------------------ selective scan

def _scan(n=2, channels=8, groups=2, states=4, tokens=10, dtype=B.RN_F32, softplus=1, u=8, dt=8, b=8, c=8, z=8):
    return ops.rn_scan_shape(n, channels, groups, states, tokens, dtype, softplus, u, dt, b, c, z)


def test_scan_arguments():
    L, ref = ops.load_ops(), ops.ctypes.byref
    sizes = (L.reuse_ops_scan_saved_bytes, L.reuse_ops_scan_scratch_bytes, L.reuse_ops_scan_backward_scratch_bytes)
    s, one, none = _scan(), _scan(tokens=2), _scan(n=0, tokens=0)
    given = {k: P for k in ("u", "dt", "b", "c", "a", "d", "z", "dt_bias")}
    into = {k: P for k in ("du", "ddt", "db", "dc", "dz", "da", "dd", "ddt_bias", "dstate")}
    inputs = lambda **kw: ref(ops.rn_scan_inputs(**{**given, **kw}))  # noqa: E731
    grads = lambda **kw: ref(ops.rn_scan_grads(**{**into, **kw}))  # noqa: E731
    saved, fwd_bytes, bwd_bytes = (f(ref(s)) for f in sizes)
    assert all(x >= 256 and x % 256 == 0 for x in (saved, fwd_bytes, bwd_bytes)) and saved >= 2 * 8 * 4 * 4
    fwd = _caller(L.reuse_ops_scan_forward, shape=ref(s), given=inputs(), off=P, state=None, final=None, out=P, saved=None,
                  saved_bytes=0, scratch=P, bytes=fwd_bytes, stream=None)
    back = _caller(L.reuse_ops_scan_backward, shape=ref(s), given=inputs(), off=P, saved=P, saved_bytes=saved, dout=P, dfinal=None,
                   grads=grads(), scratch=P, bytes=bwd_bytes, stream=None)
    step = _caller(L.reuse_ops_scan_step, shape=ref(one), given=inputs(), ids=None, slots=2, state=P, out=2 * P, stream=None)
    for kw, text in ((dict(n=-1), "n must"), (dict(n=65536), "n must"), (dict(channels=0), "channels"), (dict(groups=0), "channels"),
                     (dict(channels=65538), "channels"), (dict(groups=3), "channels"), (dict(states=0), "states"),
                     (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(n=0), "without sequences"),
                     (dict(dtype=B.RN_U8), "dtype"), (dict(u=7), "stride"), (dict(dt=7), "stride"), (dict(b=7), "stride"),
                     (dict(c=7), "stride"), (dict(u=1 << 23), "2^23"), (dict(b=1 << 23), "2^23")):
        t = _scan(**kw)
        assert all(f(ref(t)) == 0 for f in sizes), kw
        for call in (fwd, back, step):
            _err(call(shape=ref(t)), B.RN_EINVAL, text)
    wide = _scan(states=65, b=130, c=130)
    assert all(f(ref(wide)) == 0 for f in sizes) and all(f(None) == 0 for f in sizes)
    for call in (fwd, back, step):
        _err(call(shape=ref(wide)), B.RN_EUNSUPPORTED, "64")
        _err(call(shape=None), B.RN_EINVAL, "shape")
        _err(call(given=None), B.RN_EINVAL, "inputs")
        for name in ("u", "dt", "b", "c", "a"):
            _err(call(given=inputs(**{name: None})), B.RN_EINVAL, "NULL")
        for t in (_scan(tokens=2, z=7), _scan(tokens=2, z=1 << 23)):
            _err(call(shape=ref(t)), B.RN_EINVAL, "stride")
    odd = _scan(n=3)
    for call in (fwd, back):
        _err(call(shape=ref(odd), off=None), B.RN_EINVAL, "multiple")
        _err(call(scratch=None), B.RN_EINVAL, "scratch")
        _err(call(scratch=P + 8), B.RN_EINVAL, "aligned")
        _err(call(bytes=255), B.RN_ENOSPACE, "scratch")
    _err(fwd(out=None), B.RN_EINVAL, "NULL")
    _err(fwd(saved=P, saved_bytes=saved - 1), B.RN_ENOSPACE, "saved")
    for name in ("du", "ddt", "db", "dc", "da"):
        _err(back(grads=grads(**{name: None})), B.RN_EINVAL, "NULL")
    _err(back(grads=None), B.RN_EINVAL, "gradients")
    _err(back(dout=None), B.RN_EINVAL, "NULL")
    _err(back(saved=None), B.RN_EINVAL, "NULL")
    _err(back(saved_bytes=saved - 1), B.RN_ENOSPACE, "saved")
    _err(back(given=inputs(z=None)), B.RN_EINVAL, "dz without z")
    _err(back(dfinal=P), B.RN_EINVAL, "dfinal")
    _err(step(shape=ref(s)), B.RN_EINVAL, "one token a stream")
    _err(step(slots=1), B.RN_EINVAL, "slots")
    _err(step(slots=-1, ids=P), B.RN_EINVAL, "slots")
    _err(step(state=None), B.RN_EINVAL, "NULL")
    _err(step(out=None), B.RN_EINVAL, "NULL")
    apart = _scan(tokens=2, u=9)
    _err(step(shape=ref(apart), out=P), B.RN_EINVAL, "not contiguous")
    for t in (_scan(tokens=2, dt=9), _scan(tokens=2, z=9)):
        _err(step(shape=ref(t), out=P), B.RN_EINVAL, "not contiguous")
    for name in ("b", "c"):
        _err(step(given=inputs(**{name: 2 * P})), B.RN_EINVAL, "neither b nor c")
    for name in ("u", "dt", "b", "c", "z"):
        _err(fwd(given=inputs(**{name: 2 * P}), out=2 * P), B.RN_EINVAL, "one of the inputs")
        for grad in ("du", "ddt", "db", "dc", "dz"):
            away = {k: 9 * P for k in ("du", "ddt", "db", "dc", "dz")}
            _err(back(given=inputs(**{name: 2 * P}), dout=3 * P, grads=grads(**{**away, grad: 2 * P})), B.RN_EINVAL, "lies over")
            _err(back(dout=3 * P, grads=grads(**{**away, grad: 3 * P})), B.RN_EINVAL, "lies over")
    assert fwd(shape=ref(none), scratch=None) == step(shape=ref(none), slots=0, state=None) == B.RN_OK


def test_scan_sizes_stay_in_bounds():
    """Scratch and saved bytes grow with the tokens, not with sequences times channels times states."""
    L, ref = ops.load_ops(), ops.ctypes.byref
    many = ops.rn_scan_shape(65535, 4096, 1, 16, 65535, B.RN_BF16, 1, 4096, 4096, 16, 16, 4096)
    long = ops.rn_scan_shape(1, 4096, 1, 16, 1 << 20, B.RN_BF16, 1, 4096, 4096, 16, 16, 4096)
    state = 4096 * 16 * 4
    assert L.reuse_ops_scan_saved_bytes(ref(long)) <= ((1 << 16) + 1) * state + 512
    assert L.reuse_ops_scan_scratch_bytes(ref(long)) <= 1 << 30
    sums = 64 * 65535 * 2 * 16 * 4
    # the sums of b's and c's gradients, and parts of a bounded number of blocks; ends of chunks that 65535 tokens can have
    assert L.reuse_ops_scan_backward_scratch_bytes(ref(many)) <= sums + (1 << 28)


def test_scan_tensors(calls):
    t, n = 6, 2
    u, b, a, d, s = torch.zeros(t, 8), torch.zeros(t, 2, 4), torch.zeros(8, 4), torch.zeros(8), torch.zeros(n, 8, 4)
    off = torch.tensor([0, 2, 6], dtype=torch.int32)
    out, final, saved = ops.scan_forward(u, u, a, b, b, d, u, d, seq_off=off, state=s, save=True)
    got = ops.scan_backward(out, u, u, a, b, b, d, u, d, seq_off=off, saved=saved)
    assert [tuple(g.shape) for g in got] == [(6, 8), (6, 8), (8, 4), (6, 2, 4), (6, 2, 4), (8,), (6, 8), (8,), (2, 8, 4)]
    bare = ops.scan_backward(out, u, u, a, b, b, seq_off=off, saved=saved, want_dstate=False)
    assert [g is None for g in bare] == [False] * 5 + [True] * 4
    assert ops.scan_step(u[:2], u[:2], a, b[:2], b[:2], s).shape == (2, 8)
    calls.clear()
    for bad, args, kw in ((ValueError, (u[0], u, a, b, b), dict(n=1)), (ValueError, (u, u[:5], a, b, b), dict(n=1)),
                          (ValueError, (u, u.bfloat16(), a, b, b), dict(n=1)), (ValueError, (u, u, a[:7], b, b), dict(n=1)),
                          (TypeError, (u, u, a.bfloat16(), b, b), dict(n=1)), (ValueError, (u, u, a, b[:, :, :3], b), dict(n=1)),
                          (ValueError, (u, u, a, torch.zeros(t, 3, 4), torch.zeros(t, 3, 4)), dict(n=1)),
                          (ValueError, (u, u, a, b.transpose(1, 2), b), dict(n=1)), (ValueError, (u, u, a, b, b), {}),
                          (ValueError, (u, u, a, b, b), dict(n=4)), (ValueError, (u, u, a, b, b, d[:3]), dict(n=1)),
                          (ValueError, (u, u, a, b, b, d, u[:, :4]), dict(n=1)), (ValueError, (u, u, a, b, b), dict(n=1, state=s)),
                          (ValueError, (u, u, a, b, b), dict(n=2, final=s[:1])), (ValueError, (u, u, a, b, b), dict(n=2, out=u[:5])),
                          (ValueError, (u.t(), u, a, b, b), dict(n=1)), (TypeError, (u, u, a, b, b), dict(seq_off=off.long()))):
        with pytest.raises(bad):
            ops.scan_forward(*args, **kw)
    big = torch.zeros(t, 1, 65)
    for call, kw in ((ops.scan_forward, {}), (ops.scan_backward, dict(saved=saved))):
        with pytest.raises(B.ReuseNetError, match="64"):
            call(*([u] if call is ops.scan_backward else []), u, u, torch.zeros(8, 65), big, big, n=1, **kw)
    with pytest.raises(TypeError, match="saved"):
        ops.scan_backward(out, u, u, a, b, b, seq_off=off)
    with pytest.raises(ValueError, match="saved"):
        ops.scan_backward(out, u, u, a, b, b, seq_off=off, saved=saved[:-1])
    with pytest.raises(ValueError, match="slots"):
        ops.scan_step(u, u, a, b, b, s)
    for call, args in ((ops.scan_forward, [u, u, a, b, b, d, u, d, True, off, None, s]),
                       (ops.scan_backward, [out, u, u, a, b, b, d, u, d, True, off, None, saved, s]),
                       (ops.scan_step, [u[:2], u[:2], a, b[:2], b[:2], s, d, u[:2], d])):
        for i, x in enumerate(args):
            if isinstance(x, torch.Tensor) and x.is_floating_point():
                some = list(args)
                some[i] = x.clone().requires_grad_()
                with pytest.raises(ValueError, match="requires grad"):
                    call(*some)
    assert not calls
