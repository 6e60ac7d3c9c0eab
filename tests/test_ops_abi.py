"""The operators' C ABI (include/reuse_ops.h): every declared symbol is there, bad
arguments are refused with a status and a text before any launch, and the torch
functions refuse tensors that the kernels would read or write wrongly.  None of
it needs a GPU: every call below ends in the checks (or has nothing to do)."""
import ctypes
import os
import re

import pytest
import torch

from paper_1909_05632_amd import binding as B
from paper_1909_05632_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_and_binding_name_the_same_calls():
    text = open(os.path.join(ROOT, "include", "reuse_ops.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    assert sorted(set(re.findall(r"\b(reuse_ops_\w+)\s*\(", text))) == sorted(ops.EXPORTS)
    lib = ops.load_ops()
    for name in ops.EXPORTS:
        assert hasattr(lib, name), name


def _shape(n=2, hk=1, hv=2, dk=16, dv=16, tokens=10, dtype=B.RN_F32, scale=1.0, qs=None, ks=None, vs=None):
    return ops.rn_delta_shape(n, hk, hv, dk, dv, tokens, dtype, scale, hk * dk if qs is None else qs,
                              hk * dk if ks is None else ks, hv * dv if vs is None else vs)


P = 256          # a pointer that is not NULL; no call below gets as far as using it


def _err(status, want, text):
    assert status == want, (status, ops.reuse_ops_last_error())
    assert text in ops.reuse_ops_last_error(), ops.reuse_ops_last_error()


def test_layer_norm_arguments():
    L = ops.load_ops()
    fwd = dict(rows=4, width=8, x=P, xs=8, dtype=B.RN_F32, w=P, b=P, eps=1e-5, y=P, ys=8, stats=None, stream=None)

    def call(**kw):
        return L.reuse_ops_layer_norm(*{**fwd, **kw}.values())

    _err(call(rows=-1), B.RN_EINVAL, "rows")
    _err(call(width=0), B.RN_EINVAL, "width")
    _err(call(dtype=B.RN_U8), B.RN_EINVAL, "dtype")
    _err(call(x=None), B.RN_EINVAL, "NULL")
    _err(call(y=None), B.RN_EINVAL, "NULL")
    _err(call(xs=7), B.RN_EINVAL, "stride")
    _err(call(ys=7), B.RN_EINVAL, "stride")
    _err(call(eps=-1.0), B.RN_EINVAL, "eps")
    _err(call(eps=float("nan")), B.RN_EINVAL, "eps")
    assert call(rows=0, x=None, y=None) == B.RN_OK
    need = L.reuse_ops_layer_norm_backward_scratch_bytes(4, 8)
    assert need > 0 and need % 256 == 0
    assert L.reuse_ops_layer_norm_backward_scratch_bytes(-1, 8) == 0
    assert L.reuse_ops_layer_norm_backward_scratch_bytes(4, 0) == 0
    bwd = dict(rows=4, width=8, dy=P, dys=8, x=P, xs=8, dtype=B.RN_F32, w=None, stats=P, dx=P, dxs=8, dw=P, db=P,
               acc=0, scratch=P, bytes=need, stream=None)

    def back(**kw):
        return L.reuse_ops_layer_norm_backward(*{**bwd, **kw}.values())

    _err(back(rows=1 << 50), B.RN_EINVAL, "rows")
    _err(back(dtype=9), B.RN_EINVAL, "dtype")
    for name in ("dy", "x", "stats", "dx"):
        _err(back(**{name: None}), B.RN_EINVAL, "NULL")
    _err(back(dys=3), B.RN_EINVAL, "stride")
    _err(back(scratch=None), B.RN_EINVAL, "scratch")
    _err(back(scratch=P + 4), B.RN_EINVAL, "aligned")
    _err(back(bytes=need - 1), B.RN_ENOSPACE, "need")
    assert back(rows=0, dw=None, db=None) == B.RN_OK


def test_sample_arguments():
    L = ops.load_ops()
    params = ops.rn_sample_params(1.0, 0, 1.0, 0.0)
    base = dict(n=2, vocab=6, logits=P, stride=6, dtype=B.RN_F32, u=P, params=ctypes.byref(params), tokens=P,
                logprobs=None, stream=None)

    def call(**kw):
        return L.reuse_ops_sample(*{**base, **kw}.values())

    _err(call(n=-1), B.RN_EINVAL, "n must")
    _err(call(vocab=0), B.RN_EINVAL, "vocab")
    _err(call(vocab=ops.RN_SAMPLE_MAX_VOCAB + 1), B.RN_EINVAL, "vocab")
    _err(call(dtype=B.RN_U8), B.RN_EINVAL, "dtype")
    _err(call(params=None), B.RN_EINVAL, "params")
    for name in ("logits", "u", "tokens"):
        _err(call(**{name: None}), B.RN_EINVAL, "NULL")
    _err(call(stride=5), B.RN_EINVAL, "stride")
    assert call(n=0, logits=None, u=None, tokens=None) == B.RN_OK


def test_delta_shapes_and_sizes():
    L = ops.load_ops()
    bad = [(dict(n=-1), "n must"), (dict(n=70000), "n must"), (dict(hk=0), "heads_v"), (dict(hv=3, hk=2), "heads_v"),
           (dict(hv=2048), "heads_v"), (dict(dk=0), "dk"), (dict(dv=-4), "dk"), (dict(tokens=-1), "tokens"),
           (dict(tokens=1 << 31), "tokens"), (dict(n=0), "without sequences"), (dict(dtype=B.RN_U8), "dtype"),
           (dict(qs=15), "stride"), (dict(ks=15), "stride"), (dict(vs=31), "stride")]
    sizes = (L.reuse_ops_delta_saved_bytes, L.reuse_ops_delta_scratch_bytes, L.reuse_ops_delta_backward_scratch_bytes)
    for kw, text in bad:
        s = _shape(**kw)
        assert all(f(ctypes.byref(s)) == 0 for f in sizes), kw
        _err(L.reuse_ops_delta_forward(ctypes.byref(s), *[P] * 5, None, None, P, P, None, 0, P, 1 << 30, None),
             B.RN_EINVAL, text)
        _err(L.reuse_ops_delta_step(ctypes.byref(s), *[P] * 5, None, 8, P, P, None), B.RN_EINVAL, text)
    for kw in (dict(dk=129), dict(dv=256)):
        s = _shape(**kw)
        assert all(f(ctypes.byref(s)) == 0 for f in sizes)
        _err(L.reuse_ops_delta_forward(ctypes.byref(s), *[P] * 5, None, None, P, P, None, 0, P, 1 << 30, None),
             B.RN_EUNSUPPORTED, "128")
    assert all(f(None) == 0 for f in sizes)
    small, large = _shape(), _shape(tokens=1000)
    for f in sizes:
        assert 256 <= f(ctypes.byref(small)) < f(ctypes.byref(large)) and f(ctypes.byref(small)) % 256 == 0


def test_delta_arguments():
    L = ops.load_ops()
    s = _shape()
    need = L.reuse_ops_delta_scratch_bytes(ctypes.byref(s))
    fwd = dict(shape=ctypes.byref(s), q=P, k=P, v=P, g=P, beta=P, off=P, state=None, final=None, out=P, saved=None,
               saved_bytes=0, scratch=P, bytes=need, stream=None)

    def call(**kw):
        return L.reuse_ops_delta_forward(*{**fwd, **kw}.values())

    _err(call(shape=None), B.RN_EINVAL, "shape")
    for name in ("q", "k", "v", "g", "beta", "out"):
        _err(call(**{name: None}), B.RN_EINVAL, "NULL")
    _err(call(scratch=None), B.RN_EINVAL, "scratch")
    _err(call(scratch=P + 8), B.RN_EINVAL, "aligned")
    _err(call(bytes=need - 1), B.RN_ENOSPACE, "scratch")
    _err(call(saved=P, saved_bytes=16), B.RN_ENOSPACE, "saved")
    odd = _shape(n=3)
    _err(call(shape=ctypes.byref(odd), off=None), B.RN_EINVAL, "multiple")
    none = _shape(n=0, tokens=0)
    assert call(shape=ctypes.byref(none), scratch=None) == B.RN_OK
    kept = L.reuse_ops_delta_saved_bytes(ctypes.byref(s))
    need = L.reuse_ops_delta_backward_scratch_bytes(ctypes.byref(s))
    bwd = dict(shape=ctypes.byref(s), q=P, k=P, v=P, g=P, beta=P, off=P, saved=P, saved_bytes=kept, dout=P, dfinal=None,
               dq=P, dk=P, dv=P, dg=P, dbeta=P, dstate=None, scratch=P, bytes=need, stream=None)

    def back(**kw):
        return L.reuse_ops_delta_backward(*{**bwd, **kw}.values())

    for name in ("q", "k", "v", "g", "beta", "dout", "dq", "dk", "dv", "dg", "dbeta", "saved", "scratch"):
        _err(back(**{name: None}), B.RN_EINVAL, "NULL")
    _err(back(saved_bytes=kept - 1), B.RN_ENOSPACE, "saved")
    _err(back(bytes=need - 1), B.RN_ENOSPACE, "scratch")
    _err(back(saved=P + 64), B.RN_EINVAL, "aligned")
    _err(back(dfinal=2 * P, dstate=2 * P), B.RN_EINVAL, "dfinal")
    one = _shape(tokens=2)
    step = dict(shape=ctypes.byref(one), q=P, k=P, v=P, g=P, beta=P, ids=None, slots=2, state=P, out=P, stream=None)

    def stp(**kw):
        return L.reuse_ops_delta_step(*{**step, **kw}.values())

    _err(stp(shape=ctypes.byref(s)), B.RN_EINVAL, "one token a stream")
    _err(stp(slots=1), B.RN_EINVAL, "slots")
    _err(stp(slots=-1, ids=P), B.RN_EINVAL, "slots")
    _err(stp(state=None), B.RN_EINVAL, "NULL")
    assert stp(shape=ctypes.byref(none), slots=0, state=None) == B.RN_OK


def test_torch_functions_refuse_before_any_launch():
    """On tensors of the CPU, which no kernel can read, and on wrong types."""
    x, w = torch.zeros(3, 8), torch.zeros(8)
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm(x, w, w)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        ops.layer_norm(x.double(), w, w)
    with pytest.raises(TypeError, match="torch tensor"):
        ops.layer_norm([1.0], w, w)
    with pytest.raises(ValueError, match="GPU"):
        ops.layer_norm_backward(x, x, w, torch.zeros(3, 2))
    with pytest.raises(ValueError, match="GPU"):
        ops.sample(x, torch.zeros(3))
    with pytest.raises(TypeError):
        ops.sample(x.half(), torch.zeros(3))
    q, v, g = torch.zeros(4, 1, 8), torch.zeros(4, 2, 8), torch.zeros(4, 2)
    with pytest.raises(ValueError, match="GPU"):
        ops.delta_step(q, q, v, g, g, torch.zeros(4, 2, 8, 8))
    with pytest.raises(ValueError, match="seq_off"):
        ops.delta_forward(q, q, v, g, g)
    with pytest.raises(ValueError, match="even"):
        ops.delta_forward(q, q, v, g, g, n=3)
    with pytest.raises(ValueError, match="1-D"):
        ops.delta_forward(q, q, v, g, g, seq_off=torch.zeros(2, 2, dtype=torch.int32))
    with pytest.raises(TypeError, match="int32"):
        ops.delta_forward(q, q, v, g, g, seq_off=torch.tensor([0, 4]))
    with pytest.raises(ValueError, match="GPU"):
        ops.delta_backward(v, q, q, v, g, g, n=2)


def test_rows_of_views():
    """What layer_norm and sample take as rows at one stride, and what they do not."""
    t = torch.zeros(6, 4, 10)
    assert ops._rows(t, "t") == (24, 10)
    assert ops._rows(t[:, :, :7], "t") == (24, 10)
    assert ops._rows(t[:, 1], "t") == (6, 40)
    assert ops._rows(t[2], "t") == (4, 10)
    assert ops._rows(t[:, :1, :3], "t") == (6, 40)
    assert ops._rows(t[0, 0, 2:5], "t") == (1, 3)
    assert ops._rows(torch.zeros(0, 5), "t") == (0, 5)
    for bad in (t[:, :3, :7], t.transpose(1, 2), t[:, :, ::2], t[:, :1].expand(6, 4, 10), t[0, :1].expand(3, 10)):
        with pytest.raises(ValueError, match="stride"):
            ops._rows(bad, "t")
