"""What the torch functions of the operators do around their launches: which
stream's memory they take, which sizes they pass on, which tensors they refuse.
The launches themselves are left out here, so that none of it needs a GPU."""
import pytest
import torch

from paper_1909_05632_amd import ops


@pytest.fixture
def calls(monkeypatch):
    """The functions on CPU tensors; (name, arguments) of every call that would have been launched."""
    seen = []
    monkeypatch.setattr(ops, "_data", lambda x, what: ops._CODES[x.dtype])
    monkeypatch.setattr(ops, "_launch", lambda device, *call: seen.append(call))
    return seen


def _every_call(**kw):
    """Each function once on small tensors; what each returns."""
    x, w, u = torch.zeros(3, 8), torch.ones(8), torch.zeros(3)
    q, v, g, s = torch.zeros(4, 1, 8), torch.zeros(4, 2, 8), torch.zeros(4, 2), torch.zeros(4, 2, 8, 8)
    y, stats = ops.layer_norm(x, w, w, with_stats=True, **kw)
    step = ops.delta_step(q, q, v, g, g, s, **kw)
    out, final, saved = ops.delta_forward(q, q, v, g, g, n=2, save=True, **kw)
    return [y, stats, *ops.layer_norm_backward(y, x, w, stats, **kw), *ops.sample(x, u, **kw), step, out, final, saved,
            *ops.delta_backward(out, q, q, v, g, g, n=2, saved=saved, **kw)]


def test_what_a_call_makes_is_memory_of_its_stream(calls, monkeypatch):
    """Memory of another stream may still be read or written by what that stream has queued."""
    inside, made, launched = [], [], []

    class On:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            inside.append(self.stream)

        def __exit__(self, *_):
            inside.pop()

    class Side:
        device, cuda_stream = torch.device("cpu"), 7

    side, empty = Side(), ops._empty
    monkeypatch.setattr(torch.cuda, "stream", On)
    monkeypatch.setattr(ops, "_empty", lambda *a, **kw: made.append(list(inside)) or empty(*a, **kw))
    monkeypatch.setattr(ops, "_launch", lambda *a: launched.append(list(inside)))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    _every_call()
    assert len(made) == 20 and len(launched) == 6 and not any(made) and not any(launched)
    want = len(made)
    made.clear(), launched.clear()
    _every_call(stream=side)
    assert len(made) == want and all(m == [side] for m in made) and launched == [[side]] * 6 and not inside


def _delta_bytes(n, tokens, even, hk=8, hv=8, dk=64, dv=64, dtype=torch.float32):
    import ctypes
    L = ops.load_ops()
    s = ops.rn_delta_shape(n, hk, hv, dk, dv, tokens, ops._CODES[dtype], 1.0, hk * dk, hk * dk, hv * dv, even)
    return [f(ctypes.byref(s)) for f in (L.reuse_ops_delta_saved_bytes, L.reuse_ops_delta_scratch_bytes,
                                         L.reuse_ops_delta_backward_scratch_bytes)]


def test_scratch_is_what_the_call_uses():
    """Even sequences of up to 32 tokens go token by token: nothing forward, a float32 row a token
    backward.  Ragged ones of as few on average may hold no more chunks than tokens / 32."""
    for n, length in ((16384, 16), (5, 32), (1000, 1)):
        tokens = n * length
        saved, fwd, bwd = _delta_bytes(n, tokens, 1)
        rows, state = tokens * 8 * 64 * 4, 8 * 64 * 64 * 4
        assert fwd == 256 and bwd <= rows + 512
        assert saved <= rows + (n + tokens // 64) * state + 768
    # the chunk operands of one slot: the planes of K, Q and K^T, the inverse, the scores, the decays
    one = 3 * 8 * 4 * 2 * 3 * 1024 + 8 * (2 * 18 * 1024 + 768)
    _, fwd, bwd = _delta_bytes(16384, 16384 * 16, 0)
    assert fwd <= 8192 * one + 4096 and bwd <= 8192 * (one + 8 * 64 * 64 * 4 + 16) + 16384 * 16 * 8 * 64 * 4 + 4096
    assert _delta_bytes(8, 20, 0)[1] == 256                      # no sequence above 32 among 20 tokens
    _, long_even, _ = _delta_bytes(4, 4 * 640, 1)
    assert _delta_bytes(4, 4 * 640, 0)[1] == long_even >= 40 * one


def test_even_sequences_are_told_to_the_library(calls):
    q, v, g = torch.zeros(96, 1, 8), torch.zeros(96, 2, 8), torch.zeros(96, 2)
    off = torch.tensor([0, 90, 96], dtype=torch.int32)
    out, _, saved = ops.delta_forward(q, q, v, g, g, n=4, save=True)
    ops.delta_backward(out, q, q, v, g, g, n=4, saved=saved)
    out, _, saved = ops.delta_forward(q, q, v, g, g, off, save=True)
    ops.delta_backward(out, q, q, v, g, g, off, saved=saved)
    assert [c[1]._obj.even for c in calls] == [1, 1, 0, 0]
    with pytest.raises(ops.B.ReuseNetError, match="multiple"):
        ops._check(ops.load_ops().reuse_ops_delta_forward(
            ops.ctypes.byref(ops.rn_delta_shape(5, 1, 2, 8, 8, 96, 0, 1.0, 8, 8, 16, 1)), *[256] * 5, None, None, 256, 256,
            None, 0, 256, 1 << 30, None))
    with pytest.raises(ops.B.ReuseNetError, match="no seq_off"):
        ops._check(ops.load_ops().reuse_ops_delta_forward(
            ops.ctypes.byref(ops.rn_delta_shape(4, 1, 2, 8, 8, 96, 0, 1.0, 8, 8, 16, 1)), *[256] * 5, 256, None, 256, 256,
            None, 0, 256, 1 << 30, None))


def test_sizes_past_32_bits_are_refused(calls):
    """The C calls take 32-bit counts, and ctypes drops the bits above them without a word."""
    big = (1 << 32) + 8
    meta = lambda *shape, **kw: torch.empty(*shape, device="meta", **kw)  # noqa: E731
    with pytest.raises(ValueError, match="width"):
        ops.layer_norm(meta(1, big))
    with pytest.raises(ValueError, match="width"):
        ops.layer_norm_backward(meta(1, big), meta(1, big), None, meta(1, 2))
    with pytest.raises(ValueError, match="n must"):
        ops.sample(meta(big, 2), meta(big))
    q, g = meta(4, 1, 8), meta(4, 1)
    with pytest.raises(ValueError, match="slots"):
        ops.delta_step(q, q, q, g, g, meta(big, 1, 8, 8))
    q, g = meta(big, 1, 8), meta(big, 1)
    with pytest.raises(ValueError, match="n must"):
        ops.delta_step(q, q, q, g, g, meta(big, 1, 8, 8))
    with pytest.raises(ValueError, match="n must"):
        ops.delta_forward(q, q, q, g, g, n=big)
    assert not calls


def test_top_k_of_any_size_keeps_its_meaning(calls):
    """Above the vocabulary, and 0 or less: all."""
    x, u = torch.zeros(2, 9), torch.zeros(2)
    for k, want in ((5, 5), (0, 0), (-3, 0), ((1 << 32) + 5, None), (1 << 31, None), (-(1 << 32) + 5, 0), (1 << 40, None)):
        ops.sample(x, u, top_k=k)
        got = calls[-1][-3]._obj.top_k
        assert max(got, 0) == want if want is not None else got >= 9, (k, got)
    with pytest.raises(TypeError):
        ops.sample(x, u, top_k=2.5)


def test_tensors_that_require_grad_are_refused_in_grad_mode(calls):
    """The calls record nothing: a result would be cut off from its inputs without a word."""
    x, w, u = torch.zeros(3, 8), torch.ones(8), torch.zeros(3)
    q, v, g, s = torch.zeros(4, 1, 8), torch.zeros(4, 2, 8), torch.zeros(4, 2), torch.zeros(4, 2, 8, 8)
    off, stats = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(3, 2)
    s1 = s[:1].clone()
    saved = ops.delta_forward(q, q, v, g, g, off, save=True)[2]
    temperature = torch.ones(3)
    every = [(ops.layer_norm, (x, w, w), {}, 3), (ops.layer_norm_backward, (x, x, w, stats), {}, 4),
             (ops.sample, (x, u, temperature), {}, 1), (ops.delta_step, (q, q, v, g, g, s), {}, 6),
             (ops.delta_forward, (q, q, v, g, g, off, None, s1), {}, 5),
             (ops.delta_backward, (v, q, q, v, g, g, off, None, saved, s1), {}, 6)]
    calls.clear()
    for call, args, kw, floats in every:
        for i in [*range(floats)] + ([7] if call is ops.delta_forward else []) + ([9] if call is ops.delta_backward else []):
            some = list(args)
            some[i] = args[i].clone().requires_grad_()
            with pytest.raises(ValueError, match="requires grad"):
                call(*some, **kw)
            assert not calls
            with torch.no_grad():
                call(*some, **kw)
            some[i] = some[i].detach()
            call(*some, **kw)
            assert len(calls) == 2
            calls.clear()
