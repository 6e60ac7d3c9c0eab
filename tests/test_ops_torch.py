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
