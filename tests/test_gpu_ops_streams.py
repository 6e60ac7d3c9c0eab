"""Calls of the operators on a stream that is not the current one, with work
queued on both: each gives the bits it gives alone."""
import pytest
import torch

from tests.conftest import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs an MI355X GPU")]


def _delta(seed, tokens=2048):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    q, k = (torch.nn.functional.normalize(randn(tokens, 4, 64), dim=-1) for _ in range(2))
    return [q, k, randn(tokens, 4, 64), -torch.rand(tokens, 4, generator=gen, device="cuda"),
            torch.rand(tokens, 4, generator=gen, device="cuda")], randn(tokens, 4, 64)


def _train(args, dout, stream=None):
    from paper_1909_05632_amd import ops
    out, final, saved = ops.delta_forward(*args, n=4, save=True, stream=stream)
    return [out, final, *ops.delta_backward(dout, *args, n=4, saved=saved, stream=stream)]


def test_scratch_of_queued_calls_is_not_taken():
    """The current stream's calls have returned their scratch, but not yet run: calls of the same
    sizes on another stream find memory of their own."""
    a, b = _delta(1), _delta(2)
    want_a, want_b = _train(*a), _train(*b)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got_a, got_b = [], []
    for _ in range(8):
        got_a.append(_train(*a))
        got_b.append(_train(*b, stream=side))
    torch.cuda.synchronize()
    for got, want in ((got_a, want_a), (got_b, want_b)):
        assert all(torch.equal(x, y) for g in got for x, y in zip(g, want))


def test_results_that_are_dropped_are_not_reused_too_early():
    """A result that the caller does not keep: its memory goes to later work of the same stream only."""
    from paper_1909_05632_amd import ops
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, u = torch.randn(4096, 4096, generator=gen, device="cuda"), torch.rand(4096, generator=gen, device="cuda")
    w = torch.ones(4096, device="cuda")
    want = ops.sample(x, u, top_k=40)[0]
    dx, dw, db = ops.layer_norm_backward(x, x, w, ops.layer_norm(x, w, w, with_stats=True)[1])
    stats = ops.layer_norm(x, w, w, with_stats=True)[1]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    kept, marks = [], []
    for i in range(8):
        kept.append((ops.sample(x, u, top_k=40, stream=side)[0], ops.layer_norm_backward(x, x, w, stats, stream=side)[0]))
        marks.append([torch.full((4096,), float(i), device="cuda") for _ in range(4)])
    torch.cuda.synchronize()
    assert all(torch.equal(t, want) and torch.equal(d, dx) for t, d in kept)
    assert all((m == i).all() for i, ms in enumerate(marks) for m in ms)


def test_results_lie_in_the_streams_memory():
    from paper_1909_05632_amd import ops
    side = torch.cuda.Stream()
    args, dout = _delta(4, 256)
    x, w, u = torch.randn(64, 512, device="cuda"), torch.ones(512, device="cuda"), torch.rand(64, device="cuda")
    torch.cuda.synchronize()
    y, stats = ops.layer_norm(x, w, w, with_stats=True, stream=side)
    made = [y, stats, *ops.layer_norm_backward(x, x, w, stats, stream=side),
            *ops.sample(x, u, stream=side), *_train(args, dout, side)]
    side.synchronize()
    of = {}
    for seg in torch.cuda.memory_snapshot():
        at = seg["address"]
        for block in seg["blocks"]:
            of[at] = seg["stream"]
            at += block["size"]
    assert all(of[t.data_ptr()] == side.cuda_stream for t in made)


def test_a_stream_of_another_device_is_refused():
    from paper_1909_05632_amd import ops

    class Other:
        device, cuda_stream = torch.device("cuda", 1), 0

    with pytest.raises(ValueError, match="stream is on"):
        ops.layer_norm(torch.zeros(2, 8, device="cuda"), stream=Other())
