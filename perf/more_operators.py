"""Cases of the operators of a recurrent block around a policy net: residual norm, short convolution, selective scan, and the log-probabilities a policy is trained on.

A block adds what the one before it gave to the residual stream and normalises
the sum (root mean square), mixes each channel with its last few tokens, carries
a state per channel that decays by an amount of its own at every token, and the
policy at the end is evaluated: the log-probability of the choice that was made,
the entropy, the likeliest alternatives, and the gradient of the first two.  A
case is one such call, or one with its gradients; a single token's case is the
convolution and the scan together, as a stream that acts makes them.  The
smallest are one stream's frame, where the call itself is what costs, the
ordinary ones are the rollouts and training batches of this repository's
benchmark (256 and 1024 streams, 16-frame episodes, 18 actions), the largest are
of the sizes that language models run the same operators at.

Where ``own`` is false, ``run`` computes a case in elementary torch operations
in float32, rounded once at the end; where it is true, it calls the operators
of ``paper_1909_05632_amd``.  ``exact`` evaluates the definitions in float64:
the scan token by token, as its recurrence is written.
"""
from __future__ import annotations

import math
import random

import torch

own = False                # True: the framework's operators, False: plain torch

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3_MAX = 448.0


# ------------------------------------------------------------------ cases

def _norm(kind, rows, width, dtype, residual=True):
    return dict(op="norm", kind=kind, rows=rows, width=width, dtype=dtype, residual=residual)


def _logp(kind, n, vocab, dtype, top=0, masked=False, scale=2.5, temperature=1.0):
    return dict(op="logp", kind=kind, n=n, vocab=vocab, dtype=dtype, top=top, masked=masked, scale=scale,
                temperature=temperature)


def _conv(kind, n, tokens, channels, taps, dtype, ragged=False):
    return dict(op="conv", kind=kind, n=n, tokens=tokens, channels=channels, taps=taps, dtype=dtype, ragged=ragged)


def _scan(kind, n, tokens, channels, states, groups, dtype, ragged=False, gated=True):
    return dict(op="scan", kind=kind, n=n, tokens=tokens, channels=channels, states=states, groups=groups,
                dtype=dtype, ragged=ragged, gated=gated)


def _step(n, channels, states, groups, taps, dtype, gated=True):
    return dict(op="step", n=n, channels=channels, states=states, groups=groups, taps=taps, dtype=dtype, gated=gated)


def listed():
    return [
        # One stream acting: its frame's features and the residual stream.
        dict(_norm("infer", 1, 512, "f32"), name="rms-1x512"),
        # A wide model's training batch with its residual stream, forward and gradients.
        dict(_norm("train", 16384, 4096, "bf16"), name="rms-train-16384x4096-bf16"),
        # Serving 1024 streams: the norm's output in 8 bits, for a matrix product in 8 bits.
        dict(_norm("8bit", 1024, 8192, "bf16"), name="rms-8bit-1024x8192-bf16"),
        # The benchmark's training batch: 256 streams x 16 frames, 18 actions of which some are not allowed.
        dict(_logp("train", 4096, 18, "f32", masked=True, scale=1.5), name="logp-train-4096x18"),
        # A language model's policy gradient: every token's choice out of the vocabulary.
        dict(_logp("train", 2048, 131072, "bf16"), name="logp-train-2048x131072-bf16"),
        # Serving with log-probabilities: the choice and its 20 likeliest alternatives.
        dict(_logp("infer", 64, 131072, "bf16", top=20), name="logp-top-64x131072-bf16"),
        # Histories of odd lengths, forward and gradients.
        dict(_conv("train", 5, 16384, 4096, 4, "bf16", True), name="conv-train-ragged16384-bf16"),
        # One stream acting: its frame through convolution and scan.
        dict(_step(1, 512, 16, 1, 4, "f32"), name="ssm-step-1"),
        # Serving 1024 streams, one frame each: the states are read and written.
        dict(_step(1024, 2048, 16, 1, 4, "bf16"), name="ssm-step-1024-bf16"),
        # Histories of odd lengths taken in at once.
        dict(_scan("forward", 5, 16384, 4096, 16, 1, "bf16", True), name="scan-fwd-ragged16384-bf16"),
        # The benchmark's training episodes, forward and gradients.
        dict(_scan("train", 256, 4096, 256, 16, 1, "f32"), name="scan-train-256x16"),
        # Long episodes of odd lengths, forward and gradients.
        dict(_scan("train", 7, 8192, 2048, 16, 1, "bf16", True), name="scan-train-ragged8192-bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "logp", "conv", "scan", "scan", "step"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "norm":
        width = _log(rng, 18, 16384)
        rows = _log(rng, 1, min(65536, 2 ** 26 // width))
        return _norm(rng.choice(("infer", "train", "8bit")), rows, width, dtype, rng.random() < 0.7)
    if op == "logp":
        vocab = _log(rng, 2, 131072)
        n = _log(rng, 1, min(16384, 2 ** 27 // vocab))
        top = rng.choice((0, 1, 5, 20, 32))
        return _logp(rng.choice(("infer", "train")), n, vocab, dtype, min(top, vocab), rng.random() < 0.4,
                     rng.choice((0.5, 1.5, 2.5)), rng.choice((1.0, 1.0, 0.7)))
    channels = _log(rng, 16, 4096)
    if op == "conv":
        n = _log(rng, 1, 256)
        most = 2 ** 26 // channels
        kind = rng.choice(("forward", "train"))
        if rng.random() < 0.5:
            return _conv(kind, n, n * _log(rng, 1, max(1, min(2048, 16384, most) // n)), channels,
                         rng.choice((2, 3, 4)), dtype)
        return _conv(kind, n, _log(rng, n, min(16384, most)), channels, rng.choice((2, 3, 4)), dtype, True)
    states = rng.choice((1, 4, 8, 13, 16, 16, 16, 32, 64))
    groups = rng.choice((1, 1, 2, 3))
    channels -= channels % groups
    gated = rng.random() < 0.7
    if op == "step":
        n = _log(rng, 1, min(1024, 2 ** 25 // (channels * states)))
        return _step(n, channels, states, groups, rng.choice((2, 3, 4)), dtype, gated)
    kind = rng.choice(("forward", "train"))
    n = _log(rng, 1, 256)
    most = max(1, (2 ** 28 if kind == "train" else 2 ** 30) // (channels * states))
    n = min(n, most)
    if rng.random() < 0.5:
        return _scan(kind, n, n * _log(rng, 1, max(1, min(512, min(8192, most) // n))), channels, states, groups,
                     dtype, False, gated)
    return _scan(kind, n, _log(rng, n, max(n, min(8192, most))), channels, states, groups, dtype, True, gated)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        every, r = rows * width, int(case["residual"])
        forward = size * every * (1 + 2 * r) + 4 * width        # x and the residual in, their sum out
        if case["kind"] == "8bit":
            return {"bytes": float(forward + every + 4 * rows), "flops": 8.0 * every}
        if case["kind"] == "infer":
            return {"bytes": float(forward + size * every), "flops": 5.0 * every}
        # and y; dy and the sum's own gradient in, dx and dweight out
        return {"bytes": float(forward + size * every + size * every * (2 + r) + 4 * width), "flops": 14.0 * every}
    if case["op"] == "logp":
        every = case["n"] * case["vocab"]
        rows = case["n"] * (12 + 8 * case["top"])
        if case["kind"] == "infer":
            return {"bytes": float(size * every + rows), "flops": 5.0 * every}
        return {"bytes": float(2 * size * every + rows + 8 * case["n"]), "flops": 12.0 * every}
    channels = case["channels"]
    if case["op"] == "conv":
        every, taps = case["tokens"] * channels, case["taps"]
        ends = 2 * case["n"] * (taps - 1) * channels * size
        weights = 4 * channels * (taps + 1)
        if case["kind"] == "forward":
            return {"bytes": float(2 * size * every + ends + weights), "flops": (2.0 * taps + 5) * every}
        return {"bytes": float(4 * size * every + 2 * ends + 2 * weights), "flops": (8.0 * taps + 12) * every}
    states, groups, gated = case["states"], case["groups"], int(case["gated"])
    weights = 4 * channels * (states + 2)
    if case["op"] == "step":
        n, taps = case["n"], case["taps"]
        ends = 2 * n * (taps - 1) * channels * size
        io = n * (channels * (3 + gated) + 2 * groups * states) * size
        every = n * channels
        return {"bytes": float(2 * 4 * every * states + ends + io + weights + 4 * channels * (taps + 1)),
                "flops": (7.0 * states + 2 * taps + 20) * every}
    tokens = case["tokens"]
    every = tokens * channels
    ins = (every * (2 + gated) + 2 * tokens * groups * states) * size
    ends = 2 * 4 * case["n"] * channels * states
    # per state: the decay's exponent and exponential, its product, what is written, what is read
    flops = (7.0 * states + 15) * every
    if case["kind"] == "forward":
        return {"bytes": float(ins + every * size + ends + weights), "flops": flops}
    return {"bytes": float(2 * ins + 2 * every * size + 2 * ends + 2 * weights), "flops": 3 * flops}


# ------------------------------------------------------------------ inputs

def _offsets(case, seed):
    """Where each sequence begins: the tokens cut at random places (empty ones among them), or evenly."""
    n, tokens = case["n"], case["tokens"]
    if not case["ragged"]:
        return [i * (tokens // n) for i in range(n + 1)]
    rng = random.Random(seed)
    return [0] + sorted(rng.randint(0, tokens) for _ in range(n - 1)) + [tokens]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    s = {"case": dict(case), "residual": None, "z": None}
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        # A layer's output beside a residual stream that is larger and whose scale differs from row to row.
        s["x"] = randn(rows, width, dtype=dtype)
        if case["residual"]:
            s["residual"] = (2 * randn(rows, width) * torch.exp(0.5 * randn(rows, 1))).to(dtype)
        s["weight"] = 1 + 0.1 * randn(width)
        if case["kind"] == "train":
            s["dy"] = randn(rows, width, dtype=dtype)
            s["dtotal"] = randn(rows, width, dtype=dtype) if case["residual"] else None
        return s
    if case["op"] == "logp":
        n, vocab = case["n"], case["vocab"]
        logits = case["scale"] * randn(n, vocab)
        if case["masked"]:
            # Choices that are not allowed; one always is.
            off = rand(n, vocab) < 0.3
            off.scatter_(1, (rand(n, 1) * vocab).long(), False)
            logits.masked_fill_(off, -math.inf)
        # The choices made: drawn from the distribution itself.
        s["tokens"] = torch.argmax(logits - torch.log(-torch.log(rand(n, vocab).clamp_(1e-9, 1 - 1e-6))), -1).to(torch.int32)
        s["logits"] = logits.to(dtype)
        if case["kind"] == "train":
            s["dlogprobs"] = -randn(n) / n       # of -advantage log p ...
            s["dentropy"] = torch.full((n,), -0.01 / n, device="cuda")     # ... - 0.01 H, means over the batch
        return s
    channels = case["channels"]
    n, tokens = case["n"], case["n"] if case["op"] == "step" else case["tokens"]
    if case["op"] != "step":
        off = _offsets(case, seed)
        s["seq_off"] = torch.tensor(off, dtype=torch.int32, device="cuda")
    if case["op"] in ("conv", "step"):
        s["weight"] = 0.5 * randn(channels, case["taps"])
        s["bias"] = 0.1 * randn(channels)
        s["x"] = randn(tokens, channels, dtype=dtype)
        s["window"] = randn(n, case["taps"] - 1, channels, dtype=dtype)
        if case["op"] == "conv":
            if case["kind"] == "train":
                s["dout"] = randn(tokens, channels, dtype=dtype)
                s["dfinal"] = randn(n, case["taps"] - 1, channels, dtype=dtype)
            return s
    states, groups = case["states"], case["groups"]
    if case["op"] == "scan":
        x = randn(tokens, channels)
        s["u"] = (x * torch.sigmoid(x)).to(dtype)
    # Decays 1, 2, ... as such layers begin, trained a little apart; step sizes from 0.001 to 0.1.
    s["a"] = -torch.arange(1, states + 1, device="cuda").float() * torch.exp(0.2 * randn(channels, states))
    s["dt_bias"] = torch.log(torch.expm1(torch.exp(math.log(1e-3) + math.log(100.0) * rand(channels))))
    s["dt"] = (0.7 * randn(tokens, channels)).to(dtype)
    s["b"] = randn(tokens, groups, states, dtype=dtype)
    s["c"] = randn(tokens, groups, states, dtype=dtype)
    s["d"] = 1 + 0.1 * randn(channels)
    if case["gated"]:
        s["z"] = randn(tokens, channels, dtype=dtype)
    s["state"] = 0.1 * randn(n, channels, states)
    if case.get("kind") == "train":
        s["dout"] = randn(tokens, channels, dtype=dtype)
        s["dfinal"] = 0.1 * randn(n, channels, states)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if own:
        return {"norm": _norm_own, "logp": _logp_own, "conv": _conv_own, "scan": _scan_own, "step": _step_own}[case["op"]](s, case)
    return {"norm": _norm_plain, "logp": _logp_plain, "conv": _conv_plain, "scan": _scan_plain, "step": _step_plain}[case["op"]](s, case)


def _norm_own(s, case):
    from paper_1909_05632_amd import ops

    x, weight, residual = s["x"], s["weight"], s["residual"]
    if case["kind"] == "8bit":
        got = ops.rms_norm(x, weight, residual=residual, eps=EPS, quantize=True)
        return dict(zip(("y", "scales", "total"), got))
    if case["kind"] == "infer":
        got = ops.rms_norm(x, weight, residual=residual, eps=EPS)
        return {"y": got} if residual is None else {"y": got[0], "total": got[1]}
    if residual is None:
        y, rstd = ops.rms_norm(x, weight, eps=EPS, with_stats=True)
        dx, dweight = ops.rms_norm_backward(s["dy"], x, weight, rstd)
        return {"y": y, "dx": dx, "dweight": dweight}
    y, total, rstd = ops.rms_norm(x, weight, residual=residual, eps=EPS, with_stats=True)
    dx, dweight = ops.rms_norm_backward(s["dy"], total, weight, rstd, dtotal=s["dtotal"])
    return {"y": y, "total": total, "dx": dx, "dweight": dweight}


def _logp_own(s, case):
    from paper_1909_05632_amd import ops

    train = case["kind"] == "train"
    got = ops.log_probs(s["logits"], s["tokens"], temperature=case["temperature"], top=case["top"], with_stats=train)
    out = {"logprobs": got[0], "entropy": got[1]}
    if case["top"]:
        out.update(top_tokens=got[2], top_logprobs=got[3])
    if train:
        out["dlogits"] = ops.log_probs_backward(s["dlogprobs"], s["dentropy"], s["logits"], s["tokens"], got[-1],
                                                temperature=case["temperature"])
    return out


def _conv_own(s, case):
    from paper_1909_05632_amd import ops

    out, final = ops.causal_conv(s["x"], s["weight"], s["bias"], s["seq_off"], state=s["window"])
    result = {"out": out, "state": final}
    if case["kind"] == "train":
        got = ops.causal_conv_backward(s["dout"], s["x"], s["weight"], s["bias"], s["seq_off"], state=s["window"],
                                       dfinal=s["dfinal"])
        result.update(zip(("dx", "dweight", "dbias", "dstate"), got))
    return result


def _scan_own(s, case):
    from paper_1909_05632_amd import ops

    args = (s["u"], s["dt"], s["a"], s["b"], s["c"])
    more = dict(d=s["d"], z=s["z"], dt_bias=s["dt_bias"], seq_off=s["seq_off"])
    if case["kind"] == "forward":
        out, final = ops.scan_forward(*args, **more, state=s["state"])
        return {"out": out, "state": final}
    out, final, saved = ops.scan_forward(*args, **more, state=s["state"], save=True)
    got = ops.scan_backward(s["dout"], *args, **more, saved=saved, dfinal=s["dfinal"])
    result = {"out": out, "state": final}
    result.update(zip(("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias", "dstate"), got))
    return {k: v for k, v in result.items() if v is not None}


def _step_own(s, case):
    from paper_1909_05632_amd import ops

    u = ops.causal_conv_step(s["x"], s["weight"], s["window"], s["bias"])
    out = ops.scan_step(u, s["dt"], s["a"], s["b"], s["c"], s["state"], d=s["d"], z=s["z"], dt_bias=s["dt_bias"])
    return {"out": out, "window": s["window"], "state": s["state"]}


# ------------------------------------------------------------------ plain forms

def _norm_plain(s, case):
    dtype = s["x"].dtype
    total = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dtype)
    h, w = total.float(), s["weight"]
    rstd = torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS)
    out = {} if s["residual"] is None else {"total": total}
    if case["kind"] == "8bit":
        # 1/sd cancels in y over its row's largest, so that what is rounded to 8 bits does not depend on its last bits.
        t = h * w
        largest = t.abs().max(-1, keepdim=True).values
        step = torch.where(largest > 0, E4M3_MAX / largest, 0.0)
        return {"y": (t * step).to(torch.float8_e4m3fn), "scales": (largest * rstd / E4M3_MAX)[:, 0], **out}
    out["y"] = (h * rstd * w).to(dtype)
    if case["kind"] == "train":
        t, hat = s["dy"].float() * w, h * rstd
        dx = rstd * (t - hat * (t * hat).mean(-1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        out.update(dx=dx.to(dtype), dweight=(s["dy"].float() * hat).sum(0))
    return out


def _logp_plain(s, case):
    x, token = s["logits"].float(), s["tokens"].long()[:, None]
    z = (x - x.max(-1, keepdim=True).values) / case["temperature"]
    e = torch.exp(z)
    total = e.sum(-1, keepdim=True)
    p, logp = e / total, z - torch.log(total)
    plogp = torch.where(p > 0, p * logp, 0.0)
    entropy = -plogp.sum(-1, keepdim=True)
    out = {"logprobs": logp.gather(1, token)[:, 0], "entropy": entropy[:, 0]}
    if case["top"]:
        order = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :case["top"]]
        out.update(top_tokens=order.to(torch.int32), top_logprobs=logp.gather(1, order))
    if case["kind"] == "train":
        dlogits = -p * s["dlogprobs"][:, None]
        dlogits.scatter_add_(1, token, s["dlogprobs"][:, None])
        dlogits -= s["dentropy"][:, None] * (plogp + p * entropy)
        out["dlogits"] = (dlogits / case["temperature"]).to(s["logits"].dtype)
    return out


def _sequence_of(s, tokens):
    """Each token's sequence."""
    off = s["seq_off"].long()
    n = off.numel() - 1
    return torch.repeat_interleave(torch.arange(n, device="cuda"), off[1:] - off[:-1], output_size=tokens)


def _conv_plain(s, case):
    """Every sequence behind the window before it, in one array of rows."""
    dtype, taps, tokens = s["x"].dtype, case["taps"], case["tokens"]
    n, channels, w = case["n"], case["channels"], s["weight"]
    off = s["seq_off"].long()
    at = torch.arange(tokens, device="cuda") + (_sequence_of(s, tokens) + 1) * (taps - 1)
    back = torch.arange(taps - 1, device="cuda")
    seq = torch.arange(n, device="cuda")[:, None] * (taps - 1)
    first, last = off[:-1, None] + seq + back, off[1:, None] + seq + back
    rows = torch.empty(tokens + n * (taps - 1), channels, device="cuda")
    rows[at] = s["x"].float()
    rows[first] = s["window"].float()
    pre = s["bias"] + sum(rows[at - (taps - 1) + k] * w[:, k] for k in range(taps))
    gate = torch.sigmoid(pre)
    out = {"out": (pre * gate).to(dtype), "state": rows[last].to(dtype)}
    if case["kind"] == "train":
        dpre = s["dout"].float() * gate * (1 + pre * (1 - gate))
        drows = torch.zeros_like(rows)
        drows[last] = s["dfinal"].float()
        for k in range(taps):
            drows[at - (taps - 1) + k] += dpre * w[:, k]
        out.update(dx=drows[at].to(dtype), dstate=drows[first].to(dtype), dbias=dpre.sum(0),
                   dweight=torch.stack([(dpre * rows[at - (taps - 1) + k]).sum(0) for k in range(taps)], 1))
    return out


def _every_sum(a, b):
    """h_t = a_t h_(t-1) + b_t for all t, by doubling: each pass joins every row with the one that far before it."""
    reach = 1
    while reach < a.shape[0]:
        b = torch.cat([b[:reach], torch.addcmul(b[reach:], a[reach:], b[:-reach])])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def _of_channels(x, channels):
    """[tokens][groups][states] as every channel sees it."""
    x = x.float()
    return x.repeat_interleave(channels // x.shape[1], 1)


def _scan_plain(s, case):
    """All tokens in one array: a sequence's first has a decay of 0, its state goes into what it adds."""
    dtype, tokens, channels = s["u"].dtype, case["tokens"], case["channels"]
    off, u = s["seq_off"].long(), s["u"].float()
    some = off[1:] > off[:-1]
    seq = _sequence_of(s, tokens)
    first = torch.zeros(tokens + 1, dtype=torch.bool, device="cuda").index_fill_(0, off[:-1], True)[:tokens, None, None]
    raw = s["dt"].float() + s["dt_bias"]
    step = _softplus(raw)
    b, c = _of_channels(s["b"], channels), _of_channels(s["c"], channels)
    decay = torch.exp(step[..., None] * s["a"])
    add = (step * u)[..., None] * b
    start = torch.where(first, s["state"][seq], 0.0)
    h = _every_sum(torch.where(first, 0.0, decay), torch.addcmul(add, decay, start))
    y = (h * c).sum(-1) + s["d"] * u
    if s["z"] is not None:
        z = s["z"].float()
        gate = torch.sigmoid(z)
        out = y * z * gate
    else:
        out = y
    final = torch.where(some[:, None, None], h[(off[1:] - 1).clamp(min=0)], s["state"])
    result = {"out": out.to(dtype), "state": final}
    if case["kind"] != "train":
        return result
    dy = s["dout"].float()
    if s["z"] is not None:
        result["dz"] = (dy * y * gate * (1 + z * (1 - gate))).to(dtype)
        dy = dy * z * gate
    last = torch.zeros(tokens + 1, dtype=torch.bool, device="cuda").index_fill_(0, off[1:], True)[1:, None, None]
    grad = dy[..., None] * c + torch.where(last, s["dfinal"][seq], 0.0)
    after = torch.where(last, 0.0, torch.cat([decay[1:], decay[:1]]))
    grad = _every_sum(after.flip(0), grad.flip(0)).flip(0)
    kept = h - add                                  # what the decay left of the state before
    through = grad * kept
    group = channels // case["groups"]
    by_group = lambda x: x.view(tokens, case["groups"], group, -1).sum(2).to(dtype)  # noqa: E731
    dstep = (through * s["a"]).sum(-1) + u * (grad * b).sum(-1)
    draw_ = dstep * torch.sigmoid(raw)
    result.update(du=(step * (grad * b).sum(-1) + s["d"] * dy).to(dtype), ddt=draw_.to(dtype),
                  da=(through * step[..., None]).sum(0), db=by_group(grad * (step * u)[..., None]),
                  dc=by_group(h * dy[..., None]), dd=(dy * u).sum(0), ddt_bias=draw_.sum(0))
    left = (grad * decay)[off[:-1].clamp(max=tokens - 1)]
    result["dstate"] = torch.where(some[:, None, None], left, s["dfinal"])
    return result


def _step_plain(s, case):
    dtype, channels = s["x"].dtype, case["channels"]
    rows = torch.cat([s["window"], s["x"][:, None]], 1)
    pre = s["bias"] + (rows.float() * s["weight"].t()).sum(1)
    u = (pre * torch.sigmoid(pre)).to(dtype).float()
    s["window"].copy_(rows[:, 1:])
    step = _softplus(s["dt"].float() + s["dt_bias"])[..., None]
    b, c = _of_channels(s["b"], channels), _of_channels(s["c"], channels)
    s["state"].mul_(torch.exp(step * s["a"])).add_(step * u[..., None] * b)
    y = (s["state"] * c).sum(-1) + s["d"] * u
    if s["z"] is not None:
        z = s["z"].float()
        y = y * z * torch.sigmoid(z)
    return {"out": y.to(dtype), "window": s["window"], "state": s["state"]}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _norm_exact, "logp": _logp_exact, "conv": _conv_exact, "scan": _scan_exact, "step": _step_exact}[case["op"]](s, case)


def _norm_exact(s, case):
    # The sum is defined as rounded to its type: what follows is of the rounded one.
    total = s["x"] if s["residual"] is None else (s["x"].double() + s["residual"].double()).to(s["x"].dtype)
    x, w = total.double(), s["weight"].double()
    sd = torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS)
    y = x / sd * w
    out = {"y": y} if s["residual"] is None else {"y": y, "total": total.double()}
    if case["kind"] == "8bit":
        scale = y.abs().amax(-1, keepdim=True) / E4M3_MAX
        out.update(y=(y / torch.where(scale > 0, scale, 1.0)).to(torch.float8_e4m3fn).double(), scales=scale[:, 0])
    if case["kind"] == "train":
        dy = s["dy"].double()
        t = dy * w
        inner = (t * x).sum(-1, keepdim=True) / x.shape[-1]
        dx = t / sd - x * inner / sd ** 3
        out["dx"] = dx if s["dtotal"] is None else dx + s["dtotal"].double()
        out["dweight"] = (dy * (x / sd)).sum(0)
    return out


def _logp_exact(s, case):
    parts = []
    n = s["logits"].shape[0]
    for lo in range(0, n, 256):
        rows = slice(lo, lo + 256)
        x = s["logits"][rows].double() / case["temperature"]
        token = s["tokens"][rows].long()
        lse = torch.logsumexp(x, -1, keepdim=True)
        logp = x - lse
        p = torch.exp(logp)
        entropy = -torch.where(p > 0, p * logp, 0.0).sum(-1)
        part = {"logprobs": logp[torch.arange(token.numel(), device="cuda"), token], "entropy": entropy}
        if case["top"]:
            part["top_logprobs"] = torch.sort(logp, dim=-1, descending=True).values[:, :case["top"]]
        if case["kind"] == "train":
            dlp, dent = s["dlogprobs"][rows, None].double(), s["dentropy"][rows, None].double()
            hot = torch.zeros_like(p)
            hot[torch.arange(token.numel(), device="cuda"), token] = 1
            slope = torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
            part["dlogits"] = (dlp * (hot - p) - dent * slope) / case["temperature"]
        parts.append(part)
    out = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
    if case["top"]:
        out["top_tokens"] = None
    return out


def _silu(x):
    return x / (1 + torch.exp(-x))


def _silu_slope(x):
    g = 1 / (1 + torch.exp(-x))
    return g + x * g * (1 - g)


def _conv_exact(s, case):
    """Sequence by sequence, as a sum over the taps of the rows before each."""
    off, taps, w = s["seq_off"].tolist(), case["taps"], s["weight"].double()
    names = ("out", "state") + (("dx", "dstate") if case["kind"] == "train" else ())
    parts = {k: [] for k in names}
    dweight, dbias = torch.zeros_like(w), torch.zeros(w.shape[0], dtype=torch.float64, device="cuda")
    for i in range(case["n"]):
        x = torch.cat([s["window"][i], s["x"][off[i]:off[i + 1]]]).double()
        m = off[i + 1] - off[i]
        pre = s["bias"].double().expand(m, -1).clone()
        for k in range(taps):
            pre += x[k:k + m] * w[:, k]
        parts["out"].append(_silu(pre))
        parts["state"].append(x[m:][None])
        if case["kind"] == "train":
            dpre = s["dout"][off[i]:off[i + 1]].double() * _silu_slope(pre)
            dx = torch.zeros_like(x)
            dx[m:] += s["dfinal"][i].double()
            for k in range(taps):
                dx[k:k + m] += dpre * w[:, k]
                dweight[:, k] += (dpre * x[k:k + m]).sum(0)
            dbias += dpre.sum(0)
            parts["dx"].append(dx[taps - 1:])
            parts["dstate"].append(dx[None, :taps - 1])
    out = {k: torch.cat(v) for k, v in parts.items()}
    if case["kind"] == "train":
        out.update(dweight=dweight, dbias=dbias)
    return out


def _scan_exact(s, case):
    """The recurrence token by token, longest sequences first, and its adjoint walked back."""
    n, train, channels = case["n"], case["kind"] == "train", case["channels"]
    off, group = s["seq_off"].tolist(), channels // case["groups"]
    lengths = [b - a for a, b in zip(off, off[1:])]
    order = sorted(range(n), key=lambda j: -lengths[j])
    begin = torch.tensor([off[j] for j in order], device="cuda")
    order_t = torch.tensor(order, device="cuda")
    counts = [sum(x > t for x in lengths) for t in range(max(lengths))]
    a, d = s["a"].double(), s["d"].double()
    u, raw = s["u"].double(), s["dt"].double() + s["dt_bias"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw))
    b, c = (s[k].double().repeat_interleave(group, 1) if case["groups"] > 1 else s[k].double() for k in ("b", "c"))
    state = s["state"].double()[order_t]
    y = torch.zeros_like(u)
    kept = []
    for t, m in enumerate(counts):
        at = begin[:m] + t
        if train:
            kept.append(state[:m].clone())
        now = state[:m] * torch.exp(step[at][..., None] * a) + (step[at] * u[at])[..., None] * b[at]
        y[at] = (now * c[at]).sum(-1)
        state[:m] = now
    y += d * u
    final = torch.empty_like(state)
    final[order_t] = state
    z = None if s["z"] is None else s["z"].double()
    result = {"out": y if z is None else y * _silu(z), "state": final}
    if not train:
        return result
    dout = s["dout"].double()
    dy = dout if z is None else dout * _silu(z)
    if z is not None:
        result["dz"] = dout * y * _silu_slope(z)
    g = s["dfinal"].double()[order_t]
    du, dstep, da = torch.zeros_like(u), torch.zeros_like(u), torch.zeros_like(a)
    db, dc = (torch.zeros(case["tokens"], case["groups"], case["states"], dtype=torch.float64, device="cuda") for _ in range(2))
    for t in reversed(range(len(counts))):
        m, at = counts[t], begin[:counts[t]] + t
        st, ut = step[at][..., None], u[at][..., None]
        decay = torch.exp(st * a)
        mid = kept[t] * decay
        now = mid + st * ut * b[at]
        kept[t] = None
        by_group = lambda v: v.view(m, case["groups"], group, -1).sum(2)  # noqa: E731
        dc[at] = by_group(now * dy[at][..., None])
        d_now = g[:m] + dy[at][..., None] * c[at]
        db[at] = by_group(d_now * st * ut)
        into = (d_now * b[at]).sum(-1)
        du[at] = step[at] * into
        dstep[at] = (d_now * mid * a).sum(-1) + u[at] * into
        da += (d_now * mid * st).sum(0)
        g[:m] = d_now * decay
    dstate = torch.empty_like(g)
    dstate[order_t] = g
    ddt = dstep / (1 + torch.exp(-raw))
    result.update(du=du + d * dy, ddt=ddt, da=da, db=db, dc=dc, dd=(dy * u).sum(0), ddt_bias=ddt.sum(0), dstate=dstate)
    return result


def _step_exact(s, case):
    group = case["channels"] // case["groups"]
    x = torch.cat([s["window"], s["x"][:, None]], 1)
    pre = s["bias"].double() + (x.double() * s["weight"].double().t()).sum(1)
    # What passes from the convolution to the scan is defined as rounded to the type of both.
    u = _silu(pre).to(s["x"].dtype).double()
    raw = s["dt"].double() + s["dt_bias"].double()
    step = torch.logaddexp(raw, torch.zeros_like(raw))[..., None]
    b, c = (s[k].double().repeat_interleave(group, 1) for k in ("b", "c"))
    state = s["state"].double() * torch.exp(step * s["a"].double()) + step * u[..., None] * b
    y = (state * c).sum(-1) + s["d"].double() * u
    return {"out": y if s["z"] is None else y * _silu(s["z"].double()), "window": x[:, 1:].double(), "state": state}
