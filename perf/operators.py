"""Cases of the operators around a policy net: layer norm, the gated delta rule's memory, and the sampling of actions.

A policy over streams of frames normalises each frame's features, carries a
memory from frame to frame (a matrix per head that decays, forgets what it
holds under a key and writes the new value), and draws an action from its
logits.  A case is one such call, or one with its gradients: the smallest are a
single stream's frame, where the call itself is what costs, the ordinary ones
are the rollouts and training batches of this repository's benchmark (256 and
1024 streams, 16-frame episodes, 6 and 18 actions, 80 features), the largest
are of the sizes that language models run the same operators at.

Where ``own`` is false, ``run`` computes a case in elementary torch operations
in float32, rounded once at the end; where it is true, it calls the operators
of ``paper_1909_05632_amd``.  ``exact`` evaluates the definitions in float64:
the memory token by token, as its recurrence is written.
"""
from __future__ import annotations

import math
import random

import torch

own = False                # True: the framework's operators, False: plain torch

CHUNK = 64                 # tokens that the plain form of the memory takes at a time
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------ cases

def _norm(rows, width, dtype, train):
    return dict(op="norm", rows=rows, width=width, dtype=dtype, train=train)


def _delta(kind, n, tokens, hk, hv, dk, dv, dtype, ragged=False):
    return dict(op="delta", kind=kind, n=n, tokens=tokens, hk=hk, hv=hv, dk=dk, dv=dv, dtype=dtype, ragged=ragged)


def _sample(n, vocab, dtype, per_row, scale):
    return dict(op="sample", n=n, vocab=vocab, dtype=dtype, per_row=per_row, scale=scale)


def listed():
    return [
        # One stream acting: the features of its frame.
        dict(_norm(1, 512, "f32", False), name="norm-1x512"),
        # A training batch: 256 streams x 64 frames of 80 features, forward and gradients.
        dict(_norm(16384, 80, "f32", True), name="norm-train-16384x80"),
        # A wide model's training batch in bfloat16, forward and gradients.
        dict(_norm(16384, 4096, "bf16", True), name="norm-train-16384x4096-bf16"),
        # One stream's memory, one frame.
        dict(_delta("step", 1, 1, 2, 4, 64, 64, "f32"), name="delta-step-1"),
        # Serving 1024 streams, one frame each: half a gigabyte of states read and written.
        dict(_delta("step", 1024, 1024, 4, 8, 128, 128, "bf16"), name="delta-step-1024-bf16"),
        # The benchmark's training episodes seen forward: 256 streams x 16 frames.
        dict(_delta("forward", 256, 4096, 4, 4, 64, 64, "f32"), name="delta-fwd-256x16"),
        # Histories of odd lengths taken in at once, heads sharing keys.
        dict(_delta("forward", 5, 16384, 4, 16, 128, 128, "bf16", True), name="delta-fwd-ragged16384-bf16"),
        # The same training episodes with their gradients.
        dict(_delta("train", 256, 4096, 4, 4, 64, 64, "f32"), name="delta-train-256x16"),
        # Long episodes of odd lengths with their gradients, heads sharing keys.
        dict(_delta("train", 7, 8192, 4, 8, 128, 128, "bf16", True), name="delta-train-ragged8192-bf16"),
        # One stream's action out of 6.
        dict(_sample(1, 6, "f32", False, 1.5), name="sample-1x6"),
        # 1024 streams' actions out of 18, each stream with settings of its own.
        dict(_sample(1024, 18, "f32", True, 1.5), name="sample-1024x18"),
        # The largest: as many choices as a language model's vocabulary has.
        dict(_sample(256, 131072, "bf16", True, 2.5), name="sample-256x131072-bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "delta", "delta", "sample"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "norm":
        width = _log(rng, 18, 8192)
        return _norm(_log(rng, 1, min(65536, 2 ** 26 // width)), width, dtype, rng.random() < 0.6)
    if op == "sample":
        vocab = _log(rng, 2, 131072)
        return _sample(_log(rng, 1, min(4096, 2 ** 25 // vocab)), vocab, dtype, rng.random() < 0.6,
                       rng.choice((0.5, 1.5, 2.5)))
    kind = rng.choice(("step", "forward", "train"))
    hk, group = rng.choice((1, 2, 3, 4)), rng.choice((1, 1, 2, 4))
    dk, dv = rng.choice((32, 48, 64, 72, 96, 100, 128)), rng.choice((32, 40, 64, 80, 90, 128))
    per_head = hk * group * dk * dv
    if kind == "step":
        n = _log(rng, 1, min(1024, 2 ** 27 // per_head))
        return _delta(kind, n, n, hk, hk * group, dk, dv, dtype)
    n = _log(rng, 1, 256)
    most = (2 ** 30 if kind == "train" else 2 ** 32) // per_head
    if rng.random() < 0.5:
        frames = _log(rng, 1, max(1, min(512, 16384, most) // n))
        return _delta(kind, n, n * frames, hk, hk * group, dk, dv, dtype)
    return _delta(kind, n, _log(rng, n, max(n, min(8192, most))), hk, hk * group, dk, dv, dtype, True)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        every = rows * width
        if not case["train"]:
            return {"bytes": 2.0 * size * every + 8 * width, "flops": 7.0 * every}
        return {"bytes": 4.0 * size * every + 16 * width, "flops": 18.0 * every}
    if case["op"] == "sample":
        n, vocab = case["n"], case["vocab"]
        return {"bytes": float(size * n * vocab + n * (12 + 16 * case["per_row"])), "flops": 4.0 * n * vocab}
    tokens, hk, hv, dk, dv = (case[k] for k in ("tokens", "hk", "hv", "dk", "dv"))
    qkv = tokens * (2 * hk * dk + hv * dv) * size + tokens * hv * 8
    states = 2 * case["n"] * hv * dk * dv * 4
    out = tokens * hv * dv * size
    # k^T S, the rank-one update and q^T S, each 2 dk dv; their gradients twice that.
    flops = 6.0 * tokens * hv * dk * dv
    if case["kind"] != "train":
        return {"bytes": float(qkv + states + out), "flops": flops}
    # and dO, the gradients of all inputs, and of the first and last states
    return {"bytes": float(2 * qkv + 2 * states + 2 * out), "flops": 3 * flops}


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

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    def rand(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    dtype = DTYPES[case["dtype"]]
    s = {"case": dict(case)}
    if case["op"] == "norm":
        rows, width = case["rows"], case["width"]
        # Features after a ReLU-like layer: their mean is not 0, their scale differs from row to row.
        s["x"] = ((randn(rows, width) + 0.7) * torch.exp(randn(rows, 1))).to(dtype)
        s["weight"] = 1 + 0.1 * randn(width)
        s["bias"] = 0.1 * randn(width)
        if case["train"]:
            s["dy"] = randn(rows, width, dtype=dtype)
        return s
    if case["op"] == "sample":
        n, vocab = case["n"], case["vocab"]
        s["logits"] = (case["scale"] * randn(n, vocab)).to(dtype)
        s["u"] = rand(n)
        if case["per_row"]:
            # Every stream has its own settings; some are greedy, some leave a filter off.
            s["temperature"] = torch.where(rand(n) < 0.1, torch.zeros(n, device="cuda"), 0.5 + rand(n))
            s["top_k"] = torch.where(rand(n) < 0.3, torch.zeros(n, device="cuda"),
                                     1 + rand(n) * min(vocab, 200)).to(torch.int32)
            s["top_p"] = torch.where(rand(n) < 0.3, torch.ones(n, device="cuda"), 0.3 + 0.69 * rand(n))
            s["min_p"] = torch.where(rand(n) < 0.5, torch.zeros(n, device="cuda"), 0.2 * rand(n))
        else:
            s.update(temperature=0.9, top_k=0, top_p=0.95, min_p=0.0)
        return s
    n, tokens, hk, hv, dk, dv = (case[k] for k in ("n", "tokens", "hk", "hv", "dk", "dv"))
    # Keys and queries of unit length that change little from frame to frame; values of any size.
    near = randn(1, hk, dk)
    k = near * 0.5 + randn(tokens, hk, dk)
    q = near * 0.5 + randn(tokens, hk, dk)
    s["k"] = (k / k.norm(dim=-1, keepdim=True)).to(dtype)
    s["q"] = (q / q.norm(dim=-1, keepdim=True)).to(dtype)
    s["v"] = randn(tokens, hv, dv, dtype=dtype)
    s["g"] = -torch.exp(math.log(1e-3) + (math.log(1.0) - math.log(1e-3)) * rand(tokens, hv))
    s["beta"] = torch.sigmoid(randn(tokens, hv))
    s["state"] = 0.1 * randn(n, hv, dk, dv)
    s["scale"] = dk ** -0.5
    if case["kind"] != "step":
        off = _offsets(case, seed)
        s["seq_off"] = torch.tensor(off, dtype=torch.int32, device="cuda")
        s["longest"] = max(b - a for a, b in zip(off, off[1:]))
    if case["kind"] == "train":
        s["dout"] = randn(tokens, hv, dv, dtype=dtype)
        s["dfinal"] = 0.1 * randn(n, hv, dk, dv)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    case = s["case"]
    if case["op"] == "norm":
        return (_norm_own if own else _norm_plain)(s, case["train"])
    if case["op"] == "sample":
        return (_sample_own if own else _sample_plain)(s)
    if case["kind"] == "step":
        return (_step_own if own else _step_plain)(s)
    return (_delta_own if own else _delta_plain)(s, case["kind"] == "train")


def _norm_own(s, train):
    from paper_1909_05632_amd import ops

    if not train:
        return {"y": ops.layer_norm(s["x"], s["weight"], s["bias"], EPS)}
    y, stats = ops.layer_norm(s["x"], s["weight"], s["bias"], EPS, with_stats=True)
    dx, dweight, dbias = ops.layer_norm_backward(s["dy"], s["x"], s["weight"], stats)
    return {"y": y, "dx": dx, "dweight": dweight, "dbias": dbias}


def _sample_own(s):
    from paper_1909_05632_amd import ops

    tokens, logprobs = ops.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                                  top_p=s["top_p"], min_p=s["min_p"])
    return {"tokens": tokens, "logprobs": logprobs}


def _step_own(s):
    from paper_1909_05632_amd import ops

    out = ops.delta_step(s["q"], s["k"], s["v"], s["g"], s["beta"], s["state"], scale=s["scale"])
    return {"out": out, "state": s["state"]}


def _delta_own(s, train):
    from paper_1909_05632_amd import ops

    args = (s["q"], s["k"], s["v"], s["g"], s["beta"], s["seq_off"])
    if not train:
        out, final = ops.delta_forward(*args, state=s["state"], scale=s["scale"])
        return {"out": out, "state": final}
    out, final, saved = ops.delta_forward(*args, state=s["state"], scale=s["scale"], save=True)
    dq, dk, dv, dg, dbeta, dstate = ops.delta_backward(s["dout"], *args, saved=saved, dfinal=s["dfinal"],
                                                       scale=s["scale"])
    return {"out": out, "state": final, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "dbeta": dbeta, "dstate": dstate}


# ------------------------------------------------------------------ plain forms

def _norm_plain(s, train):
    x, w = s["x"].float(), s["weight"]
    mean = x.mean(-1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(-1, keepdim=True) + EPS)
    xhat = (x - mean) * rstd
    out = {"y": (xhat * w + s["bias"]).to(s["x"].dtype)}
    if train:
        dy = s["dy"].float()
        dxhat = dy * w
        dx = rstd * (dxhat - dxhat.mean(-1, keepdim=True) - xhat * (dxhat * xhat).mean(-1, keepdim=True))
        out.update(dx=dx.to(s["x"].dtype), dweight=(dy * xhat).sum(0), dbias=dy.sum(0))
    return out


LOG2E = 1.4426950408889634
LN2 = 0.6931471805599453
ONE = 2.0 ** 31            # the weight of a row's largest logit


def _per_row(v, n, dtype):
    return v.to(dtype) if isinstance(v, torch.Tensor) else torch.full((n,), v, dtype=dtype, device="cuda")


def _sample_plain(s):
    """Weights are whole multiples of 2^-31 of the largest logit's, so their sums have one value in any order."""
    logits, u = s["logits"].float(), s["u"]
    n, vocab = logits.shape
    temp = _per_row(s["temperature"], n, torch.float32)[:, None]
    top_k = _per_row(s["top_k"], n, torch.int64)[:, None]
    top_p = _per_row(s["top_p"], n, torch.float32)[:, None]
    min_p = _per_row(s["min_p"], n, torch.float32)[:, None]
    greedy = temp <= 0
    z = (logits - logits.max(-1, keepdim=True).values) * (LOG2E / torch.where(greedy, 1.0, temp))
    e = torch.exp2(z)
    weight = torch.round(e * ONE).long() * (e >= min_p)
    order = torch.sort(logits, dim=-1, descending=True, stable=True).indices
    sorted_w = weight.gather(1, order)
    rank = torch.arange(vocab, device="cuda")[None]
    sorted_w = sorted_w * ((rank < top_k) | (top_k <= 0)) * ((rank == 0) | ~greedy)
    total = sorted_w.sum(-1, keepdim=True).double()
    before = (sorted_w.cumsum(-1) - sorted_w).double()
    sorted_w = sorted_w * ((before < top_p.double() * total) | (rank == 0))
    kept = torch.zeros_like(weight).scatter_(1, order, sorted_w)
    upto = kept.cumsum(-1)
    total = upto[:, -1:]
    target = torch.minimum((u[:, None].double() * total.double()).long(), total - 1)
    token = (upto <= target).sum(-1)
    share = torch.log2(total[:, 0].double().mul(1 / ONE).float())
    logprob = (z.gather(1, token[:, None])[:, 0] - share) * LN2
    return {"tokens": token.to(torch.int32), "logprobs": torch.where(greedy[:, 0], 0.0, logprob)}


def _step_plain(s):
    group = s["v"].shape[1] // s["q"].shape[1]
    q, k = (s[x].float().repeat_interleave(group, 1) for x in ("q", "k"))
    state, beta = s["state"], s["beta"][..., None]
    state.mul_(torch.exp(s["g"])[..., None, None])
    held = (k[..., None] * state).sum(-2)
    state.add_(k[..., None] * (beta * (s["v"].float() - held))[..., None, :])
    out = s["scale"] * (q[..., None] * state).sum(-2)
    return {"out": out.to(s["v"].dtype), "state": state}


def _padded(s):
    """Tokens as [n][heads][chunks][CHUNK][...] with zeros after each sequence's end, and where each came from."""
    off = s["seq_off"].long()
    n, chunks = off.numel() - 1, max(1, -(-s["longest"] // CHUNK))
    at = off[:-1, None] + torch.arange(chunks * CHUNK, device="cuda")
    valid = at < off[1:, None]
    at = at.clamp_(max=max(0, s["q"].shape[0] - 1))
    group = s["v"].shape[1] // s["q"].shape[1]

    def lay(x):
        x = x.float()
        if x.shape[1] != s["v"].shape[1]:
            x = x.repeat_interleave(group, 1)
        x = x[at] * valid.view(*valid.shape, *([1] * (x.dim() - 1)))
        return x.transpose(1, 2).reshape(n, x.shape[2], chunks, CHUNK, *x.shape[3:])

    def back(x, dtype):
        x = x.reshape(n, x.shape[1], chunks * CHUNK, *x.shape[4:]).transpose(1, 2)
        return x[valid].to(dtype)

    return lay, back, chunks


def _delta_plain(s, train):
    """The chunked form: within a chunk the written values V' solve (I + A) V' = beta (V - e^c K S), S the state before it."""
    lay, back, chunks = _padded(s)
    q, k, v, g, beta = (lay(s[x]) for x in ("q", "k", "v", "g", "beta"))
    q = q * s["scale"]
    c = g.cumsum(-1)
    i = torch.arange(CHUNK, device="cuda")
    decay = torch.exp((c[..., :, None] - c[..., None, :]).masked_fill(i[:, None] < i, -math.inf))
    kt = k.transpose(-1, -2).contiguous()
    score = torch.matmul(q, kt) * decay
    a = beta[..., None] * torch.matmul(k, kt) * decay * (i[:, None] > i)
    inv = torch.eye(CHUNK, device="cuda").expand_as(a).clone()
    for r in range(1, CHUNK):              # forward substitution
        inv[..., r, :r] = -torch.matmul(a[..., r:r + 1, :r], inv[..., :r, :r].contiguous())[..., 0, :]
    grown, left = torch.exp(c)[..., None], torch.exp(c[..., -1:] - c)[..., None]
    whole = torch.exp(c[..., -1])[..., None, None]
    k_in, k_out, q_in = k * grown, k * left, q * grown
    state = s["state"]
    before, held, new, out = [], [], [], []
    for t in range(chunks):
        before.append(state)
        held.append(torch.matmul(k_in[:, :, t], state))
        new.append(torch.matmul(inv[:, :, t], beta[:, :, t, :, None] * (v[:, :, t] - held[t])))
        out.append(torch.matmul(q_in[:, :, t], state) + torch.matmul(score[:, :, t], new[t]))
        state = whole[:, :, t] * state + torch.matmul(k_out[:, :, t].transpose(-1, -2).contiguous(), new[t])
    result = {"out": back(torch.stack(out, 2), s["v"].dtype), "state": state}
    if not train:
        return result

    dout, dstate = lay(s["dout"]), s["dfinal"]
    score_t, inv_t = (x.transpose(-1, -2).contiguous() for x in (score, inv))
    after, dnew, dwrite = [None] * chunks, [None] * chunks, [None] * chunks
    for t in reversed(range(chunks)):
        after[t] = dstate
        dnew[t] = torch.matmul(score_t[:, :, t], dout[:, :, t]) + torch.matmul(k_out[:, :, t], dstate)
        dwrite[t] = torch.matmul(inv_t[:, :, t], dnew[t])
        dstate = (whole[:, :, t] * dstate + torch.matmul(q_in[:, :, t].transpose(-1, -2).contiguous(), dout[:, :, t])
                  - torch.matmul((k_in * beta[..., None])[:, :, t].transpose(-1, -2).contiguous(), dwrite[t]))
    before, held, new, after, dwrite = (torch.stack(x, 2) for x in (before, held, new, after, dwrite))
    before_t, after_t, new_t = (x.transpose(-1, -2).contiguous() for x in (before, after, new))
    dv = beta[..., None] * dwrite
    dscore = torch.matmul(dout, new_t) * (i[:, None] >= i)
    da = -torch.matmul(dwrite, new_t) * (i[:, None] > i)
    dq_in, dk_in, dk_out = torch.matmul(dout, before_t), -torch.matmul(dv, before_t), torch.matmul(new, after_t)
    in_score, in_a = dscore * decay, da * decay * beta[..., None]
    dq = grown * dq_in + torch.matmul(in_score, k)
    dk = (grown * dk_in + left * dk_out + torch.matmul(in_score.transpose(-1, -2).contiguous(), q)
          + torch.matmul(in_a, k) + torch.matmul(in_a.transpose(-1, -2).contiguous(), k))
    pairs = dscore * score + da * a
    out_part = (k_out * dk_out).sum(-1)
    dc = pairs.sum(-1) - pairs.sum(-2) + (q_in * dq_in).sum(-1) + (k_in * dk_in).sum(-1) - out_part
    dc[..., -1] += out_part.sum(-1) + (whole * before * after).sum((-1, -2))
    dbeta = (dwrite * (v - held)).sum(-1) + (da * torch.matmul(k, kt) * decay).sum(-1)
    dg = dc.flip(-1).cumsum(-1).flip(-1)
    hk, tokens, group = s["q"].shape[1], s["q"].shape[0], s["v"].shape[1] // s["q"].shape[1]
    dq, dk = (back(x, torch.float32).view(tokens, hk, group, -1).sum(2).to(s["q"].dtype) for x in (dq * s["scale"], dk))
    result.update(dq=dq, dk=dk, dv=back(dv, s["v"].dtype), dg=back(dg, torch.float32),
                  dbeta=back(dbeta, torch.float32), dstate=dstate)
    return result


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _norm_exact(s, case["train"])
    if case["op"] == "sample":
        return _sample_exact(s)
    return _delta_exact(s, case)


def _norm_exact(s, train):
    x, w = s["x"].double(), s["weight"].double()
    var, mean = torch.var_mean(x, dim=-1, correction=0, keepdim=True)
    sd = torch.sqrt(var + EPS)
    out = {"y": (x - mean) / sd * w + s["bias"].double()}
    if train:
        xhat, t = (x - mean) / sd, s["dy"].double() * w
        out["dx"] = (t - t.mean(-1, keepdim=True) - xhat * (t * xhat).mean(-1, keepdim=True)) / sd
        out["dweight"] = (s["dy"].double() * xhat).sum(0)
        out["dbias"] = s["dy"].double().sum(0)
    return out


def _sample_exact(s):
    """The log-probability that each row's draw has; None where a draw lies too near an edge between two to tell."""
    n, vocab = s["logits"].shape
    temp, top_p, min_p = (_per_row(s[x], n, torch.float64) for x in ("temperature", "top_p", "min_p"))
    top_k = _per_row(s["top_k"], n, torch.int64)
    result = torch.zeros(n, dtype=torch.float64, device="cuda")
    near = 3e-8
    for lo in range(0, n, 64):
        rows = slice(lo, lo + 64)
        x, t = s["logits"][rows].double(), temp[rows, None]
        p = torch.softmax(x / torch.where(t > 0, t, 1.0), -1)
        ordered, order = torch.sort(x, dim=-1, descending=True, stable=True)
        p = p.gather(1, order)
        rank = torch.arange(vocab, device="cuda")[None]
        ratio = p / p[:, :1]
        p = p * (ratio >= min_p[rows, None]) * ((rank < top_k[rows, None]) | (top_k[rows, None] <= 0))
        p = p / p.sum(-1, keepdim=True)
        cum = p.cumsum(-1) - p
        p = p * ((cum < top_p[rows, None]) | (rank == 0))
        p = p / p.sum(-1, keepdim=True)
        spread = torch.zeros_like(p).scatter_(1, order, p)
        cum = spread.cumsum(-1)
        u = s["u"][rows, None].double()
        edge = (((cum - u).abs() < near) & (spread > 0)).any(-1)
        if bool((edge & (t[:, 0] > 0)).any()):
            return None
        token = (cum <= u).sum(-1, keepdim=True).clamp_(max=vocab - 1)
        result[rows] = torch.where(t[:, 0] > 0, torch.log(spread.gather(1, token)[:, 0]), 0.0)
    return {"tokens": None, "logprobs": result}


def _delta_exact(s, case):
    """The recurrence token by token, longest sequences first, and its adjoint walked back."""
    n, train = case["n"], case["kind"] == "train"
    off = _offsets(case, seed=0) if case["kind"] == "step" else s["seq_off"].tolist()
    group = case["hv"] // case["hk"]
    q, k, v, g, beta = (s[x].double() for x in ("q", "k", "v", "g", "beta"))
    q, k = (x.repeat_interleave(group, 1) for x in (q * s["scale"], k))
    lengths = [b - a for a, b in zip(off, off[1:])]
    order = sorted(range(n), key=lambda j: -lengths[j])
    begin = torch.tensor([off[j] for j in order], device="cuda")
    order_t = torch.tensor(order, device="cuda")
    state = s["state"].double()[order_t]
    out = torch.zeros(v.shape, dtype=torch.float64, device="cuda")
    kept, counts = [], []
    for t in range(max(lengths)):
        m = sum(x > t for x in lengths)
        counts.append(m)
        at = begin[:m] + t
        if train:
            kept.append(state[:m].clone())
        now = state[:m] * torch.exp(g[at])[..., None, None]
        err = beta[at][..., None] * (v[at] - torch.matmul(k[at][..., None, :], now)[..., 0, :])
        now += k[at][..., None] * err[..., None, :]
        out[at] = torch.matmul(q[at][..., None, :], now)[..., 0, :]
        state[:m] = now
    final = torch.empty_like(state)
    final[order_t] = state
    result = {"out": out, "state": final}
    if not train:
        return result
    dout, ds = s["dout"].double(), s["dfinal"].double()[order_t]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dg, dbeta = torch.zeros_like(g), torch.zeros_like(beta)
    for t in reversed(range(len(counts))):
        m, at = counts[t], begin[:counts[t]] + t
        kt, bt, do = k[at], beta[at][..., None], dout[at]
        a = torch.exp(g[at])[..., None, None]
        mid = kept[t] * a                                       # decayed, not yet written to
        gap = v[at] - torch.matmul(kt[..., None, :], mid)[..., 0, :]
        now = mid + kt[..., None] * (bt * gap)[..., None, :]
        dq[at] = torch.matmul(now, do[..., None])[..., 0]
        d = ds[:m] + q[at][..., None] * do[..., None, :]
        derr = torch.matmul(kt[..., None, :], d)[..., 0, :]      # of beta (v - k^T mid)
        dbeta[at] = (derr * gap).sum(-1)
        dv[at] = bt * derr
        dk[at] = torch.matmul(d, (bt * gap)[..., None])[..., 0] - torch.matmul(mid, (bt * derr)[..., None])[..., 0]
        d = d - kt[..., None] * (bt * derr)[..., None, :]
        dg[at] = (d * mid).sum((-1, -2))
        ds[:m] = d * a
        kept[t] = None
    dstate = torch.empty_like(ds)
    dstate[order_t] = ds
    dq, dk = (x.view(x.shape[0], case["hk"], group, -1).sum(2) for x in (dq * s["scale"], dk))
    result.update(dq=dq, dk=dk, dv=dv, dg=dg, dbeta=dbeta, dstate=dstate)
    return result
