"""The operators on whole token arrays: layer norm, the gated linear recurrence and the distillation loss, as cases to measure.

Each case is a dict of plain values: the operator, its direction, type and sizes.  prepare() makes the inputs that a user's
program holds before the call; run() makes one pass, in plain torch operations, or, with `own` set, through
paper_1705_09786_amd.operators; exact() gives the same outputs in 64 bits from the operators' definitions.

  layer norm     y = (x - mean) / sqrt(var + eps) * w + b over the last axis
  recurrence     h_t = (1 - z_t) h_{t-1} + z_t act(c_t), z = sigmoid(gate), packed sequences, h before the first row = h0
  distillation   T^2 w KL(p || q), p = softmax of a teacher's K top logits / T, q = softmax of the student's logits / T
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def _norm(name, **kw):
    return dict(dict(name=name, op="norm", mode="train", dtype="bf16", rows=4096, cols=2048), **kw)


def _scan(name, **kw):
    return dict(dict(name=name, op="scan", mode="train", dtype="bf16", hidden=2048, sequences=8, min_len=1, max_len=4096, act="none"), **kw)


def _distill(name, **kw):
    return dict(dict(name=name, op="distill", mode="train", dtype="bf16", rows=4096, vocab=32000, top=64, temperature=2.0), **kw)


def listed():
    return [
        # serving: one new token for each of 48 sequences, the recurrent state kept between the calls
        _scan("scan_step", mode="step", sequences=48, min_len=1, max_len=1),
        # the benchmark's recurrent workload as one array: 4,000 sequences of 4 .. 32 tokens, hidden 128, scored forward only
        _scan("scan_short_sequences", mode="forward", dtype="f32", hidden=128, sequences=4000, min_len=4, max_len=32, act="tanh"),
        # reading one very long document: parallel over time or not at all
        _scan("scan_long_document", mode="forward", sequences=1, min_len=65536, max_len=65536),
        # a training step of the recurrence on packed documents of very different lengths
        _scan("scan_train", hidden=2560, sequences=24, min_len=16, max_len=3400),
        # the same at a hidden size that is no multiple of anything, with the GRU's tanh, in 32 bits
        _scan("scan_train_odd", dtype="f32", hidden=150, sequences=300, min_len=1, max_len=700, act="tanh"),
        # serving: the norm in front of a layer for 48 single tokens
        _norm("norm_step", mode="forward", rows=48, cols=2048),
        # a training step's norm over a batch of 32,768 tokens
        _norm("norm_train", rows=32768, cols=4096),
        # rows of the trees' hidden size in 32 bits: many short rows
        _norm("norm_train_short_rows", dtype="f32", rows=17088, cols=150),
        # wide rows of odd length, forward only
        _norm("norm_wide_odd", mode="forward", dtype="f16", rows=2500, cols=11111),
        # the last few tokens of a batch: four rows of the trees' vocabulary in 32 bits, parallel over the vocabulary or not at all
        _distill("distill_few_rows", dtype="f32", rows=4, vocab=20000, top=16),
        # a training step's loss and gradient
        _distill("distill_train", rows=8192, vocab=32000, top=64),
        # a large vocabulary and a teacher that kept more of its logits
        _distill("distill_large_vocabulary", rows=4096, vocab=131072, top=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "scan", "scan", "distill"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if op == "norm":
        cols = _log_int(rng, 16, 16384)
        rows = _log_int(rng, 1, min(65536, 100_000_000 // cols))
        return dict(op=op, mode=rng.choice(("train", "train", "forward")), dtype=dtype, rows=rows, cols=cols)
    if op == "scan":
        hidden = _log_int(rng, 16, 4096)
        mode = rng.choice(("train", "train", "forward", "step"))
        if mode == "step":
            return dict(op=op, mode=mode, dtype=dtype, hidden=hidden, sequences=_log_int(rng, 1, 1024), min_len=1, max_len=1,
                        act=rng.choice(("none", "tanh")))
        tokens = _log_int(rng, 16, min(131072, 85_000_000 // hidden))
        sequences = _log_int(rng, 1, min(4000, tokens))
        longest = max(1, 2 * tokens // sequences - 1)
        return dict(op=op, mode=mode, dtype=dtype, hidden=hidden, sequences=sequences,
                    min_len=rng.choice((0, 1)) if sequences >= 8 else 1, max_len=longest, act=rng.choice(("none", "tanh")))
    vocab = _log_int(rng, 1000, 160000)
    rows = _log_int(rng, 1, min(16384, 250_000_000 // vocab))
    return dict(op=op, mode=rng.choice(("train", "train", "forward")), dtype=dtype, rows=rows, vocab=vocab,
                top=_log_int(rng, 1, 256), temperature=rng.choice((1.0, 2.0, 4.0)))


def _lengths(c, gen):
    """Lengths of the packed sequences, from the seed, their sum the same for every seed; 0 is a length."""
    got = torch.randint(c["min_len"], c["max_len"] + 1, (c["sequences"],), generator=gen).tolist()
    over = sum(got) - _tokens(c)
    for k, n in enumerate(got):
        got[k] = max(c["min_len"], min(c["max_len"], n - over))
        over -= n - got[k]
    return torch.tensor(got)


def prepare(c, seed):
    dev = "cuda"
    host = torch.Generator()
    host.manual_seed(seed)
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    t = DTYPES[c["dtype"]]
    s = dict(c)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    if c["op"] == "norm":
        # a residual stream: features with offsets of their own, a few of them much larger than the rest
        scale = torch.exp(0.5 * normal(c["cols"]))
        s["x"] = (normal(c["rows"], c["cols"]) * scale + 0.5 * normal(c["cols"])).to(t)
        s["weight"] = 1.0 + 0.1 * normal(c["cols"])
        s["bias"] = 0.1 * normal(c["cols"])
        if c["mode"] == "train":
            s["dy"] = (0.1 * normal(c["rows"], c["cols"])).to(t)
    elif c["op"] == "scan":
        n, h = c["sequences"], c["hidden"]
        offsets = torch.zeros(n + 1, dtype=torch.int64)
        offsets[1:] = torch.cumsum(_lengths(c, host), 0)
        total = int(offsets[-1])
        # gates whose features remember from one token to some hundreds of them
        reach = torch.rand(h, generator=gen, device=dev) * 7.0 - 6.0
        s["gate"] = (normal(total, h) + reach).to(t)
        s["cand"] = normal(total, h).to(t)
        s["h0"] = 0.3 * normal(n, h)
        s["offsets"] = offsets.to(dev)
        if c["mode"] == "train":
            s["dh"] = (0.1 * normal(total, h)).to(t)
            s["dlast"] = 0.1 * normal(n, h)
    else:
        rows, vocab, top = c["rows"], c["vocab"], min(c["top"], c["vocab"])
        # the teacher's entries lie anywhere in the vocabulary, once each, and the student has begun to learn them
        lane = vocab // top
        pick = torch.randint(0, lane, (rows, top), generator=gen, device=dev)
        s["index"] = pick + lane * torch.arange(top, device=dev)
        s["teacher"] = 9.0 + 2.5 * normal(rows, top)
        logits = 1.5 * normal(rows, vocab)
        logits.scatter_add_(1, s["index"], 0.7 * s["teacher"])
        s["logits"] = logits.to(t)
        s["weight"] = (torch.rand(rows, generator=gen, device=dev) < 0.9) / float(rows)
    return s


# ------------------------------------------------------------------ plain forms, in 32 bits
def _norm_plain(s):
    t = s["x"].dtype
    x = s["x"].float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    n = d * rstd
    y = (n * s["weight"] + s["bias"]).to(t)
    if s["mode"] == "forward":
        return y
    dy = s["dy"].float()
    q = dy * s["weight"]
    dx = rstd * (q - q.mean(1, keepdim=True) - n * (q * n).mean(1, keepdim=True))
    return y, dx.to(t), (dy * n).sum(0), dy.sum(0)


def _compose(a, b):
    """Every row's state of x_t = a_t x_{t-1} + b_t, x before the first row 0, by doubling the span that a row has taken in."""
    span = 1
    while span < a.shape[0]:
        b = torch.cat([b[:span], b[span:] + a[span:] * b[:-span]])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _gates(s):
    z = torch.sigmoid(s["gate"].float())
    a = torch.sigmoid(-s["gate"].float())
    v = s["cand"].float()
    return z, a, torch.tanh(v) if s["act"] == "tanh" else v


def _scan_plain(s):
    t = s["gate"].dtype
    z, a, v = _gates(s)
    if s["mode"] == "step":
        s["h0"].copy_(a * s["h0"] + z * v)
        return s["h0"].to(t), s["h0"]
    begin, end = s["offsets"][:-1], s["offsets"][1:]
    some = end > begin
    first, last = begin[some], end[some] - 1
    b = z * v
    b[first] += a[first] * s["h0"][some]
    keep = a.clone()
    keep[first] = 0.0
    h = _compose(keep, b)
    end_state = s["h0"].clone()
    end_state[some] = h[last]
    if s["mode"] == "forward":
        return h.to(t), end_state
    before = torch.roll(h, 1, 0)
    before[first] = s["h0"][some]
    g = s["dh"].float()
    g[last] += s["dlast"][some]
    g = _compose(torch.roll(keep, -1, 0).flip(0), g.flip(0)).flip(0)
    dgate = g * z * a * (v - before)
    dcand = g * z * (1.0 - v * v) if s["act"] == "tanh" else g * z
    dh0 = s["dlast"].clone()
    dh0[some] = a[first] * g[first]
    return h.to(t), end_state, dgate.to(t), dcand.to(t), dh0


def _distill_plain(s):
    t, temp, rows = s["logits"].dtype, s["temperature"], s["logits"].shape[0]
    x = s["logits"].float() / temp
    x = x - x.max(1, keepdim=True).values
    e = torch.exp(x)
    norm = e.sum(1, keepdim=True)
    y = s["teacher"] / temp
    y = y - y.max(1, keepdim=True).values
    f = torch.exp(y)
    mass = f.sum(1, keepdim=True)
    p = f / mass
    log_p, log_q = y - torch.log(mass), x.gather(1, s["index"]) - torch.log(norm)
    loss = s["weight"] * temp * temp * (p * (log_p - log_q)).sum(1)
    if s["mode"] == "forward":
        return loss
    grad = (e / norm).scatter_add_(1, s["index"], -p)
    return loss, (grad * (s["weight"] * temp).reshape(rows, 1)).to(t)


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    from paper_1705_09786_amd import operators as ops
    if s["op"] == "norm":
        if s["mode"] == "forward":
            return ops.layer_norm(s["x"], s["weight"], s["bias"], EPS)
        y, mean, rstd = ops.layer_norm(s["x"], s["weight"], s["bias"], EPS, stats=True)
        return (y,) + ops.layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd)
    if s["op"] == "scan":
        if s["mode"] == "step":
            return ops.gated_scan_step(s["gate"], s["cand"], s["h0"], activation=s["act"]), s["h0"]
        train = s["mode"] == "train"
        h, last, carry = ops.gated_scan(s["gate"], s["cand"], s["offsets"], h0=s["h0"], activation=s["act"], last=True, carry=train)
        if not train:
            return h, last
        grads = ops.gated_scan_backward(s["dh"], s["gate"], s["cand"], carry, s["offsets"], h0=s["h0"], dlast=s["dlast"],
                                        activation=s["act"])
        if s["dh"].dtype == torch.float32:
            # the plain form adds dlast to dh in place where dh is in 32 bits: a pass leaves the same behind, so that further
            # passes over one state have the same inputs in both
            begin, end = s["offsets"][:-1], s["offsets"][1:]
            s["dh"].index_add_(0, (end - 1).clamp_(min=0), s["dlast"] * (end > begin)[:, None])
        return (h, last) + grads
    loss, grad = ops.distill_loss(s["logits"], s["teacher"], s["index"], s["temperature"], s["weight"], grad=s["mode"] == "train")
    return loss if grad is None else (loss, grad)


def run(s):
    if own:
        return _run_own(s)
    return {"norm": _norm_plain, "scan": _scan_plain, "distill": _distill_plain}[s["op"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def _tokens(c):
    """Rows of all sequences together."""
    return max(1, c["sequences"] * (c["min_len"] + c["max_len"]) // 2)


def work(c):
    e = BYTES[c["dtype"]]
    if c["op"] == "norm":
        n = c["rows"] * c["cols"]
        if c["mode"] == "forward":
            return {"bytes": 2 * n * e + 8 * c["cols"], "flops": 8 * n}
        return {"bytes": 4 * n * e + 16 * c["cols"], "flops": 20 * n}
    if c["op"] == "scan":
        n, state = _tokens(c) * c["hidden"], c["sequences"] * c["hidden"] * 4
        if c["mode"] != "train":
            return {"bytes": 3 * n * e + 2 * state, "flops": 10 * n}
        return {"bytes": 6 * n * e + 4 * state, "flops": 30 * n}
    n = c["rows"] * c["vocab"]
    small = c["rows"] * c["top"] * 12 + 8 * c["rows"]
    if c["mode"] == "forward":
        return {"bytes": n * e + small, "flops": 4 * n}
    return {"bytes": 2 * n * e + small, "flops": 8 * n}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _norm_exact(s):
    x, w = s["x"].double(), s["weight"].double()
    cols = x.shape[1]
    mean = x.sum(1) / cols
    var = (x * x).sum(1) / cols - mean * mean
    std = torch.sqrt(var + EPS)
    n = (x - mean[:, None]) / std[:, None]
    y = n * w + s["bias"].double()
    if s["mode"] == "forward":
        return y
    dy = s["dy"].double()
    # the derivative of n by x, term by term: through x itself, the mean and the variance
    dn = dy * w
    dvar = -0.5 * (dn * n).sum(1) / (var + EPS)
    dmean = -dn.sum(1) / std
    dx = dn / std[:, None] + dmean[:, None] / cols + dvar[:, None] * 2.0 * (x - mean[:, None]) / cols
    return y, dx, (dy * n).sum(0), dy.sum(0)


def _scan_exact(s):
    gate, cand, h0 = s["gate"].double(), s["cand"].double(), s["h0"].double()
    z = 1.0 / (1.0 + torch.exp(-gate))
    keep = 1.0 / (1.0 + torch.exp(gate))
    v = torch.tanh(cand) if s["act"] == "tanh" else cand
    if s["mode"] == "step":
        out = keep * h0 + z * v
        return out, out
    # all sequences side by side, one time step after the other, the longest sequences first
    begin = s["offsets"][:-1].cpu()
    length = s["offsets"][1:].cpu() - begin
    order = torch.argsort(length, descending=True)
    longest = int(length.max())
    if longest > 70000:
        return None
    begin, length = begin[order], length[order]
    live = [int(n) for n in (torch.bincount(length, minlength=longest + 1).flip(0).cumsum(0).flip(0))[1:]]
    begin, order = begin.to(gate.device), order.to(gate.device)
    state = h0[order].clone()
    h = torch.empty_like(gate)
    train = s["mode"] == "train"
    before = torch.empty_like(gate) if train else None
    for k in range(longest):
        n = live[k]
        row = begin[:n] + k
        if train:
            before[row] = state[:n]
        state[:n] = keep[row] * state[:n] + z[row] * v[row]
        h[row] = state[:n]
    last = torch.empty_like(h0)
    last[order] = state
    if not train:
        return h, last
    dh = s["dh"].double()
    back = s["dlast"].double()[order].clone()
    dgate, dcand = torch.empty_like(gate), torch.empty_like(gate)
    for k in reversed(range(longest)):
        n = live[k]
        row = begin[:n] + k
        g = dh[row] + back[:n]
        dgate[row] = g * (v[row] - before[row]) * z[row] * keep[row]
        dcand[row] = g * z[row] * ((1.0 - v[row] ** 2) if s["act"] == "tanh" else 1.0)
        back[:n] = g * keep[row]
    dh0 = torch.empty_like(h0)
    dh0[order] = back
    return h, last, dgate, dcand, dh0


def _distill_exact(s):
    x, y, temp = s["logits"].double() / s["temperature"], s["teacher"].double() / s["temperature"], s["temperature"]
    log_q = torch.log_softmax(x, 1)
    log_p = torch.log_softmax(y, 1)
    p = torch.exp(log_p)
    loss = s["weight"].double() * temp ** 2 * (p * (log_p - log_q.gather(1, s["index"]))).sum(1)
    if s["mode"] == "forward":
        return loss
    target = torch.zeros_like(log_q).scatter_add_(1, s["index"], p)
    return loss, s["weight"].double()[:, None] * temp * (torch.exp(log_q) - target)


def exact(c, seed):
    s = prepare(c, seed)
    return {"norm": _norm_exact, "scan": _scan_exact, "distill": _distill_exact}[s["op"]](s)
