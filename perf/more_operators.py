"""Operators of a recurrent model with matrix states that is trained by rewards, as cases to measure: the gated delta rule, the clipped
policy loss and the global gradient norm with clipping.

Each case is a dict of plain values: the operator, its direction, type and sizes.  prepare() makes the inputs that a user's
program holds before the call; run() makes one pass, in plain torch operations, or, with `own` set, through
paper_1705_09786_amd.operators; exact() gives the same outputs in 64 bits from the operators' definitions.

  delta rule   per head, with a state S of dk x dv:  S <- exp(decay_t) S,  e_t = v_t - S^T k_t,  S <- S + beta_t k_t e_t^T,
               o_t = S^T q_t / sqrt(dk); packed sequences, S before the first row = h0; key heads may be shared by several heads
  policy loss  w (-min(r A, clip(r) A) + kl (e^d - d - 1)), r = exp(lp - old), d = reference - lp, lp = log softmax(logits / T)[index]
  clipping     norm = sqrt of the sum of all squares over many tensors, out = gradient * min(1, max_norm / norm)
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 64


def _delta(name, **kw):
    return dict(dict(name=name, op="delta", mode="train", dtype="bf16", heads=16, key_heads=16, dk=128, dv=128, sequences=8, min_len=1,
                     max_len=2048), **kw)


def _policy(name, **kw):
    return dict(dict(name=name, op="policy", mode="train", dtype="bf16", rows=4096, vocab=32000, temperature=1.0, kl=0.05), **kw)


def _clip(name, **kw):
    return dict(dict(name=name, op="clip", mode="clip", dtype="bf16", tensors=400, smallest=1024, largest=4194304, max_norm=1.0), **kw)


def listed():
    return [
        # serving: one new token for each of 48 sequences, whose states are kept between the calls
        _delta("delta_step", mode="step", sequences=48, min_len=1, max_len=1),
        # serving one user with a small model
        _delta("delta_step_one", mode="step", dtype="f16", heads=4, key_heads=4, dk=64, dv=64, sequences=1, min_len=1, max_len=1),
        # reading one long document: parallel over time or bound by its length
        _delta("delta_long_document", mode="forward", sequences=1, min_len=32768, max_len=32768),
        # the benchmark's recurrent workload as one array: sequences of 4 .. 32 tokens, scored forward only, in 32 bits
        _delta("delta_short_sequences", mode="forward", dtype="f32", heads=4, key_heads=4, dk=32, dv=32, sequences=1000, min_len=4, max_len=32),
        # a training step on packed documents of very different lengths, two heads to a key
        _delta("delta_train", key_heads=8, sequences=24, min_len=16, max_len=1350),
        # the same at sizes that are no multiple of anything, in 32 bits: three heads over a hidden size of 150
        _delta("delta_train_odd", dtype="f32", heads=3, key_heads=3, dk=50, dv=75, sequences=100, min_len=1, max_len=300),
        # the last few tokens of a batch, over the trees' vocabulary
        _policy("policy_few_rows", dtype="f32", rows=4, vocab=20000),
        # a training step's loss and gradient
        _policy("policy_train", rows=8192),
        # the log-probabilities of sampled tokens, as they are kept for the ratio, over a large and odd vocabulary
        _policy("policy_logprob_large", mode="logprob", dtype="f16", rows=2048, vocab=151111, temperature=0.7),
        # the parameters of a small tree model in 32 bits
        _clip("clip_small_model", dtype="f32", tensors=24, smallest=150, largest=90000),
        # a large model's gradients, many small ones among them
        _clip("clip_large_model", tensors=600),
        # the norm alone, as it is watched during training
        _clip("clip_norm_only", mode="norm", dtype="f32", tensors=97, smallest=999999, largest=7777777),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("delta", "delta", "delta", "policy", "clip"))
    dtype = rng.choice(("f32", "bf16", "bf16", "f16"))
    if op == "delta":
        key_heads, group = _log_int(rng, 1, 16), rng.choice((1, 1, 2, 4))
        dk, dv = _log_int(rng, 16, 128), _log_int(rng, 16, 192)
        heads = key_heads * group
        shape = dict(op=op, dtype=dtype, heads=heads, key_heads=key_heads, dk=dk, dv=dv)
        mode = rng.choice(("train", "train", "forward", "step"))
        if mode == "step":
            most = max(1, 48 * 16 * 128 * 128 // (heads * dk * dv))
            return dict(shape, mode=mode, sequences=_log_int(rng, 1, min(1024, most)), min_len=1, max_len=1)
        most = (16384 if mode == "train" else 32768) * 16 * 128 * 128 // (heads * dk * dv)
        tokens = _log_int(rng, 16, min(16384 if mode == "train" else 32768, most))
        sequences = _log_int(rng, 1, max(1, min(1000, tokens, 67_000_000 // (heads * dk * dv))))
        longest = max(1, 2 * tokens // sequences - 1)
        return dict(shape, mode=mode, sequences=sequences, min_len=rng.choice((0, 1)) if sequences >= 8 else 1, max_len=longest)
    if op == "policy":
        vocab = _log_int(rng, 1000, 160000)
        rows = _log_int(rng, 1, min(16384, 250_000_000 // vocab))
        return dict(op=op, mode=rng.choice(("train", "train", "logprob")), dtype=dtype, rows=rows, vocab=vocab,
                    temperature=rng.choice((1.0, 0.7, 1.3)), kl=rng.choice((0.0, 0.05, 0.2)))
    tensors = _log_int(rng, 1, 800)
    largest = _log_int(rng, 10, min(16_000_000, 250_000_000 // tensors))
    return dict(op=op, mode=rng.choice(("clip", "norm")), dtype=dtype, tensors=tensors, smallest=_log_int(rng, 1, largest), largest=largest,
                max_norm=rng.choice((0.5, 1.0, 1e6)))


def _lengths(c, gen):
    """Lengths of the packed sequences, from the seed, their sum the same for every seed; 0 is a length."""
    got = torch.randint(c["min_len"], c["max_len"] + 1, (c["sequences"],), generator=gen).tolist()
    over = sum(got) - _tokens(c)
    for k, n in enumerate(got):
        got[k] = max(c["min_len"], min(c["max_len"], n - over))
        over -= n - got[k]
    return got


def _sizes(c):
    """The tensors' sizes, between the smallest and the largest, spread over their logarithm, in no order."""
    ratio = math.log(c["largest"] / c["smallest"])
    return [int(c["smallest"] * math.exp(ratio * ((k * 0.6180339887498949) % 1.0))) for k in range(c["tensors"])]


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

    if c["op"] == "delta":
        n, heads, key_heads, dk, dv = c["sequences"], c["heads"], c["key_heads"], c["dk"], c["dv"]
        lengths = _lengths(c, host)
        total = sum(lengths)
        offsets = torch.zeros(n + 1, dtype=torch.int64)
        offsets[1:] = torch.cumsum(torch.tensor(lengths), 0)
        s["lengths"], s["offsets"] = lengths, offsets.to(dev)
        # keys and queries of length one that share a direction, as a layer's do
        for name in ("q", "k"):
            x = normal(total, key_heads, dk) + 0.5 * normal(key_heads, dk)
            s[name] = (x / (x * x).sum(2, keepdim=True).sqrt()).to(t).reshape(total, key_heads * dk)
        s["v"] = normal(total, heads * dv).to(t)
        # heads that remember from some tokens to some thousands of them
        reach = torch.exp(-7.0 * torch.rand(heads, generator=gen, device=dev))
        s["decay"] = -reach * torch.log1p(torch.exp(normal(total, heads)))
        s["beta"] = torch.sigmoid(normal(total, heads))
        s["h0"] = 0.1 * normal(n, heads, dk, dv)
        if c["mode"] == "train":
            s["do"] = (0.1 * normal(total, heads * dv)).to(t)
            s["dlast"] = 0.1 * normal(n, heads, dk, dv)
    elif c["op"] == "policy":
        rows, vocab = c["rows"], c["vocab"]
        s["index"] = torch.randint(0, vocab, (rows,), generator=gen, device=dev)
        # the tokens taken are likely ones
        logits = 1.5 * normal(rows, vocab)
        logits.scatter_add_(1, s["index"][:, None], 3.0 * normal(rows, 1) + 8.0)
        s["logits"] = logits.to(t)
        if c["mode"] == "train":
            x = s["logits"].float() / c["temperature"]
            lp = x.gather(1, s["index"][:, None])[:, 0] - torch.logsumexp(x, 1)
            # a policy some updates away from the one that drew the tokens, and from the reference
            s["old"] = lp + 0.2 * normal(rows)
            s["reference"] = lp + 0.3 * normal(rows)
            s["advantage"] = normal(rows)
            s["weight"] = (torch.rand(rows, generator=gen, device=dev) < 0.9) / float(rows)
    else:
        # layers whose gradients are of very different sizes
        scale = torch.exp(1.5 * torch.randn(c["tensors"], generator=host)).tolist()
        s["grads"] = [(0.01 * f * normal(n)).to(t) for n, f in zip(_sizes(c), scale)]
        if c["mode"] == "clip":
            # the optimizer's buffer, the tensors one behind the other
            s["flat"] = torch.empty(sum(_sizes(c)), dtype=t, device=dev)
            s["out"] = list(s["flat"].split(_sizes(c)))
    return s


# ------------------------------------------------------------------ plain forms, in 32 bits
def _chunks(lengths, dev):
    """The rows of every chunk (chunks, CHUNK), -1 where a sequence has ended, and for each position along the sequences the chunks
    and the sequences there."""
    rows, steps, first = [], [], 0
    for q, n in enumerate(lengths):
        for j, at in enumerate(range(0, n, CHUNK)):
            if j == len(steps):
                steps.append(([], []))
            steps[j][0].append(len(rows))
            steps[j][1].append(q)
            rows.append((first + at, min(CHUNK, n - at)))
        first += n
    table = torch.tensor(rows, device=dev).reshape(-1, 2)
    lane = torch.arange(CHUNK, device=dev)
    index = torch.where(lane < table[:, 1:], table[:, :1] + lane, -1)
    return index, [(torch.tensor(a, device=dev), torch.tensor(b, device=dev)) for a, b in steps]


def _take(x, index, heads, group):
    """Rows of an array as (chunks, heads, CHUNK, features), zeros where there are none."""
    got = x.float()[index.clamp(min=0)] * (index >= 0)[..., None]
    got = got.reshape(index.shape[0], CHUNK, heads, -1).transpose(1, 2)
    return got.repeat_interleave(group, 1).contiguous()


def _put(x, index, rows, group):
    """The other way, the heads of a group added up."""
    n, heads, _, width = x.shape
    x = x.reshape(n, heads // group, group, CHUNK, width).sum(2).transpose(1, 2).reshape(n, CHUNK, -1)
    out = torch.zeros(rows, x.shape[2], device=x.device)
    keep = index >= 0
    out[index[keep]] = x[keep]
    return out


def _turn(x):
    return x.transpose(-1, -2).contiguous()


def _delta_plain(s):
    t, heads, dk, dv = s["q"].dtype, s["heads"], s["dk"], s["dv"]
    group, scale = heads // s["key_heads"], dk ** -0.5
    if s["mode"] == "step":
        n = s["q"].shape[0]
        q, k = (s[x].float().reshape(n, -1, dk).repeat_interleave(group, 1)[..., None] for x in ("q", "k"))
        state = s["h0"] * torch.exp(s["decay"])[..., None, None]
        e = s["v"].float().reshape(n, heads, 1, dv) - (k * state).sum(2, keepdim=True)
        s["h0"].copy_(state + s["beta"][..., None, None] * k * e)
        return (scale * (q * s["h0"]).sum(2)).to(t).reshape(n, -1), s["h0"]
    index, steps = _chunks(s["lengths"], s["q"].device)
    rows = s["q"].shape[0]
    Q, K = (_take(s[x], index, s["key_heads"], group) for x in ("q", "k"))
    V = _take(s["v"], index, heads, 1)
    beta = _take(s["beta"], index, heads, 1)
    G = torch.cumsum(_take(s["decay"], index, heads, 1), 2)
    lane = torch.arange(CHUNK, device=Q.device)
    below, upto = lane[:, None] > lane, lane[:, None] >= lane
    D = torch.exp(torch.where(upto, G - G.transpose(-1, -2), torch.zeros((), device=Q.device)))
    KT = _turn(K)
    M = torch.where(below, D * (K @ KT), torch.zeros((), device=Q.device))
    P = torch.where(upto, scale * D * (Q @ KT), torch.zeros((), device=Q.device))
    # the inverse of 1 + M diag(beta), row after row
    A = M * beta.transpose(-1, -2)
    inverse = torch.eye(CHUNK, device=Q.device).expand_as(A).contiguous()
    for i in range(1, CHUNK):
        inverse[:, :, i, :i] -= (A[:, :, i:i + 1, :i] @ inverse[:, :, :i, :i])[:, :, 0]
    grow, end = torch.exp(G), G[:, :, -1:, :]
    rest, whole = torch.exp(end - G), torch.exp(end)
    O, E = torch.empty_like(V), torch.empty_like(V)
    before = torch.empty(index.shape[0], heads, dk, dv, device=Q.device)
    state = s["h0"].clone()
    KR = _turn(rest * K)
    for c, seq in steps:
        S = state[seq]
        before[c] = S
        e = inverse[c] @ (V[c] - grow[c] * (K[c] @ S))
        E[c] = e
        O[c] = scale * grow[c] * (Q[c] @ S) + P[c] @ (beta[c] * e)
        state[seq] = whole[c] * S + KR[c] @ (beta[c] * e)
    o = _put(O, index, rows, 1).to(t)
    if s["mode"] == "forward":
        return o, state
    dO = _take(s["do"], index, heads, 1)
    # 1 - diag(beta) N is the inverse of 1 + diag(beta) M, where 1 - N diag(beta) is the one above
    other = torch.eye(CHUNK, device=Q.device) - beta * (inverse @ M)
    part, other = _turn(P) @ dO, _turn(other)
    behind, X = torch.empty_like(before), torch.empty_like(V)
    dstate = s["dlast"].clone()
    QT, KG = _turn(scale * grow * Q), _turn(grow * K)
    for c, seq in reversed(steps):
        dS = dstate[seq]
        behind[c] = dS
        x = other[c] @ (part[c] + rest[c] * (K[c] @ dS))
        X[c] = x
        dstate[seq] = whole[c] * dS + QT[c] @ dO[c] - KG[c] @ (beta[c] * x)
    Y, W = beta * X, beta * E
    WT = _turn(W)
    dP = torch.where(upto, scale * D * (dO @ WT), torch.zeros((), device=Q.device))
    dM = torch.where(below, -D * (Y @ WT), torch.zeros((), device=Q.device))
    ST = _turn(before)
    dQ = scale * grow * (dO @ ST) + dP @ K
    row = dM @ K - grow * (Y @ ST)
    last = rest * (W @ _turn(behind))
    col = _turn(dP) @ Q + _turn(dM) @ K + last
    dG = (Q * dQ + K * row - K * col).sum(3, keepdim=True)
    dG[:, :, -1:] += (K * last).sum((2, 3), keepdim=True) + whole * (before * behind).sum((2, 3), keepdim=True)
    ddecay = dG.flip(2).cumsum(2).flip(2)
    return (o, state, _put(dQ, index, rows, group).to(t), _put(row + col, index, rows, group).to(t), _put(Y, index, rows, 1).to(t),
            _put(ddecay, index, rows, 1), _put((X * E).sum(3, keepdim=True), index, rows, 1), dstate)


def _policy_plain(s):
    t, temp, rows = s["logits"].dtype, s["temperature"], s["logits"].shape[0]
    x = s["logits"].float() / temp
    x = x - x.max(1, keepdim=True).values
    e = torch.exp(x)
    # 64 bits for the sums and what follows: a ratio next to its limit decides whether a row has a gradient
    norm = e.sum(1, keepdim=True, dtype=torch.float64)
    lp = x.gather(1, s["index"][:, None]).double()[:, 0] - torch.log(norm[:, 0])
    if s["mode"] == "logprob":
        return lp.float()
    a, w, kl = s["advantage"].double(), s["weight"].double(), s["kl"]
    r = torch.exp(lp - s["old"])
    d = s["reference"] - lp
    near = torch.exp(d)
    loss = w * (-torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + kl * (near - d - 1.0))
    inside = torch.where(a >= 0, r <= 1.2, r >= 0.8)
    g = w / temp * (kl * (1.0 - near) - inside * r * a)
    grad = -(e / norm.float()) * g.float()[:, None]
    grad.scatter_add_(1, s["index"][:, None], g.float()[:, None])
    return loss.float(), lp.float(), grad.to(t)


def _clip_plain(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for g in s["grads"]:
        x = g.float()
        total += (x * x).sum(dtype=torch.float64)
    norm = torch.sqrt(total)
    if s["mode"] == "norm":
        return norm.float()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * factor)
    return norm.float(), s["flat"]


# ------------------------------------------------------------------ the framework's calls
def _run_own(s):
    from paper_1705_09786_amd import operators as ops
    if s["op"] == "delta":
        args = [s[x] for x in ("q", "k", "v", "decay", "beta")]
        if s["mode"] == "step":
            return ops.gated_delta_step(*args, s["h0"], key_heads=s["key_heads"]), s["h0"]
        train = s["mode"] == "train"
        o, last, carry = ops.gated_delta(*args, s["offsets"], key_heads=s["key_heads"], h0=s["h0"], last=True, carry=train)
        if not train:
            return o, last
        return (o, last) + ops.gated_delta_backward(s["do"], *args, carry, s["offsets"], key_heads=s["key_heads"], dlast=s["dlast"])
    if s["op"] == "policy":
        if s["mode"] == "logprob":
            return ops.token_logprob(s["logits"], s["index"], s["temperature"])
        return ops.policy_loss(s["logits"], s["index"], s["old"], s["advantage"], reference=s["reference"], kl=s["kl"], clip=0.2,
                               temperature=s["temperature"], weight=s["weight"])
    if s["mode"] == "norm":
        return ops.clip_gradients(s["grads"])
    return ops.clip_gradients(s["grads"], s["max_norm"], out=s["out"]), s["flat"]


def run(s):
    if own:
        return _run_own(s)
    return {"delta": _delta_plain, "policy": _policy_plain, "clip": _clip_plain}[s["op"]](s)


# ------------------------------------------------------------------ what a pass cannot do without
def _tokens(c):
    """Rows of all sequences together."""
    return max(1, c["sequences"] * (c["min_len"] + c["max_len"]) // 2)


def work(c):
    e = BYTES[c["dtype"]]
    if c["op"] == "delta":
        n, heads, dk, dv = _tokens(c), c["heads"], c["dk"], c["dv"]
        keys, values, state = n * c["key_heads"] * dk * e, n * heads * dv * e, c["sequences"] * heads * dk * dv * 4
        forward = {"bytes": 2 * keys + 2 * values + 8 * n * heads + 2 * state, "flops": 7 * n * heads * dk * dv}
        if c["mode"] != "train":
            return forward
        # q, k, v, do and the gates once, o and the five gradients; the states in front and behind, and their gradients
        return {"bytes": 4 * keys + 4 * values + 16 * n * heads + 4 * state, "flops": 27 * n * heads * dk * dv}
    if c["op"] == "policy":
        n = c["rows"] * c["vocab"]
        if c["mode"] == "logprob":
            return {"bytes": n * e + 12 * c["rows"], "flops": 4 * n}
        return {"bytes": 2 * n * e + 32 * c["rows"], "flops": 8 * n}
    n = sum(_sizes(c))
    return {"bytes": n * e, "flops": 2 * n} if c["mode"] == "norm" else {"bytes": 2 * n * e, "flops": 3 * n}


# ------------------------------------------------------------------ 64 bits, from the definitions
def _delta_exact(s):
    heads, dk, dv = s["heads"], s["dk"], s["dv"]
    group, rows, n = heads // s["key_heads"], s["q"].shape[0], s["sequences"]
    q, k = (s[x].double().reshape(rows, -1, dk).repeat_interleave(group, 1) for x in ("q", "k"))
    q = q / math.sqrt(dk)
    v = s["v"].double().reshape(rows, heads, dv)
    a, beta = torch.exp(s["decay"].double()), s["beta"].double()
    dev = q.device

    def forward(S, row):
        """One token of every live sequence: the decayed state, the error and the new state."""
        S = a[row][..., None, None] * S
        e = v[row] - (k[row][..., None] * S).sum(2)
        return S, e, S + (beta[row][..., None] * k[row])[..., None] * e[:, :, None]

    if s["mode"] == "step":
        S = forward(s["h0"].double(), torch.arange(rows, device=dev))[2]
        return (q[..., None] * S).sum(2).reshape(rows, -1), S
    # all sequences side by side, one token after the other, the longest sequences first
    length = torch.tensor(s["lengths"])
    begin = torch.cumsum(length, 0) - length
    order = torch.argsort(length, descending=True)
    longest = int(length.max())
    if longest > 40000:
        return None
    live = [int(m) for m in (torch.bincount(length, minlength=longest + 1).flip(0).cumsum(0).flip(0))[1:]]
    begin, order = begin[order].to(dev), order.to(dev)
    train = s["mode"] == "train"
    # a backward pass has some tokens' states in memory and forms the others again from every block's first
    block = max(1, min(64, 3_000_000_000 // (n * heads * dk * dv * 8)))
    state = s["h0"].double()[order]
    kept = []
    o = torch.empty(rows, heads, dv, dtype=torch.float64, device=dev)
    for t in range(longest):
        m = live[t]
        row = begin[:m] + t
        if train and t % block == 0:
            kept.append(state[:m].clone())
        state[:m] = forward(state[:m], row)[2]
        o[row] = (q[row][..., None] * state[:m]).sum(2)
    last = torch.empty_like(state)
    last[order] = state
    o = o.reshape(rows, -1)
    if not train:
        return o, last
    do = s["do"].double().reshape(rows, heads, dv)
    dstate = s["dlast"].double()[order]
    dq, dk_, dv_ = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    da, dbeta = torch.empty_like(a), torch.empty_like(beta)
    for t0 in reversed(range(0, longest, block)):
        S, seen = kept.pop(), []
        for t in range(t0, min(longest, t0 + block)):
            S = S[:live[t]]
            decayed, e, after = forward(S, begin[:live[t]] + t)
            seen.append((S, decayed, e, after))
            S = after
        for t in reversed(range(t0, min(longest, t0 + block))):
            old, decayed, e, after = seen.pop()
            m = live[t]
            row = begin[:m] + t
            key, b = k[row], beta[row][..., None]
            dS = dstate[:m] + q[row][..., None] * do[row][:, :, None]
            dq[row] = (after * do[row][:, :, None]).sum(3)
            kd = (key[..., None] * dS).sum(2)                  # the gradient of beta e
            dbeta[row] = (kd * e).sum(2)
            de = b * kd
            dv_[row] = de
            dk_[row] = b * (dS * e[:, :, None]).sum(3) - (decayed * de[:, :, None]).sum(3)
            dS = dS - key[..., None] * de[:, :, None]
            da[row] = (dS * old).sum((2, 3))
            dstate[:m] = a[row][..., None, None] * dS
    dh0 = torch.empty_like(dstate)
    dh0[order] = dstate
    shared = (rows, s["key_heads"], group, dk)
    dq = (dq / math.sqrt(dk)).reshape(shared).sum(2).reshape(rows, -1)
    return o, last, dq, dk_.reshape(shared).sum(2).reshape(rows, -1), dv_.reshape(rows, -1), da * a, dbeta, dh0


def _policy_exact(s):
    index = s["index"][:, None]
    log_q = torch.log_softmax(s["logits"].double() / s["temperature"], 1)
    lp = log_q.gather(1, index)[:, 0]
    if s["mode"] == "logprob":
        return lp
    a, w, kl = s["advantage"].double(), s["weight"].double(), s["kl"]
    ratio, d = torch.exp(lp - s["old"].double()), s["reference"].double() - lp
    # a row gains up to the limit on the side that its advantage asks for
    gain = torch.where(a >= 0, a * ratio.clamp(max=1.2), a * ratio.clamp(min=0.8))
    loss = w * (kl * (torch.expm1(d) - d) - gain)
    free = torch.where(a >= 0, ratio <= 1.2, ratio >= 0.8).double()
    by_lp = -w * (kl * torch.expm1(d) + free * a * ratio)
    grad = -torch.exp(log_q)
    grad.scatter_add_(1, index, torch.ones_like(lp)[:, None])
    return loss, lp, grad.mul_((by_lp / s["temperature"])[:, None])


def _clip_exact(s):
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g.double()) for g in s["grads"]]))
    if s["mode"] == "norm":
        return norm
    return norm, torch.cat([g.double() * (s["max_norm"] / norm if norm > s["max_norm"] else 1.0) for g in s["grads"]])


def exact(c, seed):
    s = prepare(c, seed)
    return {"delta": _delta_exact, "policy": _policy_exact, "clip": _clip_exact}[s["op"]](s)
