"""The operators on whole arrays in 64 bits on the CPU, from their formulas, with bounds for what 32-bit arithmetic may add.

Every reference returns (value, bound): `bound` is what a kernel that computes in 32 bits may be off by before the result is rounded,
in units of 2^-24 (half a step of binary32, the error of one operation relative to its result), formed beside the value from the sizes
of the terms that meet: `allowed` turns both into a tolerance for a result of a type."""
import math

import torch

U = 2.0 ** -24


def allowed(value, bound, dtype):
    """Half a step of the result's type, the steps of its smallest numbers, and the arithmetic in front of it."""
    info = torch.finfo(dtype)
    return value.abs() * (info.eps / 2) + info.tiny * info.eps + U * bound * 1.01


def check(name, got, ref, dtype=None):
    value, bound = ref
    dtype = got.dtype if dtype is None else dtype
    got = got.detach().cpu().double()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    tol = allowed(value, bound, dtype)
    big = value.abs() > torch.finfo(dtype).max   # a result beyond the type is its infinity
    diff = torch.where(big, torch.zeros_like(value), (got - value).abs())
    bad = ~(diff <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of what is allowed, first at %s: %.9g for %.9g" % (
        name, int(bad.sum()), bad.numel(), float((diff / tol)[bad].max()), bad.nonzero()[0].tolist(), float(got[bad][0]), float(value[bad][0]))


# ------------------------------------------------------------------ layer norm
def _serial(cols):
    """Additions one behind the other in a row's sum: a lane's own, then the joins over lanes and waves."""
    return math.ceil(cols / 64) + 16


def norm(x, w, b, eps):
    """y, mean, rstd."""
    x = x.double()
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(x.shape[1], dtype=torch.float64) if b is None else b.double()
    n = _serial(x.shape[1])
    mean = x.mean(1, keepdim=True)
    e_mean = n * x.abs().mean(1, keepdim=True)
    d = x - mean
    e_d = e_mean + d.abs()
    var = (d * d).mean(1, keepdim=True) + eps
    e_var = 2 * (d.abs() * e_d).mean(1, keepdim=True) + (n + 2) * var
    rstd = var ** -0.5
    e_rstd = rstd * (0.5 * e_var / var + 4)
    y = d * rstd * w + b
    e_y = (e_d * rstd + d.abs() * e_rstd + 2 * d.abs() * rstd) * w.abs() + y.abs() + b.abs()
    return (y, e_y), (mean[:, 0], e_mean[:, 0]), (rstd[:, 0], e_rstd[:, 0])


def norm_backward(dy, x, w, mean, rstd):
    """dx, dw, db for the statistics that the call is given."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    cols, rows = x.shape[1], x.shape[0]
    w = torch.ones(cols, dtype=torch.float64) if w is None else w.double()
    n = (x - mean) * rstd
    e_n = 3 * n.abs()
    q = dy * w
    steps = _serial(cols)
    m0, m1 = q.mean(1, keepdim=True), (q * n).mean(1, keepdim=True)
    e_m0 = (steps + 2) * q.abs().mean(1, keepdim=True)
    e_m1 = (steps + 6) * (q * n).abs().mean(1, keepdim=True)
    dx = rstd * (q - m0 - n * m1)
    e_dx = rstd * (2 * q.abs() + e_m0 + n.abs() * e_m1 + e_n * m1.abs() + 4 * (q.abs() + m0.abs() + (n * m1).abs()))
    # rows one behind the other in a part, then the parts
    down = rows + 64
    return (dx, e_dx), ((dy * n).sum(0), (down + 5) * (dy * n).abs().sum(0)), (dy.sum(0), down * dy.abs().sum(0))


# ------------------------------------------------------------------ gated linear recurrence
def spans(sequences, rows):
    """[(begin, end)] of None, offsets or a pair."""
    if sequences is None:
        return [(0, rows)]
    if isinstance(sequences, (tuple, list)):
        return list(zip(sequences[0].tolist(), sequences[1].tolist()))
    o = sequences.tolist()
    return list(zip(o[:-1], o[1:]))


def _gates(gate, cand, tanh):
    g = gate.double()
    z, keep = torch.sigmoid(g), torch.sigmoid(-g)
    v = torch.tanh(cand.double()) if tanh else cand.double()
    # e^-|g|: its argument's rounding, |g| log2(e) ln(2) units, and its own last place; sum, estimate and product one or two each
    return z, keep, v, 8 + 2 * g.abs().clamp(max=128)


def scan(gate, cand, sequences, h0, tanh):
    """h (0 in rows of no sequence), last, and the pieces that the backward pass needs."""
    z, keep, v, c = _gates(gate, cand, tanh)
    rows, hidden = gate.shape
    lens = spans(sequences, rows)
    h, e = torch.zeros(rows, hidden, dtype=torch.float64), torch.zeros(rows, hidden, dtype=torch.float64)
    before, e_before = h.clone(), h.clone()
    last, e_last = (torch.zeros(len(lens), hidden, dtype=torch.float64) for _ in range(2))
    for s, (b, n) in enumerate(lens):
        x = torch.zeros(hidden, dtype=torch.float64) if h0 is None else h0[s].double()
        size, err = x.abs(), torch.zeros(hidden, dtype=torch.float64)
        for t in range(b, n):
            before[t], e_before[t] = x, err + 40 * size
            x = keep[t] * x + z[t] * v[t]
            size = keep[t] * size + z[t] * v[t].abs()
            err = keep[t] * err + c[t] * size
            # the maps of up to 40 groups of rows meet between a row and its state, one rounding each
            h[t], e[t] = x, err + 40 * size
        last[s], e_last[s] = x, err + 40 * size
        if n <= b:
            e_last[s] = 0
    return (h, e), (last, e_last), (before, e_before)


def scan_backward(dh, dlast, gate, cand, sequences, h0, tanh):
    """dgate, dcand (0 in rows of no sequence), dh0."""
    z, keep, v, c = _gates(gate, cand, tanh)
    rows, hidden = gate.shape
    lens = spans(sequences, rows)
    (before, e_before) = scan(gate, cand, sequences, h0, tanh)[2]
    zero = torch.zeros(rows, hidden, dtype=torch.float64)
    G, e_G, size = zero.clone(), zero.clone(), zero.clone()
    dh0, e_dh0 = (torch.zeros(len(lens), hidden, dtype=torch.float64) for _ in range(2))
    for s, (b, n) in enumerate(lens):
        x = torch.zeros(hidden, dtype=torch.float64) if dlast is None else dlast[s].double()
        big, err = x.abs(), torch.zeros(hidden, dtype=torch.float64)
        for t in range(n - 1, b - 1, -1):
            G[t] = dh[t].double() + x
            size[t] = dh[t].double().abs() + big
            e_G[t] = err + 40 * size[t]
            x = keep[t] * G[t]
            big = keep[t] * size[t]
            err = keep[t] * err + (c[t] + 2) * big
        dh0[s], e_dh0[s] = x, (err + 40 * big if n > b else 0)
    act = 1 - v * v if tanh else torch.ones_like(v)
    zk, diff, e_v = z * keep, v - before, 4 * v.abs()
    dgate = G * zk * diff
    e_gate = e_G * zk * diff.abs() + G.abs() * zk * (e_before + e_v + diff.abs()) + (2 * c + 4) * dgate.abs()
    dcand = G * z * act
    e_cand = e_G * z * act + G.abs() * z * (2 * v.abs() * e_v + 2 if tanh else 0) + (c + 3) * dcand.abs()
    return (dgate, e_gate), (dcand, e_cand), (dh0, e_dh0)


def step(gate, cand, state, tanh):
    z, keep, v, c = _gates(gate, cand, tanh)
    h = keep * state.double() + z * v
    return h, (c + 6) * (keep * state.double().abs() + z * v.abs())


# ------------------------------------------------------------------ distillation
def distill(logits, teacher, index, temperature, weight):
    """loss, dlogits."""
    x, y, T = logits.double(), teacher.double(), float(temperature)
    rows, classes = x.shape
    w = torch.ones(rows, dtype=torch.float64) if weight is None else weight.double()
    loss, e_loss = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    grad, e_grad = torch.zeros(rows, classes, dtype=torch.float64), torch.zeros(rows, classes, dtype=torch.float64)
    for r in range(rows):
        used = (index[r] >= 0) & (index[r] < classes) & (y[r] != -math.inf)
        if w[r] == 0 or not used.any():
            continue
        cls = index[r][used].long()
        lp, lq = torch.log_softmax(y[r][used] / T, 0), torch.log_softmax(x[r] / T, 0)
        p, q = lp.exp(), lq.exp()
        live = p > 0
        loss[r] = w[r] * T * T * (p[live] * (lp[live] - lq[cls[live]])).sum()
        # a term's exponent is off by the roundings of its difference, its scale and their product (3 units of it), a sum by its additions
        sums = _serial(classes) + 40
        far_p, far_q = -lp + math.log(len(cls)), -lq + math.log(classes)
        e_term = p * (3 * far_p.clamp(max=200) + 3 * far_q[cls] + lp.abs() + lq[cls].abs() + 2 * sums)
        e_loss[r] = w[r].abs() * T * T * (e_term[live].sum() + 8 * (p[live] * (lp[live].abs() + lq[cls[live]].abs())).sum())
        at = torch.zeros(classes, dtype=torch.float64).index_add_(0, cls, p)
        e_at = torch.zeros(classes, dtype=torch.float64).index_add_(0, cls, p * (3 * far_p.clamp(max=200) + len(cls) + sums))
        grad[r] = w[r] * T * (q - at)
        e_grad[r] = w[r].abs() * T * (q * (3 * far_q.clamp(max=200) + sums + 8) + e_at)
        # q below 2^-126 of the largest term may be taken for zero
        e_grad[r] += w[r].abs() * T * 2.0 ** -120
    return (loss, e_loss), (grad, e_grad)
