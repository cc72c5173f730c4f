"""The gated delta rule, the policy loss and clipping in 64 bits on the CPU, from their formulas, with bounds for what 32-bit arithmetic
may add, in units of 2^-24 (as ops_reference has them).

The delta rule's values come from its recurrence, row by row. Its bounds follow the kernels' chunks of 32 rows: what a chunk's own
arithmetic adds is bounded by the sizes of the terms that meet, and an error of the state in front of it goes on as the state itself does,
shrunk by the norm of a row's map a (1 - beta k k^T), a max(1, |1 - beta k.k|). A sum of n products in parts of 8 bits has up to six
partial products of each and a rounding for every addition: 6 n units of the sum of their absolute values."""
import math

import torch

from ops_reference import U, _serial, spans

C, B = 32, 64
F64 = torch.float64
# Parts of an operand below 2^-126, the smallest normal number of bf16 as of binary32, may be taken for zero: a product of a sum then
# lacks up to 2^-126 times its other factor (up to 4 here), six partial products of each of up to 320 terms.
LOST = 2.0 ** -126 / U * 4 * 6 * 320


def _by_heads(x, heads):
    """(rows, heads x features) as (heads, rows, features)."""
    return x.double().reshape(x.shape[0], heads, -1).transpose(0, 1)


def _flat(x):
    return x.transpose(0, 1).reshape(x.shape[1], -1)


def _sum(n):
    """Units of a sum of n products. (A power e^x of a chunk's decays is off by |x| units, its exponent being rounded to 24 bits, and is 0 below x =
    -104: less than this from n = 14 on, the fewest keys that are tested with decays as strong.)"""
    return 6 * n + 24


class _Chunk:
    """A chunk's matrices and their bounds, per head."""

    def __init__(s, q, k, decay, beta, scale):
        dk, n = k.shape[2], k.shape[1]
        s.q, s.k, s.beta = q, k, beta[:, :, None]
        G = torch.cumsum(decay.clamp(min=-1000.0), 1)[:, :, None]
        s.grow, s.rest, s.whole = torch.exp(G), torch.exp(G[:, -1:] - G), torch.exp(G[:, -1:])
        low = torch.ones(n, n).tril().bool()
        D = torch.where(low, torch.exp(torch.where(low, G - G.transpose(1, 2), torch.zeros((), dtype=F64))), torch.zeros((), dtype=F64))
        s.nq, s.nk = q.norm(dim=2, keepdim=True), k.norm(dim=2, keepdim=True)
        pairs_k, pairs_q = s.nk * s.nk.transpose(1, 2), s.nq * s.nk.transpose(1, 2)
        strict = low & ~torch.eye(n).bool()
        M = torch.where(strict, D * (k @ k.transpose(1, 2)), torch.zeros((), dtype=F64))
        e_M = torch.where(strict, D * (_sum(dk) * pairs_k), torch.zeros((), dtype=F64)) + 8 * M.abs()
        s.P = scale * D * (q @ k.transpose(1, 2))
        s.e_P = scale * D * _sum(dk) * pairs_q + 8 * s.P.abs()
        bt = s.beta.transpose(1, 2)
        eye = torch.eye(n, dtype=F64)
        Tb = torch.linalg.inv(eye + M * bt)
        s.N = Tb @ M
        Ta = eye - s.beta * s.N
        s.e_N = Tb.abs() @ e_M @ Ta.abs() + (n + 8) * (Tb.abs() @ ((M * bt).abs() @ s.N.abs() + M.abs()))
        s.rho = torch.exp(decay)[:, :, None] * torch.clamp((1 - s.beta * s.nk ** 2).abs(), min=1.0)


def delta(q, k, v, decay, beta, sequences, key_heads, scale, h0, dtype):
    """o, last, and for the backward pass E, the states in front of every block, with bounds; (value, bound) each."""
    heads = decay.shape[1]
    group, rows = heads // key_heads, q.shape[0]
    q, k = (_by_heads(x, key_heads).repeat_interleave(group, 0) for x in (q, k))
    v, decay, beta = _by_heads(v, heads), decay.double().T, beta.double().T
    dk, dv = q.shape[2], v.shape[2]
    scale = dk ** -0.5 if scale is None else scale
    lens = spans(sequences, rows)
    o, e_o, E, e_E = (torch.zeros(heads, rows, dv, dtype=F64) for _ in range(4))
    last, e_last = (torch.zeros(len(lens), heads, dk, dv, dtype=F64) for _ in range(2))
    fronts = []
    rough = 0.0 if dtype == torch.float32 else 3 * 2.0 ** 9   # o's products in two parts
    for s, (b, n) in enumerate(lens):
        S = torch.zeros(heads, dk, dv, dtype=F64) if h0 is None else h0[s].double().clone()
        e_S = torch.zeros(heads, 1, dv, dtype=F64)
        front = []
        for at in range(b, n, C):
            if (at - b) % B == 0:
                front.append((S.clone(), e_S.clone()))
            r = slice(at, min(n, at + C))
            m = _Chunk(q[:, r], k[:, r], decay[:, r], beta[:, r], scale)
            size = S.norm(dim=1, keepdim=True)
            R = v[:, r].abs() + m.grow * m.nk * size
            e_R = m.grow * m.nk * _sum(dk) * size + 6 * R
            nb = m.N.abs() * m.beta.transpose(1, 2)
            abs_E = R + nb @ R
            own = e_R + nb @ e_R + _sum(C) * (nb @ R) + (m.e_N * m.beta.transpose(1, 2)) @ R
            e_V = m.beta * (own + 2 * abs_E)
            steps = torch.cumprod(m.rho, 1)
            before = torch.cat([torch.ones_like(steps[:, :1]), steps[:, :-1]], 1)
            e_E[:, r] = own + m.nk * torch.exp(decay[:, r])[:, :, None] * before * e_S
            abs_V = m.beta * abs_E
            e_o[:, r] = (scale * m.nq * steps * e_S + scale * m.grow * m.nq * (_sum(dk) + rough) * size + m.P.abs() @ e_V +
                         (_sum(C) + rough) * (m.P.abs() @ abs_V) + m.e_P @ abs_V)
            w = (m.rest * m.nk).transpose(1, 2)
            e_S = steps[:, -1:] * e_S + w @ e_V + _sum(C) * (w @ abs_V) + 4 * m.whole * size
            for t in range(at, min(n, at + C)):
                S = torch.exp(decay[:, t])[:, None, None] * S
                err = v[:, t] - (k[:, t, :, None] * S).sum(1)
                S = S + beta[:, t, None, None] * k[:, t, :, None] * err[:, None]
                E[:, t] = err
                o[:, t] = scale * (q[:, t, :, None] * S).sum(1)
        last[s], e_last[s] = S, e_S.expand(heads, dk, dv) if n > b else 0.0
        fronts.append(front)
    return (_flat(o), _flat(e_o) + LOST), (last, e_last + LOST), (E, e_E + LOST), fronts


def delta_backward(do, q, k, v, decay, beta, sequences, key_heads, scale, h0, dlast, dtype):
    """dq, dk, dv, ddecay, dbeta, dh0."""
    heads = decay.shape[1]
    group, rows = heads // key_heads, q.shape[0]
    (E, e_E), fronts = delta(q, k, v, decay, beta, sequences, key_heads, scale, h0, dtype)[2:]
    q, k = (_by_heads(x, key_heads).repeat_interleave(group, 0) for x in (q, k))
    v, do, decay, beta = _by_heads(v, heads), _by_heads(do, heads), decay.double().T, beta.double().T
    dk, dv = q.shape[2], v.shape[2]
    scale = dk ** -0.5 if scale is None else scale
    lens = spans(sequences, rows)
    X, e_X = (torch.zeros(heads, rows, dv, dtype=F64) for _ in range(2))
    dq, e_dq, dkey, e_dkey = (torch.zeros(heads, rows, dk, dtype=F64) for _ in range(4))
    da, e_da = (torch.zeros(heads, rows, 1, dtype=F64) for _ in range(2))
    dh0, e_dh0 = (torch.zeros(len(lens), heads, dk, dv, dtype=F64) for _ in range(2))
    for s, (b, n) in enumerate(lens):
        states = [torch.zeros(heads, dk, dv, dtype=F64) if h0 is None else h0[s].double()]
        for t in range(b, n):   # the values, row by row: the states in front of every row
            S = torch.exp(decay[:, t])[:, None, None] * states[-1]
            states.append(S + beta[:, t, None, None] * k[:, t, :, None] * E[:, t, None])
        dS = torch.zeros(heads, dk, dv, dtype=F64) if dlast is None else dlast[s].double().clone()
        e_S = torch.zeros(heads, 1, dv, dtype=F64)
        behind = {}
        for at in reversed(range(b, n, C)):
            end = min(n, at + C)
            r = slice(at, end)
            if at == b + (n - 1 - b) // C * C or (at - b) // C % 2:
                behind[(at - b) // B] = (dS.clone(), e_S.clone())
            m = _Chunk(q[:, r], k[:, r], decay[:, r], beta[:, r], scale)
            size, PT = dS.norm(dim=1, keepdim=True), m.P.transpose(1, 2).abs()
            V = m.rest * m.nk * size + PT @ do[:, r].abs()
            e_V = m.rest * m.nk * (_sum(dk) + 6) * size + (_sum(C) + 4) * (PT @ do[:, r].abs()) + m.e_P.transpose(1, 2) @ do[:, r].abs()
            nt = m.N.abs().transpose(1, 2)
            abs_X = V + nt @ (m.beta * V)
            own = e_V + nt @ (m.beta * (e_V + 2 * V)) + _sum(C) * (nt @ (m.beta * V)) + m.e_N.transpose(1, 2) @ (m.beta * V) + abs_X
            after = torch.flip(torch.cumprod(torch.flip(m.rho, [1]), 1), [1])   # of the rows from here on
            later = torch.cat([after[:, 1:], torch.ones_like(after[:, :1])], 1)
            e_X[:, r] = own + m.nk * later * e_S
            w, wq = (m.grow * m.nk).transpose(1, 2), (scale * m.grow * m.nq).transpose(1, 2)
            e_S = (after[:, :1] * e_S + w @ (m.beta * (own + 4 * abs_X)) + _sum(C) * (w @ (m.beta * abs_X)) + (_sum(C) + 8) * (wq @ do[:, r].abs()) +
                   4 * m.whole * size)
            for t in reversed(range(at, end)):
                old, new = states[t - b], states[t - b + 1]
                a = torch.exp(decay[:, t])[:, None, None]
                dS = dS + scale * q[:, t, :, None] * do[:, t, None]
                dq[:, t] = scale * (new * do[:, t, None]).sum(2)
                X[:, t] = (k[:, t, :, None] * dS).sum(1)
                de = beta[:, t, None] * X[:, t]
                dkey[:, t] = beta[:, t, None] * (dS * E[:, t, None]).sum(2) - (a * old * de[:, None]).sum(2)
                dS = dS - k[:, t, :, None] * de[:, None]
                da[:, t, 0] = (dS * a * old).sum((1, 2))
                dS = a * dS
        dh0[s], e_dh0[s] = dS, e_S.expand(heads, dk, dv) if n > b else 0.0
        for j, at in enumerate(range(b, n, B)):   # bounds of what is formed block by block
            r = slice(at, min(n, at + B))
            (S0, e0), (S1, e1) = fronts[s][j], behind[j]
            m = _Chunk(q[:, r], k[:, r], decay[:, r], beta[:, r], scale)
            G = torch.cumsum(decay[:, r].clamp(min=-1000.0), 1)[:, :, None]
            rows_in = G.shape[1]
            low = torch.ones(rows_in, rows_in).tril().bool()
            D = torch.where(low, torch.exp(torch.where(low, G - G.transpose(1, 2), torch.zeros((), dtype=F64))), torch.zeros((), dtype=F64))
            W, Y = m.beta * E[:, r].abs(), m.beta * X[:, r].abs()
            e_W, e_Y = m.beta * (e_E[:, r] + 2 * E[:, r].abs()), m.beta * (e_X[:, r] + 2 * X[:, r].abs())
            d, nv = do[:, r].abs(), _sum(dv)

            def product(x, e_x, y, e_y, terms):
                return x @ y, e_x @ y + x @ e_y + terms * (x @ y)

            zero = torch.zeros_like(d)
            pq, e_pq = product(d, zero, W.transpose(1, 2), e_W.transpose(1, 2), nv + 8)
            pm, e_pm = product(Y, e_Y, W.transpose(1, 2), e_W.transpose(1, 2), nv + 8)
            pq, e_pq, pm, e_pm = scale * D * pq, scale * D * e_pq, D * pm, D * e_pm
            es0, es1 = e0.expand_as(S0).transpose(1, 2), e1.expand_as(S1).transpose(1, 2)
            A0, A1 = S0.abs().transpose(1, 2), S1.abs().transpose(1, 2)
            q1, e_q1 = product(d, zero, A0, es0, nv + 8)
            k1, e_k1 = product(Y, e_Y, A0, es0, nv + 8)
            k2, e_k2 = product(W, e_W, A1, es1, nv + 8)
            ak, aq = k[:, r].abs(), q[:, r].abs()
            t = _sum(B) + 8
            abs_q = scale * m.grow * q1 + pq @ ak
            e_q = scale * m.grow * e_q1 + e_pq @ ak + t * (pq @ ak)
            abs_row = m.grow * k1 + pm @ ak
            e_row = m.grow * e_k1 + e_pm @ ak + t * (pm @ ak)
            T = lambda x: x.transpose(1, 2)  # noqa: E731
            abs_col = m.rest * k2 + T(pq) @ aq + T(pm) @ ak
            e_col = m.rest * e_k2 + T(e_pq) @ aq + T(e_pm) @ ak + t * (T(pq) @ aq + T(pm) @ ak)
            e_dq[:, r], e_dkey[:, r] = e_q + 2 * abs_q, e_row + e_col + 4 * (abs_row + abs_col)
            dot = lambda x, y: (x * y).sum(2, keepdim=True)  # noqa: E731
            size = dot(aq, abs_q) + dot(ak, abs_row + abs_col)
            e_dot = dot(aq, e_q) + dot(ak, e_row + e_col) + (2 * dk + 16) * size
            tail = m.whole * ((A0 * A1).sum((1, 2), keepdim=True)) + (ak * (m.rest * k2)).sum((1, 2), keepdim=True)
            e_tail = (m.whole * ((A0 * es1 + A1 * es0).sum((1, 2), keepdim=True)) + (ak * (m.rest * e_k2)).sum((1, 2), keepdim=True) +
                      (dk * dv / 16 + rows_in + 64) * tail)
            e_da[:, r] = torch.flip(torch.cumsum(torch.flip(e_dot + 16 * size, [1]), 1), [1]) + e_tail + 16 * tail
    # X and E are products of their own for dbeta and dv
    db, e_db = (X * E).sum(2), (X.abs() * e_E + E.abs() * e_X + (dv + 16) * (X * E).abs()).sum(2)
    dv_, e_dv = beta[:, :, None] * X, beta[:, :, None].abs() * (e_X + 2 * X.abs())
    inside = torch.zeros(rows, dtype=F64)
    for b, n in lens:
        inside[b:n] = 1.0

    def shared(x):
        return _flat((x * inside[None, :, None]).reshape(key_heads, group, rows, -1).sum(1))

    def joined(x):
        return _flat(x * inside[None, :, None])

    return ((shared(dq), shared(e_dq + group * dq.abs()) + LOST), (shared(dkey), shared(e_dkey + group * dkey.abs()) + LOST),
            (joined(dv_), joined(e_dv) + LOST), (joined(da), joined(e_da) + LOST), (joined(db[:, :, None]), joined(e_db[:, :, None]) + LOST),
            (dh0, e_dh0 + LOST))


def delta_step(q, k, v, decay, beta, state, key_heads, scale):
    """o, state."""
    heads = decay.shape[1]
    group = heads // key_heads
    n, dk = q.shape[0], q.shape[1] // key_heads
    scale = dk ** -0.5 if scale is None else scale
    q, k = (x.double().reshape(n, key_heads, dk).repeat_interleave(group, 1)[..., None] for x in (q, k))
    v = v.double().reshape(n, heads, 1, -1)
    S = torch.exp(decay.double())[..., None, None] * state.double()
    e = v - (k * S).sum(2, keepdim=True)
    bt = beta.double()[..., None, None]
    new = S + bt * k * e
    size_e = v.abs() + (k * S).abs().sum(2, keepdim=True)
    e_e = (dk + 16) * size_e
    e_new = 6 * S.abs() + (bt * k).abs() * (e_e + 4 * size_e) + new.abs()
    o = scale * (q * new).sum(2)
    qk = (q * k).abs().sum(2, keepdim=True)
    e_o = scale * ((dk + 16) * (q * S).abs().sum(2, keepdim=True) + bt.abs() * qk * (e_e + (dk + 16) * size_e))
    return (o.reshape(n, -1), e_o.reshape(n, -1)), (new, e_new)


def check_norm(name, got, value):
    """The 2-norm of the difference: half a step of the type where each element is rounded, and 64 units for the arithmetic. Roundings are
    as often up as down, so those of n terms add up to sqrt(n) of them: 28 for 128 products of six parts, and the chain from a state to
    the next, and from there to a gradient, has some five such sums, of 28 sqrt(5) = 63 together."""
    step = torch.finfo(got.dtype).eps / 2
    got, value = got.detach().cpu().double(), value.double()
    assert got.shape == value.shape and got.isfinite().all(), name
    off, size = float((got - value).norm()), float(value.norm())
    assert off <= (step + 64 * U) * size + U * LOST * math.sqrt(value.numel()), "%s: off by %.3g of its norm, %.3g allowed" % (name, off / size if size else off, step + 64 * U)


# ------------------------------------------------------------------ policy loss
def policy(logits, index, old, advantage, reference, kl, low, high, temperature, weight):
    """loss, logprob, dlogits."""
    x = logits.double() / temperature
    rows, classes = x.shape
    w = torch.ones(rows, dtype=F64) if weight is None else weight.double()
    there = (index >= 0) & (index < classes)
    at = index.clamp(0, classes - 1).long()[:, None]
    log_q = torch.log_softmax(x, 1)
    qs = log_q.exp()
    lp = log_q.gather(1, at)[:, 0]
    far = (x.max(1, keepdim=True).values - x).clamp(max=200)
    # a term: the difference, its product with the scale and exp2, relative to it; then the sum
    e_term = 4 + 3 * far
    e_lp = (qs * e_term).sum(1) + _serial(classes)
    A = torch.zeros(rows, dtype=F64) if advantage is None else advantage.double()
    d = lp - old.double() if old is not None else torch.zeros_like(lp)
    limited = torch.where(A >= 0, d > math.log1p(high), d < (math.log1p(-low) if low < 1 else -math.inf))
    r = torch.where(limited, torch.where(A >= 0, torch.full_like(d, 1 + high), torch.full_like(d, 1 - low)), d.exp())
    loss, e_loss = -A * r, torch.where(limited, torch.zeros_like(r), (A * r).abs() * e_lp)
    by, e_by = torch.where(limited, torch.zeros_like(r), -A * r), e_loss.clone()
    if reference is not None:
        g = reference.double() - lp
        near = torch.expm1(g)
        loss, e_loss = loss + kl * (near - g), e_loss + abs(kl) * near.abs() * e_lp
        by, e_by = by - kl * near, e_by + abs(kl) * (near + 1) * e_lp
    f, e_f = w * by / temperature, w.abs() * e_by / temperature
    one = torch.zeros_like(qs).scatter_(1, at, 1.0)
    e_q = qs * (e_term + e_lp[:, None] + 4)
    e_q = torch.where(one > 0, (qs * e_lp[:, None]), e_q)   # its own from the log-probability
    grad = f[:, None] * (one - qs)
    e_grad = e_f[:, None] * (one - qs).abs() + f.abs()[:, None] * e_q + 2 * grad.abs() + f.abs()[:, None] * 2.0 ** -100
    off = ~there | (w == 0)
    for t in (loss, e_loss, grad, e_grad):
        t[off] = 0.0
    lp, e_lp = torch.where(there, lp, torch.zeros_like(lp)), torch.where(there, e_lp, torch.zeros_like(lp))
    return (w * loss, w.abs() * e_loss + 2 * (w * loss).abs()), (lp, e_lp), (grad, e_grad)


# ------------------------------------------------------------------ clipping
def clip(tensors, max_norm):
    """norm, and the results."""
    norm = torch.stack([(t.double() ** 2).sum() for t in tensors]).sum().sqrt()
    f = 1.0 if max_norm is None or not norm > max_norm or not torch.isfinite(norm) else float(max_norm / norm)
    e = 0.0 if f == 1.0 else 2.0
    return (norm, norm * 2.0 ** -10), [(t.double() * f, e * (t.double() * f).abs()) for t in tensors]
