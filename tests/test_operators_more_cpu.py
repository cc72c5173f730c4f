"""The gated delta rule, the policy loss and clipping as far as no GPU is needed: what the C entry points refuse, and the 64-bit
references of the GPU tests against differences and other forms of the formulas."""
import ctypes as ct

import pytest
import torch
import torch.nn.functional as F

import more_reference as more
from paper_1705_09786_amd import binding as B
from paper_1705_09786_amd import operators as ops
from test_operators_cpu import MB, P, refused

AT = {name: P + 16 * i * MB for i, name in enumerate(
    ("q", "k", "v", "decay", "beta", "h0", "o", "last", "carry", "dout", "dlast", "to_dq", "to_dk", "to_dv", "to_ddecay", "to_dbeta", "dh0", "state", "ws"))}
SHAPE = dict(dtype=B.F32, rows=100, heads=4, key_heads=2, dk=8, dv=16)


def shape(kw):
    return B.DeltaShape(*[kw.pop(k, v) for k, v in SHAPE.items()])


def sequences(seq):
    return None if seq is None else ct.byref(B.Sequences(*seq))


def arrays(kw, *names):
    """Addresses and strides of q, k, v, decay, beta and the like, by their defaults."""
    wide = dict(q=16, k=16, v=64, decay=4, beta=4, o=64, dout=64, to_dq=16, to_dk=16, to_dv=64, to_ddecay=4, to_dbeta=4)
    return [x for n in names for x in (kw.pop(n, AT[n]), kw.pop(n + "_stride", wide[n]))]


FIVE = ("q", "k", "v", "decay", "beta")


def forward(seq=(1, None, None, 0, 0), h0=None, last=None, carry=None, ws=AT["ws"], n=64 * MB, null=False, **kw):
    s = shape(kw)
    five, o = arrays(kw, *FIVE), arrays(kw, "o")
    assert not kw
    return B.lib().amp_gated_delta_forward(None if null else s, *five, 1.0, sequences(seq), h0, *o, last, carry, ws, n, None)


def backward(seq=(1, None, None, 0, 0), dlast=None, carry=AT["carry"], dh0=AT["dh0"], ws=AT["ws"], n=64 * MB, **kw):
    s = shape(kw)
    dout, five, out = arrays(kw, "dout"), arrays(kw, *FIVE), arrays(kw, "to_dq", "to_dk", "to_dv", "to_ddecay", "to_dbeta")
    assert not kw
    return B.lib().amp_gated_delta_backward(s, *dout, dlast, *five, 1.0, sequences(seq), carry, *out, dh0, ws, n, None)


def step(state=AT["state"], stride=4 * 8 * 16, **kw):
    s = shape(kw)
    five, o = arrays(kw, *FIVE), arrays(kw, "o")
    assert not kw
    return B.lib().amp_gated_delta_step(s, *five, 1.0, state, stride, *o, None)


def test_delta_shape_refusals():
    for f in (forward, backward, step):
        refused(f(dtype=3), "dtype")
        refused(f(rows=1 << 30), "rows")
        refused(f(heads=0), "heads")
        refused(f(heads=1 << 16, key_heads=1), "heads")
        refused(f(key_heads=0), "key_heads")
        refused(f(key_heads=3), "key_heads")
        refused(f(key_heads=8), "key_heads")
        refused(f(dk=0), "dk")
        refused(f(dk=129), "dk")
        refused(f(dv=0), "dv")
        refused(f(dv=1025), "dv")
        refused(f(rows=(1 << 26) + 64), "2^22")
        for name in FIVE:
            refused(f(**{name: None}), name + " is NULL")
            refused(f(**{name: AT[name] + 2}), "aligned")
            refused(f(**{name + "_stride": 1 << 60}), "spans")
        refused(f(heads=32768, key_heads=1, dv=128), "2^22")
        refused(f(heads=32768, key_heads=32768, dk=128), "2^22")
    for f, names in ((forward, ("q", "k", "v", "o")), (backward, ("q", "k", "v", "dout"))):
        for name in names:
            refused(f(**{name + "_stride": 1 << 22}), "2^22")
    refused(forward(null=True), "shape is NULL")
    refused(forward(seq=(1 << 22, P, P, 8, 0)), "2^22")


def test_delta_forward_refusals():
    refused(forward(seq=None), "sequences is NULL")
    refused(forward(seq=(2, None, None, 0, 0)), "without begin and end")
    refused(forward(seq=(2, P, None, 4, 0)), "begin and end")
    refused(forward(seq=(2, P, P + 4, 2, 0)), "index_bytes")
    refused(forward(seq=(2, P + 4, P + 12, 8, 0)), "aligned")
    refused(forward(seq=(2, P, P + 8, 8, 2)), "zero_others")
    refused(forward(o_stride=63), "overlap")
    refused(forward(o=AT["v"] + 64), "o overlaps v")
    refused(forward(o=AT["q"]), "o overlaps q")
    refused(forward(last=AT["o"]), "o overlaps last")
    refused(forward(last=AT["h0"], h0=AT["h0"]), "last overlaps h0")
    refused(forward(carry=AT["beta"]), "carry overlaps beta")
    refused(forward(ws=None), "workspace")
    refused(forward(ws=AT["ws"] + 4), "workspace")
    refused(forward(n=100), "workspace", B.AMP_ENOMEM)
    refused(forward(ws=AT["o"]), "o overlaps workspace")
    assert forward(seq=(0, None, None, 0, 0)) == B.AMP_OK
    assert forward(o=None) == B.AMP_OK   # nothing asked for


def test_delta_backward_refusals():
    for name in ("dout", "carry", "to_dq", "to_dk", "to_dv", "to_ddecay", "to_dbeta"):
        refused(backward(**{name: None}), name.replace("to_", "") + " is NULL")
    refused(backward(to_dq_stride=15), "overlap")
    refused(backward(to_dq=AT["to_dk"]), "dq overlaps dk")
    refused(backward(to_dv=AT["dout"]), "dv overlaps dout")
    refused(backward(to_ddecay=AT["decay"]), "ddecay overlaps decay")
    refused(backward(dh0=AT["carry"]), "dh0 overlaps carry")
    refused(backward(dh0=AT["dlast"], dlast=AT["dlast"]), "dh0 overlaps dlast")
    refused(backward(n=1 << 10), "workspace", B.AMP_ENOMEM)
    assert backward(seq=(0, None, None, 0, 0)) == B.AMP_OK


def test_delta_step_refusals():
    refused(step(state=None), "state is NULL")
    refused(step(stride=511), "overlap")
    refused(step(o=AT["state"]), "state overlaps o")
    refused(step(state=AT["q"]), "state overlaps q")
    refused(step(rows=(1 << 20) + 1, heads=4), "2^22")
    assert step(rows=0) == B.AMP_OK


def test_delta_sizes():
    n = ct.c_size_t()
    lib = B.lib()
    s = B.DeltaShape(*SHAPE.values())
    assert lib.amp_gated_delta_carry(s, 3, ct.byref(n)) == B.AMP_OK
    assert n.value == (100 // 64 + 3) * 4 * (64 + 8) * 16
    sizes = []
    for back in (0, 1):
        assert lib.amp_gated_delta_workspace(s, 3, back, ct.byref(n)) == B.AMP_OK
        sizes.append(n.value)
    assert sizes[1] > sizes[0] > 0
    refused(lib.amp_gated_delta_carry(s, 3, None), "floats")
    refused(lib.amp_gated_delta_workspace(s, 3, 0, None), "bytes")
    refused(lib.amp_gated_delta_carry(None, 3, ct.byref(n)), "shape")


def policy(dtype=B.F32, rows=4, classes=9, logits=P, ls=9, index=P + MB, size=8, temperature=1.0, advantage=P + 2 * MB, old=P + 3 * MB,
           reference=P + 4 * MB, kl=0.1, low=0.2, high=0.2, weight=None, loss=P + 5 * MB, logprob=P + 6 * MB, dlogits=P + 7 * MB, ds=9):
    return B.lib().amp_policy_loss(dtype, rows, classes, logits, ls, index, size, temperature, advantage, old, reference, kl, low, high, weight, loss,
                                   logprob, dlogits, ds, None)


def test_policy_refusals():
    nan, inf = float("nan"), float("inf")
    refused(policy(dtype=5), "dtype")
    refused(policy(rows=1 << 31), "rows")
    refused(policy(classes=0), "classes")
    refused(policy(size=2), "index_bytes")
    for t in (0.0, -1.0, nan, inf):
        refused(policy(temperature=t), "temperature")
    for c in (-0.1, 1.1, nan):
        refused(policy(low=c), "clip_low")
    for c in (-0.1, nan):
        refused(policy(high=c), "clip_high")
    for k in (nan, inf):
        refused(policy(kl=k), "kl")
    for name in ("logits", "index", "advantage"):
        refused(policy(**{name: None}), name + " is NULL")
    refused(policy(ds=8), "overlap")
    refused(policy(dlogits=P + 4), "dlogits overlaps logits")
    refused(policy(dlogits=P, ds=10), "dlogits overlaps logits")
    refused(policy(loss=P + 6 * MB + 4), "loss overlaps logprob")
    refused(policy(logprob=P + 3 * MB), "logprob overlaps old")
    refused(policy(old=P + 3 * MB + 2), "aligned")
    assert policy(rows=0) == B.AMP_OK
    assert policy(loss=None, logprob=None, dlogits=None) == B.AMP_OK


def clip(tensors, max_norm=1.0, norm=P + 64 * MB, ws=P + 65 * MB, n=MB, null=False):
    table = (B.Tensor * max(1, len(tensors)))(*[B.Tensor(*t) for t in tensors])
    return B.lib().amp_clip_gradients(len(tensors), None if null else table, max_norm, norm, ws, n, None)


def test_clip_refusals():
    one = (P, None, 100, B.F32)
    refused(clip([(P, None, 100, 3)]), "dtype")
    refused(clip([(None, None, 100, B.F32)]), "NULL")
    refused(clip([(P + 2, None, 100, B.F32)]), "aligned")
    refused(clip([(P, P + MB + 1, 100, B.BF16)]), "aligned")
    refused(clip([(P, None, 1 << 41, B.F32)]), "2^40")
    refused(clip([(P, None, 1 << 39, B.F32)] * 3), "2^40")
    refused(clip([one], null=True), "NULL")
    refused(clip([one], max_norm=-1.0), "max_norm")
    refused(clip([one], max_norm=float("nan")), "max_norm")
    refused(clip([one], norm=P + 64 * MB + 2), "norm")
    refused(clip([one], ws=None), "workspace")
    refused(clip([one], n=8), "workspace", B.AMP_ENOMEM)
    refused(clip([(P, P + 4, 100, B.F32)]), "overlaps")
    refused(clip([(P, P, 100, B.F32), (P, None, 100, B.F32)]), "overlaps")
    refused(clip([(P, P, 100, B.F32), (P + 396, P + 396, 100, B.F32)]), "overlaps")
    refused(clip([(P, P + MB, 100, B.F32), (P + MB, None, 10, B.F32)]), "overlaps")
    refused(clip([(P, P + MB, 100, B.F32), (P + 2 * MB, P + MB + 396, 10, B.F32)]), "overlaps")
    refused(clip([(P, None, 100, B.F32)], norm=P + 8), "overlaps")
    refused(clip([(P, P + 65 * MB, 100, B.F32)]), "overlaps")
    n = ct.c_size_t()
    refused(B.lib().amp_clip_workspace(1, None, ct.byref(n)), "NULL")
    refused(B.lib().amp_clip_workspace(1, (B.Tensor * 1)(B.Tensor(*one)), None), "bytes")
    assert B.lib().amp_clip_workspace(1, (B.Tensor * 1)(B.Tensor(*one)), ct.byref(n)) == B.AMP_OK and n.value > 0


def test_tensors_on_the_cpu_are_refused():
    x = torch.zeros(4, 8)
    for f in (lambda: ops.gated_delta(x, x, x, x[:, :1], x[:, :1]), lambda: ops.token_logprob(x, torch.zeros(4, dtype=torch.int64)),
              lambda: ops.gated_delta_step(x, x, x, x[:, :1], x[:, :1], torch.zeros(4, 1, 8, 8)), lambda: ops.clip_gradients([x])):
        with pytest.raises(B.AmpError):
            f()


# ------------------------------------------------------------------ the references
def inputs(rows=75, heads=4, key_heads=2, dk=6, dv=5):
    g = torch.Generator().manual_seed(3)

    def n(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    q, k = (F.normalize(n(rows, key_heads, dk), dim=2).reshape(rows, -1) for _ in range(2))
    return [q, k, n(rows, heads * dv), -0.1 * n(rows, heads).abs(), torch.sigmoid(n(rows, heads))], n(2, heads, dk, dv), n(rows, heads * dv), n(2, heads, dk, dv)


def test_delta_reference_against_derivatives():
    """The written-out backward pass against torch's derivatives of the recurrence, and those against differences."""
    x, h0, do, dlast = inputs()
    where = torch.tensor([0, 40, 75])
    for t in x + [h0]:
        t.requires_grad_()

    def run():
        return more.delta(*x, where, 2, 0.7, h0, torch.float32)[:2]

    (o, _), (last, _) = run()
    loss = (o * do).sum() + (last * dlast).sum()
    want = torch.autograd.grad(loss, x + [h0])
    with torch.no_grad():
        got = more.delta_backward(do, *x, where, 2, 0.7, h0, dlast, torch.float32)
        for (g, bound), w in zip(got, want):
            assert (g - w).abs().max() < 1e-12 * (1 + w.abs().max()) and (bound >= 0).all() and bound.isfinite().all()
        for t, w in zip(x + [h0], want):
            flat, dw = t.view(-1), w.reshape(-1)
            for i in (0, flat.numel() // 2, flat.numel() - 1):
                side = []
                for d in (1e-5, -1e-5):
                    flat[i] += d
                    (o, _), (last, _) = run()
                    side.append(float((o * do).sum() + (last * dlast).sum()))
                    flat[i] -= d
                assert abs((side[0] - side[1]) / 2e-5 - float(dw[i])) < 1e-6 * (1 + abs(float(dw[i])))


def test_delta_step_reference_is_a_row_of_the_recurrence():
    x, _, _, _ = inputs(2)
    h0 = torch.randn(2, 4, 6, 5, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    (o, _), (last, _) = more.delta(*x, torch.tensor([0, 1, 2]), 2, None, h0, torch.float32)[:2]
    (p, _), (state, _) = more.delta_step(*x, h0, 2, None)
    assert (o - p).abs().max() < 1e-14 and (last - state).abs().max() < 1e-14


def test_policy_reference_against_derivatives():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(40, 7, generator=g, dtype=torch.float64).requires_grad_()
    index = torch.randint(0, 7, (40,), generator=g)
    old, ref, adv = (torch.randn(40, generator=g, dtype=torch.float64) * s + m for s, m in ((0.3, -2.0), (0.3, -2.0), (1.0, 0.0)))
    w = torch.rand(40, generator=g, dtype=torch.float64)
    lp = torch.log_softmax(x / 0.7, 1).gather(1, index[:, None])[:, 0]
    r, d = torch.exp(lp - old), ref - lp
    loss = w * (-torch.minimum(r * adv, r.clamp(0.8, 1.3) * adv) + 0.1 * (torch.exp(d) - d - 1))
    want, = torch.autograd.grad(loss.sum(), x)
    with torch.no_grad():
        got = more.policy(x, index, old, adv, ref, 0.1, 0.2, 0.3, 0.7, w)
        for (v, bound), e in zip(got, (loss, lp, want)):
            assert (v - e).abs().max() < 1e-13 and (bound >= 0).all() and bound.isfinite().all()


def test_clip_reference():
    t = [torch.full((3,), 2.0), torch.full((1, 4), 1.0)]
    norm, out = more.clip(t, 2.0)
    assert norm[0] == 4.0 and (out[0][0] == 1.0).all() and (out[1][0] == 0.5).all()
    assert (more.clip(t, 5.0)[1][0][0] == 2.0).all()
