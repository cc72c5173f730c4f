"""The operators on whole arrays as far as no GPU is needed: what the C entry points and their torch wrappers refuse, and the 64-bit
references of the GPU tests against differences."""
import ctypes as ct

import pytest
import torch

import ops_reference as ref
from paper_1705_09786_amd import binding as B
from paper_1705_09786_amd import operators as ops

P = 0x20000000   # addresses that no refused call reads
MB = 1 << 20


def refused(rc, part, code=B.AMP_EINVAL):
    msg = B.lib().amp_operator_error().decode()
    assert rc == code and part in msg, (rc, msg)


def norm_forward(dtype=B.F32, rows=4, cols=8, x=P, xs=8, w=None, b=None, eps=1e-5, y=P + MB, ys=8, mean=None, rstd=None):
    return B.lib().amp_layer_norm_forward(dtype, rows, cols, x, xs, w, b, eps, y, ys, mean, rstd, None)


def test_norm_forward_refusals():
    refused(norm_forward(dtype=3), "dtype")
    refused(norm_forward(dtype=-1), "dtype")
    refused(norm_forward(rows=1 << 31), "rows")
    refused(norm_forward(cols=0), "cols")
    refused(norm_forward(cols=1 << 31), "cols")
    refused(norm_forward(eps=-1.0), "eps")
    refused(norm_forward(eps=float("nan")), "eps")
    refused(norm_forward(x=None), "x is NULL")
    refused(norm_forward(y=None), "y is NULL")
    refused(norm_forward(x=P + 2), "aligned")
    refused(norm_forward(dtype=B.BF16, x=P + 1), "aligned")
    refused(norm_forward(ys=7), "overlap")
    refused(norm_forward(xs=1 << 60), "spans")
    refused(norm_forward(y=P + 4), "y overlaps x")
    refused(norm_forward(y=P, ys=9), "y overlaps x")
    refused(norm_forward(mean=P + MB + 4), "y overlaps mean")
    refused(norm_forward(mean=P + 2 * MB, rstd=P + 2 * MB + 8), "mean overlaps rstd")
    refused(norm_forward(w=P + MB), "y overlaps weight")
    assert norm_forward(rows=0) == B.AMP_OK   # nothing to do, nothing launched


def norm_backward(dtype=B.F32, rows=400, cols=8, dy=P, dys=8, x=P + MB, xs=8, w=None, mean=P + 2 * MB, rstd=P + 3 * MB, dx=P + 4 * MB, dxs=8,
                  dw=P + 5 * MB, db=P + 6 * MB, ws=P + 7 * MB, n=16 * MB):
    return B.lib().amp_layer_norm_backward(dtype, rows, cols, dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, ws, n, None)


def test_norm_backward_refusals():
    refused(norm_backward(dtype=7), "dtype")
    refused(norm_backward(cols=0), "cols")
    for name in ("dy", "x", "mean", "rstd"):
        refused(norm_backward(**{name: None}), name + " is NULL")
    refused(norm_backward(dxs=4), "overlap")
    refused(norm_backward(dx=P + 4), "dx overlaps dy")
    refused(norm_backward(dw=P + 6 * MB + 4), "dweight overlaps dbias")
    refused(norm_backward(ws=None), "workspace")
    refused(norm_backward(ws=P + 7 * MB + 4), "workspace")
    refused(norm_backward(n=8), "workspace", B.AMP_ENOMEM)
    refused(norm_backward(ws=P + 5 * MB), "dweight overlaps workspace")
    assert norm_backward(dx=None, dw=None, db=None, ws=None, n=0) == B.AMP_OK
    n = ct.c_size_t()
    assert B.lib().amp_layer_norm_workspace(B.F32, 400, 8, ct.byref(n)) == B.AMP_OK and n.value > 0
    assert B.lib().amp_layer_norm_workspace(B.F32, 4, 8, ct.byref(n)) == B.AMP_OK and n.value == 0   # one workgroup has all rows
    refused(B.lib().amp_layer_norm_workspace(B.F32, 4, 8, None), "bytes")


def scan_forward(dtype=B.F32, act=0, rows=16, hidden=8, gate=P, gs=8, cand=P + MB, cs=8, seq=(1, None, None, 0), h0=None, h=P + 2 * MB,
                 hs=8, last=None, carry=None, ws=P + 8 * MB, n=64 * MB):
    q = None if seq is None else ct.byref(B.Sequences(*seq))
    return B.lib().amp_gated_scan_forward(dtype, act, rows, hidden, gate, gs, cand, cs, q, h0, h, hs, last, carry, ws, n, None)


def test_scan_forward_refusals():
    refused(scan_forward(dtype=9), "dtype")
    refused(scan_forward(act=1), "activation")
    refused(scan_forward(act=3), "activation")
    refused(scan_forward(hidden=0), "hidden")
    refused(scan_forward(hidden=1 << 22, gs=1 << 22, cs=1 << 22, hs=1 << 22), "hidden")
    refused(scan_forward(rows=1 << 30), "rows")
    refused(scan_forward(seq=None), "sequences is NULL")
    refused(scan_forward(seq=(2, None, None, 0)), "without begin and end")
    refused(scan_forward(seq=(2, P, None, 4)), "begin and end")
    refused(scan_forward(seq=(2, P + 3 * MB, P + 3 * MB + 4, 2)), "index_bytes")
    refused(scan_forward(seq=(2, P + 3 * MB + 4, P + 3 * MB + 12, 8)), "aligned")
    refused(scan_forward(seq=(1 << 31, P, P, 8)), "sequences")
    refused(scan_forward(gate=None), "gate is NULL")
    refused(scan_forward(cand=None), "cand is NULL")
    refused(scan_forward(h=P), "h overlaps gate")
    refused(scan_forward(h=P + MB + 32), "h overlaps cand")
    refused(scan_forward(last=P + 2 * MB), "h overlaps last")
    refused(scan_forward(last=P + 3 * MB, h0=P + 3 * MB), "last overlaps h0")
    refused(scan_forward(carry=P), "carry overlaps gate")
    refused(scan_forward(seq=(2, P + 3 * MB, P + 3 * MB + 4, 4), last=P + 3 * MB), "last overlaps begin")
    assert scan_forward(seq=(0, None, None, 0)) == B.AMP_OK
    assert scan_forward(h=None) == B.AMP_OK   # nothing asked for


def scan_backward(dtype=B.F32, act=0, rows=300, hidden=8, dh=P, ds=8, dlast=None, gate=P + MB, gs=8, cand=P + 2 * MB, cs=8,
                  seq=(1, None, None, 0), h0=None, carry=P + 3 * MB, dgate=P + 4 * MB, dgs=8, dcand=P + 5 * MB, dcs=8, dh0=None,
                  ws=P + 8 * MB, n=64 * MB):
    q = None if seq is None else ct.byref(B.Sequences(*seq))
    return B.lib().amp_gated_scan_backward(dtype, act, rows, hidden, dh, ds, dlast, gate, gs, cand, cs, q, h0, carry, dgate, dgs, dcand, dcs,
                                           dh0, ws, n, None)


def test_scan_backward_refusals():
    refused(scan_backward(act=1), "activation")
    for name in ("dh", "gate", "cand", "carry", "dgate", "dcand"):
        refused(scan_backward(**{name: None}), name + " is NULL")
    refused(scan_backward(dgate=P + 5 * MB), "dgate overlaps dcand")
    refused(scan_backward(dgs=4), "overlap")
    refused(scan_backward(dgate=P), "dgate overlaps dh")
    refused(scan_backward(dh0=P + 3 * MB), "dh0 overlaps carry")
    refused(scan_backward(dlast=P + 6 * MB, dh0=P + 6 * MB), "dh0 overlaps dlast")
    assert scan_backward(seq=(0, None, None, 0)) == B.AMP_OK


def test_scan_rows_of_no_sequence_refusals():
    refused(scan_forward(seq=(2, P + 3 * MB, P + 3 * MB + 4, 4, 2)), "zero_others")
    refused(scan_backward(seq=(1, None, None, 0, -1)), "zero_others")
    # without sequences every row is one to be zeroed: not a call that has nothing to do
    refused(scan_forward(seq=(0, None, None, 0, 1), gate=None), "gate is NULL")
    refused(scan_backward(seq=(0, None, None, 0, 1), dgate=None), "dgate is NULL")
    assert scan_forward(seq=(0, None, None, 0, 1), h=None) == B.AMP_OK


def test_scan_backward_without_rows_needs_the_carry():
    """A call without rows starts its kernel too, for dh0, and the kernel reads a row of the carry."""
    refused(scan_backward(rows=0, carry=None), "carry is NULL")
    refused(scan_backward(rows=0, carry=None, dh=None, gate=None, cand=None, dgate=None, dcand=None, seq=(2, P + 6 * MB, P + 6 * MB + 4, 4)),
            "carry is NULL")
    n = ct.c_size_t()
    assert B.lib().amp_gated_scan_carry(B.F32, 0, 8, ct.byref(n)) == B.AMP_OK and n.value == 1


def test_scan_workspace_is_checked():
    n = ct.c_size_t()
    assert B.lib().amp_gated_scan_workspace(B.F32, 100000, 8, ct.byref(n)) == B.AMP_OK
    if n.value:
        refused(scan_forward(rows=100000, h=P + 16 * MB, cand=P + 8 * MB, ws=P + 32 * MB, n=n.value - 1), "workspace", B.AMP_ENOMEM)
        refused(scan_forward(rows=100000, h=P + 16 * MB, cand=P + 8 * MB, ws=None), "workspace")
        refused(scan_forward(rows=100000, h=P + 16 * MB, cand=P + 8 * MB, ws=P + 32 * MB + 8), "workspace")
    assert B.lib().amp_gated_scan_carry(B.F32, 0, 8, ct.byref(n)) == B.AMP_OK
    assert B.lib().amp_gated_scan_workspace(B.F32, 1 << 22, 1 << 14, ct.byref(n)) == B.AMP_OK
    refused(B.lib().amp_gated_scan_workspace(B.F32, (1 << 22) + 1, 1 << 14, ct.byref(n)), "elements")
    refused(scan_forward(rows=(1 << 24) + 1, hidden=1 << 12, gs=0, cs=0, h=None), "elements")
    refused(B.lib().amp_gated_scan_carry(B.F32, 5, 8, None), "carry_rows")
    refused(B.lib().amp_gated_scan_workspace(5, 5, 8, ct.byref(n)), "dtype")


def test_scan_halves_of_one_array_do_not_overlap():
    """Gate and candidate as the halves of one projection, and their gradients likewise: refused for what comes after that check."""
    refused(scan_backward(gate=P + MB, gs=16, cand=P + MB + 32, cs=16, dgate=P + 4 * MB, dgs=16, dcand=P + 4 * MB + 32, dcs=16,
                          dh0=P + 4 * MB), "dgate overlaps dh0")
    refused(scan_backward(dgate=P + 4 * MB, dgs=16, dcand=P + 4 * MB + 28, dcs=16), "dgate overlaps dcand")


def scan_step(dtype=B.F32, act=0, rows=4, hidden=8, gate=P, gs=8, cand=P + MB, cs=8, state=P + 2 * MB, ss=8, h=P + 3 * MB, hs=8):
    return B.lib().amp_gated_scan_step(dtype, act, rows, hidden, gate, gs, cand, cs, state, ss, h, hs, None)


def test_scan_step_refusals():
    refused(scan_step(act=1), "activation")
    refused(scan_step(state=None), "state is NULL")
    refused(scan_step(gate=None), "gate is NULL")
    refused(scan_step(ss=4), "overlap")
    refused(scan_step(ss=0), "overlap")   # one state for every row
    refused(scan_step(h=P + 2 * MB), "state overlaps h")
    refused(scan_step(state=P + 4), "state overlaps gate")
    assert scan_step(rows=0) == B.AMP_OK


def distill(dtype=B.F32, rows=4, classes=50, x=P, xs=50, top=5, td=B.F32, teacher=P + MB, ts=5, index=P + 2 * MB, ib=8, ins=5, T=2.0, w=None,
            loss=P + 3 * MB, dx=P + 4 * MB, dxs=50, ws=P + 8 * MB, n=8 * MB):
    return B.lib().amp_distill_loss(dtype, rows, classes, x, xs, top, td, teacher, ts, index, ib, ins, T, w, loss, dx, dxs, ws, n, None)


def test_distill_refusals():
    refused(distill(dtype=4), "dtype")
    refused(distill(td=4), "teacher_dtype")
    refused(distill(ib=2), "index_bytes")
    refused(distill(top=0), "top")
    refused(distill(top=1025, ts=1025, ins=1025), "top")
    for T in (0.0, -1.0, float("nan"), float("inf"), 1e-7, 1e7):
        refused(distill(T=T), "temperature")
    for name, word in (("x", "logits"), ("teacher", "teacher"), ("index", "index")):
        refused(distill(**{name: None}), word + " is NULL")
    refused(distill(dx=P, dxs=51), "dlogits overlaps logits")
    refused(distill(dx=P + 4), "dlogits overlaps logits")
    refused(distill(dxs=49), "overlap")
    refused(distill(loss=P + MB), "loss overlaps teacher")
    refused(distill(index=P + 2 * MB + 4), "aligned")
    assert distill(rows=0) == B.AMP_OK
    assert distill(loss=None, dx=None) == B.AMP_OK


def test_wrappers_refuse_what_is_not_on_a_gpu():
    x, w = torch.zeros(4, 8), torch.zeros(8)
    i = torch.zeros(4, 3, dtype=torch.int64)
    for call in (lambda: ops.layer_norm(x, w), lambda: ops.layer_norm(None), lambda: ops.layer_norm(x[0]),
                 lambda: ops.layer_norm_backward(x, x, w, x[:, 0], x[:, 0]), lambda: ops.gated_scan(x, x),
                 lambda: ops.gated_scan_backward(x, x, x, x), lambda: ops.gated_scan_step(x, x, x),
                 lambda: ops.distill_loss(x, x[:, :3], i)):
        with pytest.raises(B.AmpError) as e:
            call()
        assert e.value.code == B.AMP_EINVAL


def test_wrappers_refuse_tensors_that_require_grad():
    """Checked before anything that needs a GPU; torch.no_grad() brings the call to the next check."""
    x, g = torch.zeros(4, 8), torch.zeros(4, 8, requires_grad=True)
    i = torch.zeros(4, 3, dtype=torch.int64)
    for call in (lambda: ops.layer_norm(g), lambda: ops.layer_norm_backward(x, g, None, x[:, 0], x[:, 0]), lambda: ops.gated_scan(g, x),
                 lambda: ops.gated_scan_backward(x, g, x, x), lambda: ops.gated_scan_step(g, x, x), lambda: ops.distill_loss(g, x[:, :3], i)):
        with pytest.raises(B.AmpError, match="requires grad"):
            call()
        with torch.no_grad(), pytest.raises(B.AmpError, match="not on a GPU"):
            call()


# ------------------------------------------------------------------ the references against differences, in 64 bits
def differences(f, x, eps=1e-6):
    g = torch.zeros_like(x)
    flat, out = x.reshape(-1), g.reshape(-1)
    for i in range(flat.numel()):
        old = float(flat[i])
        flat[i] = old + eps
        up = float(f())
        flat[i] = old - eps
        out[i] = (up - float(f())) / (2 * eps)
        flat[i] = old
    return g


def close(a, b):
    # central differences: eps^2 of truncation, 2^-53 / eps of rounding
    assert torch.allclose(a, b, rtol=1e-7, atol=1e-8), (a - b).abs().max()


def rand(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_norm_reference_against_differences():
    x, w, b, dy = rand(3, 7), 1 + 0.2 * rand(7, seed=1), rand(7, seed=2), rand(3, 7, seed=3)
    f = lambda: (ref.norm(x, w, b, 1e-3)[0][0] * dy).sum()
    _, (mean, _), (rstd, _) = ref.norm(x, w, b, 1e-3)
    (dx, _), (dw, _), (db, _) = ref.norm_backward(dy, x, w, mean, rstd)
    close(dx, differences(f, x))
    close(dw, differences(f, w))
    close(db, differences(f, b))


@pytest.mark.parametrize("tanh", [False, True])
def test_scan_reference_against_differences(tanh):
    seq = (torch.tensor([0, 2, 2, 7]), torch.tensor([2, 2, 6, 8]))   # an empty one, a row of none
    gate, cand, h0, dh, dlast = rand(9, 3), rand(9, 3, seed=1), rand(4, 3, seed=2), rand(9, 3, seed=3), rand(4, 3, seed=4)

    def f():
        (h, _), (last, _), _ = ref.scan(gate, cand, seq, h0, tanh)
        return (h * dh).sum() + (last * dlast).sum()
    (dgate, _), (dcand, _), (dh0, _) = ref.scan_backward(dh, dlast, gate, cand, seq, h0, tanh)
    close(dgate, differences(f, gate))
    close(dcand, differences(f, cand))
    close(dh0, differences(f, h0))


def test_distill_reference_against_differences():
    x, y = rand(4, 11), rand(4, 5, seed=1)
    index = torch.tensor([[0, 3, 10, 5, 7], [2, 2, 2, 9, -1], [-1, 11, -5, 12, 99], [1, 2, 3, 4, 6]])   # twice the same, none at all
    w = torch.tensor([1.0, 0.5, 1.0, 0.0], dtype=torch.float64)
    y[0, 2] = -float("inf")
    f = lambda: ref.distill(x, y, index, 1.7, w)[0][0].sum()
    (loss, _), (grad, _) = ref.distill(x, y, index, 1.7, w)
    assert loss[2] == 0 and loss[3] == 0 and loss[0] > 0
    close(grad, differences(f, x))
