"""The operators on whole arrays over torch tensors: layer norm, the gated linear recurrence, the distillation loss (include/amp.h has
their formulas and conventions).  Marshalling only, as in runner: outputs and workspaces come from torch, the kernels run on
torch's current stream of the tensors' device, and a refused call raises binding.AmpError.

Arrays are 2-D tensors (rows, features) on one GPU, torch.float32, bfloat16 or float16, features next to each other, any row stride;
weights, states, statistics and losses are float32 and contiguous.  No call waits for the GPU or reads from it, so each can be captured
into a HIP graph.  There is no autograd: a layer's backward pass is a call of its own, as in the rest of the library.  A tensor that
requires grad is refused while grad mode is on, since its gradient would be lost (torch.no_grad(), detach(), or the forward and
backward of a torch.autograd.Function); writes to a caller's tensor count as in-place changes of it.
"""
from __future__ import annotations

import ctypes as ct
from functools import lru_cache

import torch

from . import binding as B

DTYPES = {torch.float32: B.F32, torch.bfloat16: B.BF16, torch.float16: B.F16}
ACTIVATIONS = {"none": B.ACT_NONE, "tanh": B.ACT_TANH}
_INDEX = {torch.int32: 4, torch.int64: 8}


# A small call is bound by what it does on the host, so torch's own current device and stream are read without its Python layer
# where this torch has them (0.2 us for 1.7).
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


def _refuse(msg):
    raise B.AmpError(B.AMP_EINVAL, msg)


def _differentiated(name):
    _refuse("%s requires grad, and no gradient would reach it: call under torch.no_grad() or with detach()" % name)


# Tells torch's own autograd that a caller's tensors were written to (without the Python layer: 0.15 us less in a step of 8.7).
_written = getattr(torch._C, "_increment_version", torch.autograd.graph.increment_version)


def _check(rc):
    if rc:
        raise B.AmpError(rc, B.lib().amp_operator_error().decode())


def _call(x, name, *args):
    """A C call on the current stream of x's device, which is current during the call."""
    index, fn = x.get_device(), getattr(B.lib(), name)
    try:
        if index == _current_device():
            rc = fn(*args, _stream_of(index))
        else:
            with torch.cuda.device(index):
                rc = fn(*args, _stream_of(index))
    except ct.ArgumentError as e:   # eps or temperature is no number
        _refuse("%s: %s" % (name, e))
    if rc:
        _check(rc)


def _rows(name, x, like=None, dtypes=DTYPES, shape=None):
    """x as rows of consecutive elements: (its address, its row stride); `like`: a tensor whose device (and, for arrays of the operators'
    types, type) it has to share."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        _refuse("%s is not a 2-D tensor" % name)
    if x.requires_grad and torch.is_grad_enabled():
        _differentiated(name)
    if not x.is_cuda:
        _refuse("%s is not on a GPU" % name)
    if x.dtype not in dtypes:
        _refuse("%s is of type %s" % (name, x.dtype))
    if like is not None:
        if x.get_device() != like.get_device():
            _refuse("%s is on another device" % name)
        if dtypes is DTYPES and x.dtype != like.dtype:
            _refuse("%s is of type %s, not %s" % (name, x.dtype, like.dtype))
    if shape is not None and x.shape != shape:
        _refuse("%s is %s, %s is needed" % (name, tuple(x.shape), tuple(shape)))
    row, col = x.stride()
    if col != 1 and x.size(1) > 1:
        _refuse("%s does not have its features next to each other (call contiguous())" % name)
    return x.data_ptr(), row


def _floats(name, x, like, *shape):
    """A contiguous float32 tensor of that shape, or None: its address."""
    if x is None:
        return None
    if not isinstance(x, torch.Tensor) or x.dtype != torch.float32 or x.shape != shape or not x.is_contiguous() or x.get_device() != like.get_device():
        _refuse("%s is not a contiguous float32 tensor of shape %s on %s" % (name, shape, like.device))
    if x.requires_grad and torch.is_grad_enabled():
        _differentiated(name)
    return x.data_ptr()


def _new(x):
    """An array of x's shape and type."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


@lru_cache(maxsize=4096)
def _size(call, dtype, rows, cols):
    n = ct.c_size_t()
    _check(getattr(B.lib(), call)(dtype, rows, cols, ct.byref(n)))
    return n.value


def _workspace(call, x):
    n = _size(call, DTYPES[x.dtype], x.size(0), x.size(1))
    return (torch.empty(n, dtype=torch.uint8, device=x.device), n) if n else (None, 0)


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------ layer norm
def layer_norm(x, weight=None, bias=None, eps=1e-5, *, stats=False, out=None):
    """(x - mean) / sqrt(var + eps) * weight + bias over each row, in x's type; with stats also the rows' mean and 1 / sqrt(var + eps),
    which the backward pass needs: (y, mean, rstd).  out: a tensor to write to (may be x)."""
    px, sx = _rows("x", x)
    rows, cols = shape = x.shape
    y = _new(x) if out is None else out
    py, sy = _rows("out", y, x, shape=shape)
    pw, pb = _floats("weight", weight, x, cols), _floats("bias", bias, x, cols)
    mean = rstd = None
    if stats:
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
        rstd = torch.empty_like(mean)
    _call(x, "amp_layer_norm_forward", DTYPES[x.dtype], rows, cols, px, sx, pw, pb, eps, py, sy, _ptr(mean), _ptr(rstd))
    if out is not None:
        _written((out,))
    return (y, mean, rstd) if stats else y


def layer_norm_backward(dy, x, weight, mean, rstd, *, out=None):
    """(dx, dweight, dbias) from the gradient of y, x, the weight (or None) and the statistics of layer_norm(.., stats=True).
    out: a tensor for dx (may be dy or x)."""
    px, sx = _rows("x", x)
    rows, cols = shape = x.shape
    pd, sd = _rows("dy", dy, x, shape=shape)
    dx = _new(x) if out is None else out
    po, so = _rows("out", dx, x, shape=shape)
    if mean is None or rstd is None:
        _refuse("mean and rstd are needed")
    pm, pr, pw = _floats("mean", mean, x, rows), _floats("rstd", rstd, x, rows), _floats("weight", weight, x, cols)
    dweight = torch.empty(cols, dtype=torch.float32, device=x.device)
    dbias = torch.empty_like(dweight)
    ws, n = _workspace("amp_layer_norm_workspace", x)
    _call(x, "amp_layer_norm_backward", DTYPES[x.dtype], rows, cols, pd, sd, px, sx, pw, pm, pr, po, so, dweight.data_ptr(), dbias.data_ptr(),
          _ptr(ws), n)
    if out is not None:
        _written((out,))
    return dx, dweight, dbias


# ------------------------------------------------------------------ gated linear recurrence
def _sequences(sequences, x, zero_others):
    """(struct, number): None = one sequence of all rows; a 1-D integer tensor of n + 1 offsets; or a pair (begin, end) of n each.
    zero_others: rows of no sequence become zeros (else they are left as they were)."""
    if sequences is None:
        return B.Sequences(1, None, None, 0, 0), 1
    pair = isinstance(sequences, (tuple, list))
    if pair and len(sequences) != 2:
        _refuse("sequences is not a tensor of offsets or a pair (begin, end)")
    for t in sequences if pair else (sequences,):
        if not isinstance(t, torch.Tensor) or t.dim() != 1 or t.dtype not in _INDEX or not t.is_contiguous() or t.device != x.device:
            _refuse("sequences: contiguous 1-D int32 or int64 tensors on %s are needed" % (x.device,))
    if pair:
        begin, end = sequences
        if begin.dtype != end.dtype or begin.numel() != end.numel():
            _refuse("sequences: begin and end differ in type or length")
        n, size, pb, pe = begin.numel(), _INDEX[begin.dtype], begin.data_ptr(), end.data_ptr()
    else:
        n, size, pb = sequences.numel() - 1, _INDEX[sequences.dtype], sequences.data_ptr()
        if n < 0:
            _refuse("sequences: offsets are one more than the sequences, at least one")
        pe = pb + size
    return B.Sequences(n, pb, pe, size, zero_others) if n else B.Sequences(0, None, None, 0, zero_others), n


def _activation(name):
    if not isinstance(name, str) or name not in ACTIVATIONS:
        _refuse("activation %r: none and tanh are taken" % (name,))
    return ACTIVATIONS[name]


def gated_scan(gate, cand, sequences=None, *, h0=None, activation="none", last=False, carry=False, out=None):
    """h_t = (1 - z_t) h_{t-1} + z_t act(cand_t), z = sigmoid(gate), along every sequence: (h, last, carry).

    sequences: None (one sequence of all rows), n + 1 offsets, or a pair (begin, end), int32 or int64 on the GPU; rows of no sequence
    are left as they were in `out`, and zeros where the call makes h.  h0: the states in front of the first rows, (n, features)
    float32, None = zeros.  last=True: the states behind the last rows, (n, features) float32, else None.  carry=True: what
    gated_scan_backward starts from, else None."""
    pg, sg = _rows("gate", gate)
    rows, hidden = shape = gate.shape
    pc, sc = _rows("cand", cand, gate, shape=shape)
    act = _activation(activation)
    seq, n = _sequences(sequences, gate, out is None)
    h = _new(gate) if out is None else out
    ph, sh = _rows("out", h, gate, shape=shape)
    p0 = _floats("h0", h0, gate, n, hidden)
    dtype = DTYPES[gate.dtype]
    end = torch.empty((n, hidden), dtype=torch.float32, device=gate.device) if last else None
    car = torch.empty((_size("amp_gated_scan_carry", dtype, rows, hidden), hidden), dtype=torch.float32, device=gate.device) if carry else None
    ws, nb = _workspace("amp_gated_scan_workspace", gate)
    _call(gate, "amp_gated_scan_forward", dtype, act, rows, hidden, pg, sg, pc, sc, ct.byref(seq), p0, ph, sh, _ptr(end), _ptr(car), _ptr(ws), nb)
    if out is not None:
        _written((out,))
    return h, end, car


def gated_scan_backward(dh, gate, cand, carry, sequences=None, *, h0=None, dlast=None, activation="none", out=None):
    """(dgate, dcand, dh0) from the gradient of h (and of last: dlast), the inputs and the carry of
    gated_scan(.., carry=True).  out: a pair of tensors for dgate and dcand, in which rows of no sequence are left as they were; where
    the call makes them, the gradients of those rows are zeros."""
    pg, sg = _rows("gate", gate)
    rows, hidden = shape = gate.shape
    pc, sc = _rows("cand", cand, gate, shape=shape)
    pd, sd = _rows("dh", dh, gate, shape=shape)
    act = _activation(activation)
    seq, n = _sequences(sequences, gate, out is None)
    if out is not None and not (isinstance(out, (tuple, list)) and len(out) == 2):
        _refuse("out is not a pair of tensors")
    dgate, dcand = out if out is not None else (_new(gate), _new(gate))
    po, so = _rows("dgate", dgate, gate, shape=shape)
    pq, sq = _rows("dcand", dcand, gate, shape=shape)
    dtype = DTYPES[gate.dtype]
    if carry is None:
        _refuse("carry is needed")
    pk = _floats("carry", carry, gate, _size("amp_gated_scan_carry", dtype, rows, hidden), hidden)
    p0, pl = _floats("h0", h0, gate, n, hidden), _floats("dlast", dlast, gate, n, hidden)
    dh0 = torch.empty((n, hidden), dtype=torch.float32, device=gate.device)
    ws, nb = _workspace("amp_gated_scan_workspace", gate)
    _call(gate, "amp_gated_scan_backward", dtype, act, rows, hidden, pd, sd, pl, pg, sg, pc, sc, ct.byref(seq), p0, pk, po, so, pq, sq,
          dh0.data_ptr(), _ptr(ws), nb)
    if out is not None:
        _written((dgate, dcand))
    return dgate, dcand, dh0


_FLOAT_ROWS = (torch.float32,)


def gated_scan_step(gate, cand, state, *, activation="none", out=None):
    """One row of every sequence: state (rows, features; float32, features next to each other) becomes
    (1 - z) state + z act(cand), in place; returns h, its rounded copy."""
    pg, sg = _rows("gate", gate)
    rows, hidden = shape = gate.shape
    pc, sc = _rows("cand", cand, gate, shape=shape)
    ps, ss = _rows("state", state, gate, _FLOAT_ROWS, shape)
    h = _new(gate) if out is None else out
    ph, sh = _rows("out", h, gate, shape=shape)
    _call(gate, "amp_gated_scan_step", DTYPES[gate.dtype], _activation(activation), rows, hidden, pg, sg, pc, sc, ps, ss, ph, sh)
    _written((state,) if out is None else (state, out))
    return h


# ------------------------------------------------------------------ distillation
def distill_loss(logits, teacher, index, temperature=1.0, weight=None, *, grad=True, out=None):
    """(loss, dlogits): per row weight * T^2 * KL(softmax(teacher / T) || softmax(logits / T)) over the teacher's top entries (teacher:
    their logits, index: their classes, both (rows, top); an entry with a class outside the row or a logit of -infinity is left out),
    and the gradient of the losses' sum by the logits, in their type (None without grad).  weight: a float per row; rows of weight
    0 are left out.  out: a tensor for dlogits (may be logits)."""
    px, sx = _rows("logits", logits)
    rows, classes = shape = logits.shape
    if not isinstance(teacher, torch.Tensor) or teacher.dim() != 2:
        _refuse("teacher is not a 2-D tensor")
    if teacher.dtype not in DTYPES:
        _refuse("teacher is of type %s" % (teacher.dtype,))
    top = teacher.size(1)
    pt, st = _rows("teacher", teacher, logits, (teacher.dtype,), (rows, top))
    pi, si = _rows("index", index, logits, _INDEX, (rows, top))
    pw = _floats("weight", weight, logits, rows)
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    dlogits, pd, sd = None, None, 0
    if grad:
        dlogits = _new(logits) if out is None else out
        pd, sd = _rows("out", dlogits, logits, shape=shape)
    elif out is not None:
        _refuse("out without grad")
    ws, nb = _workspace("amp_distill_workspace", logits)
    _call(logits, "amp_distill_loss", DTYPES[logits.dtype], rows, classes, px, sx, top, DTYPES[teacher.dtype], pt, st, pi, _INDEX[index.dtype],
          si, temperature, pw, loss.data_ptr(), pd, sd, _ptr(ws), nb)
    if out is not None:
        _written((out,))
    return loss, dlogits
