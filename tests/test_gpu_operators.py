"""GPU: the operators on whole arrays against their formulas in 64 bits, element by element, within the bounds that ops_reference
derives from 32-bit arithmetic; and what they do with strides, rows of no sequence and values that are no numbers."""
import math

import pytest
import torch

import ops_reference as ref
from paper_1705_09786_amd import binding as B
from paper_1705_09786_amd import operators as ops

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAN, INF = float("nan"), float("inf")


def rand(*shape, seed=0, dtype=torch.float32, scale=1.0, shift=0.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * scale + shift).to(dtype)


def dev(*tensors):
    out = [t if t is None else t.cuda() for t in tensors]
    return out if len(out) > 1 else out[0]


def strided(t, stride, offset):
    """The same rows on the GPU, `stride` elements apart from element `offset` on, filler of NaN between them; and the filler's buffer."""
    rows, cols = t.shape
    buf = torch.full((offset + rows * stride + 64,), NAN, dtype=t.dtype, device="cuda")
    view = buf.as_strided((rows, cols), (stride, 1), offset)
    view.copy_(t)
    return view, buf


def holes(buf, view):
    """The filler around a view."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return buf[keep]


def same_bits(a, b):
    kind = {4: torch.int32, 2: torch.int16, 8: torch.int64}[a.element_size()]
    return a.shape == b.shape and a.dtype == b.dtype and torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


# ------------------------------------------------------------------ layer norm
NORM_SIZES = [(1, 1), (3, 2), (5, 37), (1, 128), (300, 150), (7, 1000), (64, 1024), (2, 4097), (130, 2048), (3, 11111), (2, 16384), (2, 40001),
              (2, 70000), (1, 131073)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_norm(dtype, rows, cols):
    x = rand(rows, cols, seed=1, dtype=dtype, scale=1.5, shift=0.7)
    w, b, dy = rand(cols, seed=2, scale=0.2, shift=1.0), rand(cols, seed=3), rand(rows, cols, seed=4, dtype=dtype)
    y, mean, rstd = ops.layer_norm(*dev(x, w, b), 1e-5, stats=True)
    ry, rm, rr = ref.norm(x, w, b, 1e-5)
    ref.check("y", y, ry)
    ref.check("mean", mean, rm)
    ref.check("rstd", rstd, rr)
    assert same_bits(y, ops.layer_norm(*dev(x, w, b), 1e-5))
    dx, dw, db = ops.layer_norm_backward(*dev(dy, x, w), mean, rstd)
    rx, rw, rb = ref.norm_backward(dy, x, w, mean.cpu(), rstd.cpu())
    ref.check("dx", dx, rx)
    ref.check("dweight", dw, rw)
    ref.check("dbias", db, rb)
    again = ops.layer_norm_backward(*dev(dy, x, w), mean, rstd)
    assert all(same_bits(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("rows,cols", [(20000, 24), (4000, 150), (2100, 2500)])
def test_norm_many_rows(rows, cols):
    x, w, dy = rand(rows, cols, seed=1, dtype=torch.bfloat16), rand(cols, seed=2), rand(rows, cols, seed=4, dtype=torch.bfloat16)
    y, mean, rstd = ops.layer_norm(*dev(x, w), stats=True)
    ref.check("y", y, ref.norm(x, w, None, 1e-5)[0])
    for name, got, want in zip(("dx", "dweight", "dbias"), ops.layer_norm_backward(*dev(dy, x, w), mean, rstd),
                               ref.norm_backward(dy, x, w, mean.cpu(), rstd.cpu())):
        ref.check(name, got, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols,stride,offset", [(150, 151, 1), (37, 64, 3), (2048, 2049, 5), (11111, 11113, 1)])
def test_norm_strides(dtype, cols, stride, offset):
    rows = 9
    x, dy, w = rand(rows, cols, seed=1, dtype=dtype), rand(rows, cols, seed=4, dtype=dtype), rand(cols, seed=2)
    (vx, _), (vd, _) = strided(x, stride, offset), strided(dy, stride + 2, offset + 1)
    vy, by = strided(torch.zeros_like(x), stride + 1, offset)
    y, mean, rstd = ops.layer_norm(vx, w.cuda(), None, stats=True, out=vy)
    assert y is vy and holes(by, vy).isnan().all()
    ref.check("y", y, ref.norm(x, w, None, 1e-5)[0])
    vo, bo = strided(torch.zeros_like(x), stride + 3, offset)
    dx, dw, _ = ops.layer_norm_backward(vd, vx, w.cuda(), mean, rstd, out=vo)
    assert holes(bo, vo).isnan().all()
    want = ref.norm_backward(dy, x, w, mean.cpu(), rstd.cpu())
    ref.check("dx", dx, want[0])
    ref.check("dweight", dw, want[1])


def test_norm_in_place_and_repeated_rows():
    x, w, dy = rand(33, 600, seed=1), rand(600, seed=2), rand(33, 600, seed=3)
    y, mean, rstd = ops.layer_norm(*dev(x, w), stats=True)
    z = x.cuda()
    assert ops.layer_norm(z, w.cuda(), out=z) is z and same_bits(z, y)
    dx, dw, db = ops.layer_norm_backward(*dev(dy, x, w), mean, rstd)
    for place in (0, 1):
        a = list(dev(dy, x))
        got = ops.layer_norm_backward(*a, w.cuda(), mean, rstd, out=a[place])
        assert got[0] is a[place] and all(same_bits(p, q) for p, q in zip(got, (dx, dw, db)))
    one = rand(1, 600, seed=5)   # one gradient for every row
    got = ops.layer_norm_backward(one.cuda().expand(33, 600), x.cuda(), w.cuda(), mean, rstd)
    for g, want in zip(got, ops.layer_norm_backward(one.cuda().repeat(33, 1), x.cuda(), w.cuda(), mean, rstd)):
        assert same_bits(g, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(700, 37), (700, 151), (700, 1021), (30, 2049), (30, 11111), (5, 40001), (3, 70003)])
def test_norm_in_place_at_odd_sizes(dtype, rows, cols):
    """Rows whose last group reaches back over elements that another thread writes."""
    x, dy, w = dev(rand(rows, cols, seed=15, dtype=dtype), rand(rows, cols, seed=16, dtype=dtype), rand(cols, seed=17, shift=1.0))
    y, mean, rstd = ops.layer_norm(x, w, stats=True)
    z = x.clone()
    assert same_bits(ops.layer_norm(z, w, out=z), y)
    want = ops.layer_norm_backward(dy, x, w, mean, rstd)
    for place in (0, 1):
        args = [dy.clone(), x.clone()]
        got = ops.layer_norm_backward(*args, w, mean, rstd, out=args[place])
        assert all(same_bits(p, q) for p, q in zip(got, want))


def test_norm_without_rows_and_plain_weights():
    x = torch.empty(0, 40, device="cuda")
    y, mean, rstd = ops.layer_norm(x, stats=True)
    dx, dw, db = ops.layer_norm_backward(x, x, None, mean, rstd)
    assert y.shape == dx.shape == (0, 40) and not dw.any() and not db.any()
    x, dy = rand(6, 77, seed=1), rand(6, 77, seed=2)
    y, mean, rstd = ops.layer_norm(x.cuda(), eps=0.0, stats=True)
    ref.check("y", y, ref.norm(x, None, None, 0.0)[0])
    ref.check("dx", ops.layer_norm_backward(*dev(dy, x), None, mean, rstd)[0], ref.norm_backward(dy, x, None, mean.cpu(), rstd.cpu())[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_far_from_zero_and_constant_rows(dtype):
    """A mean far above the deviations costs no more than the mean's own rounding; rows without any have y = bias."""
    x = rand(4, 300, seed=1, scale=0.5, shift=200.0).to(dtype)
    x[1] = 3.0
    b = rand(300, seed=2)
    y, mean, rstd = ops.layer_norm(x.cuda(), None, b.cuda(), 1e-3, stats=True)
    want = ref.norm(x, None, b, 1e-3)
    ref.check("y", y, want[0])
    ref.check("mean", mean, want[1])
    ref.check("rstd", rstd, want[2])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 40), (8, 24), (129, 5), (20000, 24), (4099, 37), (4000, 150), (513, 1000), (3001, 1021), (37, 2048), (2100, 2500),
                                       (1037, 4099), (4097, 4096), (300, 11111), (2500, 8200), (17, 16400), (70, 20011), (600, 16400), (521, 33000)])
def test_norm_parameter_gradients_count_every_row_once(dtype, rows, cols):
    """Whole numbers and statistics that are powers of two: every sum is exact in 32 bits in whatever order (up to 20,000 terms of at
    most 3 * 8 * 2, in halves: below 2^24), so that a row that is lost, doubled or given another's statistics shows."""
    g = torch.Generator("cuda").manual_seed(rows + cols)
    x, dy = (torch.randint(-3, 4, (rows, cols), device="cuda", generator=g).to(dtype) for _ in range(2))
    mean = torch.randint(-5, 6, (rows,), device="cuda", generator=g).float()
    rstd = 2.0 ** torch.randint(-1, 2, (rows,), device="cuda", generator=g).float()
    for weight in (None, torch.ones(cols, device="cuda")):
        dx, dw, db = ops.layer_norm_backward(dy, x, weight, mean, rstd)
        n = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        assert torch.equal(dw.double(), (dy.double() * n).sum(0)) and torch.equal(db.double(), dy.double().sum(0))


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 16400), (torch.bfloat16, 33000)])
def test_norm_more_long_rows_than_workgroups(dtype, cols):
    """Rows that registers do not hold, more of them than a launch has workgroups: each as in a call of a few."""
    rows = 4096 + 70
    g = torch.Generator("cuda").manual_seed(7)
    x, dy = (torch.randn(rows, cols, device="cuda", generator=g).to(dtype) for _ in range(2))
    w, b = torch.randn(cols, device="cuda", generator=g), torch.randn(cols, device="cuda", generator=g)
    y, mean, rstd = ops.layer_norm(x, w, b, stats=True)
    dx = ops.layer_norm_backward(dy, x, w, mean, rstd)[0]
    for s in (slice(0, 5), slice(60, 100), slice(rows - 75, rows)):
        y2, mean2, rstd2 = ops.layer_norm(x[s], w, b, stats=True)
        assert same_bits(y[s], y2) and same_bits(mean[s], mean2) and same_bits(rstd[s], rstd2)
        assert same_bits(dx[s], ops.layer_norm_backward(dy[s], x[s], w, mean2, rstd2)[0])


@pytest.mark.parametrize("rows", [0, 2])
def test_norm_of_more_columns_than_a_launch_joins_in_one_line(rows):
    """The parameters' gradients of 2^26 columns and more; whole numbers, whose sums are exact in any order."""
    cols = (1 << 26) + 3
    x, dy = (torch.randint(-3, 4, (rows, cols), device="cuda", generator=torch.Generator("cuda").manual_seed(k)).bfloat16() for k in range(2))
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dx, dw, db = ops.layer_norm_backward(dy, x, None, mean, rstd)
    assert torch.equal(dw, (dy.float() * x.float()).sum(0)) and torch.equal(db, dy.float().sum(0))


@pytest.mark.parametrize("cols", [37, 2048, 11111])
def test_norm_keeps_other_rows_apart(cols):
    x, dy = rand(8, cols, seed=1), rand(8, cols, seed=2)
    y, mean, rstd = ops.layer_norm(x.cuda(), stats=True)
    dx = ops.layer_norm_backward(*dev(dy, x), None, mean, rstd)[0]
    bad = x.clone()
    bad[3, cols // 2], bad[5, 0] = NAN, INF
    y2, m2, r2 = ops.layer_norm(bad.cuda(), stats=True)
    dx2 = ops.layer_norm_backward(*dev(dy, bad), None, m2, r2)[0]
    rest = [0, 1, 2, 4, 6, 7]
    assert y2[3].isnan().all() and y2[5].isnan().any() and same_bits(y2[rest], y[rest]) and same_bits(dx2[rest], dx[rest])


# ------------------------------------------------------------------ gated linear recurrence
def packed(lengths, at=0):
    o = [at]
    for n in lengths:
        o.append(o[-1] + n)
    return o


SCANS = [  # rows, hidden, sequences
    (1, 1, None), (5, 37, None), (127, 64, None), (128, 65, None), (129, 8, None), (1000, 150, None), (2050, 3, None), (700, 520, None),
    (300, 70, packed([1] * 300)), (600, 33, packed([0, 3, 0, 0, 250, 7, 130, 1, 0, 128, 81, 0])), (513, 128, packed([128, 128, 256, 1])),
    (900, 20, packed([5, 300, 9], 100)),                                                      # rows in front and behind
    (640, 96, ([0, 128, 256, 300, 512], [100, 128, 299, 512, 630])),                          # padded rows and an empty one
    (400, 40, packed([2, 5, 1, 0, 4] * 30)),
    (64, 16, packed([0, 0, 0])),                                                              # rows, and none in a sequence
    (2600, 9, packed([1] * 700 + [0] * 600 + [900, 1000])),                                   # more sequences than a tile has threads
    (1400, 1090, packed([700, 1, 0, 699])), (1700, 12, packed([1650, 50])),                   # wide and narrow: tiles alone and in groups
]


def sequences_of(s, kind):
    if s is None or isinstance(s, list):
        return s if s is None else torch.tensor(s, dtype=kind)
    return tuple(torch.tensor(v, dtype=kind) for v in s)


def on_gpu(seq):
    return seq if seq is None else tuple(t.cuda() for t in seq) if isinstance(seq, tuple) else seq.cuda()


def scan_inputs(rows, hidden, n, dtype, seed=0):
    # features that forget at once beside some that keep for hundreds of rows
    reach = torch.linspace(-6.0, 2.0, hidden)
    return ((rand(rows, hidden, seed=seed) + reach).to(dtype), rand(rows, hidden, seed=seed + 1, dtype=dtype), rand(n, hidden, seed=seed + 2),
            rand(rows, hidden, seed=seed + 3, dtype=dtype), rand(n, hidden, seed=seed + 4))


def inside(seq, rows):
    m = torch.zeros(rows, dtype=torch.bool)
    for b, e in ref.spans(seq, rows):
        m[b:e] = True
    return m


@pytest.mark.parametrize("dtype,tanh,kind", [(torch.float32, True, torch.int64), (torch.float32, False, torch.int32),
                                             (torch.bfloat16, False, torch.int64), (torch.float16, True, torch.int32)])
@pytest.mark.parametrize("case", range(len(SCANS)))
def test_scan(case, dtype, tanh, kind):
    rows, hidden, s = SCANS[case]
    seq = sequences_of(s, kind)
    n = len(ref.spans(seq, rows))
    gate, cand, h0, dh, dlast = scan_inputs(rows, hidden, n, dtype, seed=case)
    act, gseq = "tanh" if tanh else "none", on_gpu(seq)
    rh, rl, _ = ref.scan(gate, cand, seq, h0, tanh)
    rg, rc, r0 = ref.scan_backward(dh, dlast, gate, cand, seq, h0, tanh)
    m = inside(seq, rows)
    # rows of no sequence hold NaN: they are left as they were, and nothing of them reaches the others
    for t in (gate, cand, dh):
        t[~m] = NAN
    out = [torch.full((rows, hidden), 7.0, dtype=dtype, device="cuda") for _ in range(3)]
    h, last, carry = ops.gated_scan(*dev(gate, cand), gseq, h0=h0.cuda(), activation=act, last=True, carry=True, out=out[0])
    ref.check("h", h[m], (rh[0][m], rh[1][m]))
    ref.check("last", last, rl)
    dgate, dcand, dh0 = ops.gated_scan_backward(*dev(dh, gate, cand), carry, gseq, h0=h0.cuda(), dlast=dlast.cuda(), activation=act, out=out[1:])
    ref.check("dgate", dgate[m], (rg[0][m], rg[1][m]))
    ref.check("dcand", dcand[m], (rc[0][m], rc[1][m]))
    ref.check("dh0", dh0, r0)
    assert all((o[~m] == 7.0).all() for o in out)
    # the same bits again, and without what is not asked for
    h2, none, _ = ops.gated_scan(*dev(gate, cand), gseq, h0=h0.cuda(), activation=act)
    assert none is None and same_bits(h2[m], h[m])
    again = ops.gated_scan_backward(*dev(dh, gate, cand), carry, gseq, h0=h0.cuda(), dlast=dlast.cuda(), activation=act)
    assert all(same_bits(p[m], q[m]) for p, q in zip(again[:2], (dgate, dcand))) and same_bits(again[2], dh0)


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_without_states(dtype):
    rows, hidden = 300, 100
    gate, cand, _, dh, _ = scan_inputs(rows, hidden, 1, dtype)
    h, last, carry = ops.gated_scan(*dev(gate, cand), last=True, carry=True)
    rh, rl, _ = ref.scan(gate, cand, None, None, False)
    ref.check("h", h, rh)
    ref.check("last", last, rl)
    rg, rc, r0 = ref.scan_backward(dh, None, gate, cand, None, None, False)
    for name, got, want in zip(("dgate", "dcand", "dh0"), ops.gated_scan_backward(*dev(dh, gate, cand), carry), (rg, rc, r0)):
        ref.check(name, got, want)


def test_scan_no_rows_and_no_sequences():
    x = torch.empty(0, 24, device="cuda")
    h0, dlast = rand(3, 24).cuda(), rand(3, 24, seed=1).cuda()
    seq = torch.zeros(4, dtype=torch.int32, device="cuda")
    h, last, carry = ops.gated_scan(x, x, seq, h0=h0, last=True, carry=True)
    assert same_bits(last, h0)
    dg, dc, dh0 = ops.gated_scan_backward(x, x, x, carry, seq, h0=h0, dlast=dlast)
    assert dg.shape == (0, 24) and same_bits(dh0, dlast)
    assert not ops.gated_scan(x, x, last=True)[1].any()
    y = torch.full((5, 24), 3.0, device="cuda")
    h, last, carry = ops.gated_scan(y, y, seq[:1], last=True, carry=True, out=y.clone())
    assert (h == 3.0).all() and last.shape == (0, 24)
    assert ops.gated_scan_backward(y, y, y, carry, seq[:1])[2].shape == (0, 24)


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_long(dtype):
    """One sequence over many tiles, features that keep nearly everything and nearly nothing; long enough that every tile waits."""
    rows, hidden = 20011, 70
    gate, cand, h0, dh, dlast = scan_inputs(rows, hidden, 1, dtype, seed=5)
    gate[:, 3] = -INF   # keeps h0 for good
    gate[:, 4] = INF    # the candidate alone
    h, last, carry = ops.gated_scan(*dev(gate, cand), h0=h0.cuda(), last=True, carry=True)
    z, keep = torch.sigmoid(gate.double()), torch.sigmoid(-gate.double())
    x, hs = h0[0].double(), []
    for t in range(rows):
        x = keep[t] * x + z[t] * cand[t].double()
        hs.append(x)
    want = torch.stack(hs)
    # keep and z are off by some 2^-23 relative, which a feature that keeps for 1 / z rows adds up as often: (1 / z) 2^-21 of states
    # of size 1 .. 5, with 1 / z up to 400 (e^6): 2^-21 * 400 * 5 < 1e-3
    assert (h.cpu().double() - want).abs().max() <= 1e-3 + torch.finfo(dtype).eps / 2 * want.abs().max()
    assert (last.cpu().double()[0] - want[-1]).abs().max() <= 1e-3
    assert torch.equal(last.cpu()[0, 3], h0[0, 3]) and torch.equal(h.cpu()[:, 4], cand[:, 4])
    dg, dc, dh0 = ops.gated_scan_backward(*dev(dh, gate, cand), carry, h0=h0.cuda(), dlast=dlast.cuda())
    g, back = torch.empty(rows, hidden, dtype=torch.float64), dlast[0].double()
    for t in range(rows - 1, -1, -1):
        g[t] = dh[t].double() + back
        back = keep[t] * g[t]
    before = torch.cat([h0.double(), want[:-1]])
    far = 2.0 ** -21 * 400 * g.abs().max()
    for got, ex in ((dg, g * z * keep * (cand.double() - before)), (dc, g * z)):
        assert (got.cpu().double() - ex).abs().max() <= far + torch.finfo(dtype).eps / 2 * ex.abs().max()
    assert (dh0.cpu().double()[0] - back).abs().max() <= far


@pytest.mark.parametrize("dtype", TYPES)
def test_scan_strides(dtype):
    """Gate and candidate as the halves of one projection, gradients into the halves of another, odd offsets, repeated gradient rows."""
    rows, hidden = 400, 75
    gate, cand, h0, dh, dlast = scan_inputs(rows, hidden, 2, dtype)
    seq = torch.tensor([0, 150, 400]).cuda()
    h, last, carry = ops.gated_scan(*dev(gate, cand), seq, h0=h0.cuda(), last=True, carry=True)
    both, _ = strided(torch.cat([gate, cand], 1), 2 * hidden + 3, 1)
    vg, vc = both[:, :hidden], both[:, hidden:]
    vo, bo = strided(torch.zeros_like(gate), hidden + 6, 5)
    h2, last2, carry2 = ops.gated_scan(vg, vc, seq, h0=h0.cuda(), last=True, carry=True, out=vo)
    assert same_bits(h2, h) and same_bits(last2, last) and holes(bo, vo).isnan().all()
    dg, dc, d0 = ops.gated_scan_backward(*dev(dh, gate, cand), carry, seq, h0=h0.cuda(), dlast=dlast.cuda())
    vd, bd = strided(torch.zeros(rows, 2 * hidden, dtype=dtype), 2 * hidden + 1, 3)
    g2 = ops.gated_scan_backward(strided(dh, hidden + 1, 1)[0], vg, vc, carry2, seq, h0=h0.cuda(), dlast=dlast.cuda(),
                                 out=(vd[:, :hidden], vd[:, hidden:]))
    assert same_bits(g2[0], dg) and same_bits(g2[1], dc) and same_bits(g2[2], d0) and holes(bd, vd).isnan().all()
    one = dh[:1].cuda()
    a = ops.gated_scan_backward(one.expand(rows, hidden), *dev(gate, cand), carry, seq, h0=h0.cuda())
    b = ops.gated_scan_backward(one.repeat(rows, 1), *dev(gate, cand), carry, seq, h0=h0.cuda())
    assert all(same_bits(p, q) for p, q in zip(a, b))


def test_scan_keeps_other_sequences_apart():
    """NaN and infinities of one sequence, its states and its gradients reach no other, wherever tiles begin."""
    rows, hidden, lens = 900, 40, [100, 28, 2, 300, 200, 270]
    seq = torch.tensor(packed(lens)).cuda()
    gate, cand, h0, dh, dlast = scan_inputs(rows, hidden, len(lens), torch.float32)

    def run(gate, cand, h0, dh, dlast):
        h, last, carry = ops.gated_scan(*dev(gate, cand), seq, h0=h0.cuda(), last=True, carry=True)
        return (h, last) + ops.gated_scan_backward(*dev(dh, gate, cand), carry, seq, h0=h0.cuda(), dlast=dlast.cuda())
    want = run(gate, cand, h0, dh, dlast)
    gate, cand, h0, dh, dlast = (t.clone() for t in (gate, cand, h0, dh, dlast))
    gate[140, 3], cand[150, 4], cand[160, 5], dh[200, 6], gate[100, :] = NAN, INF, NAN, NAN, NAN
    h0[3], dlast[3] = NAN, -INF
    got = run(gate, cand, h0, dh, dlast)
    good = torch.ones(rows, dtype=torch.bool)
    good[130:430], good[100:128] = False, False
    seqs = torch.tensor([0, 2, 4, 5])
    for k in (0, 2, 3):
        assert same_bits(got[k][good], want[k][good])
    for k in (1, 4):
        assert same_bits(got[k][seqs], want[k][seqs])
    assert got[0][430 - 1].isnan().all()   # and inside a sequence a NaN stays one


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,hidden,s", [(300, 2, [0, 0, 5, 5, 200]), (128, 37, [3, 100]), (1000, 130, ([0, 128, 256, 300, 512], [100, 128, 299, 512, 630])),
                                           (5, 24, [0]), (700, 70, [7]), (640, 64, [640, 640]), (3000, 20, [1, 2999])])
def test_scan_makes_zeros_in_rows_of_no_sequence(dtype, rows, hidden, s):
    """h and the gradients that a call makes itself: zeros in padding, whatever it and the memory held."""
    seq = on_gpu(sequences_of(s, torch.int64))
    n = len(s) - 1 if isinstance(s, list) else len(s[0])
    gate, cand, h0, dh, dlast = scan_inputs(rows, hidden, n, dtype, seed=41)
    m = inside(sequences_of(s, torch.int64), rows)
    for t in (gate, cand, dh):
        t[~m] = NAN
    dirt = [torch.full((rows, hidden), NAN, dtype=dtype, device="cuda") for _ in range(8)]
    out = [t.clone() for t in dirt[:3]]
    del dirt   # what the calls are given next
    h, last, carry = ops.gated_scan(*dev(gate, cand), seq, h0=h0.cuda(), last=True, carry=True)
    dgate, dcand, dh0 = ops.gated_scan_backward(*dev(dh, gate, cand), carry, seq, h0=h0.cuda(), dlast=dlast.cuda())
    for t in (h, dgate, dcand):
        assert t.shape == (rows, hidden) and not t[~m].any() and not t[m].isnan().any()
    # and in tensors of the caller's they are left alone, the others having the same bits
    h2, last2, carry2 = ops.gated_scan(*dev(gate, cand), seq, h0=h0.cuda(), last=True, carry=True, out=out[0])
    g2 = ops.gated_scan_backward(*dev(dh, gate, cand), carry, seq, h0=h0.cuda(), dlast=dlast.cuda(), out=out[1:])
    for p, q in zip((h, dgate, dcand), (h2, g2[0], g2[1])):
        assert q[~m].isnan().all() and same_bits(p[m], q[m])
    assert same_bits(last, last2) and same_bits(dh0, g2[2])


@pytest.mark.parametrize("lens", [[1536], [300, 1236], [64] * 24])
@pytest.mark.parametrize("feature", [5, 64, 129])
def test_scan_keeps_other_features_apart(feature, lens):
    """A gate that is no number, in every tile of three groups of them in turn: the other features keep their bits, its own the states in
    front of it and those of other sequences."""
    rows, hidden = 1536, 130
    o = packed(lens)
    seq = torch.tensor(o).cuda()
    gate, cand, h0, dh, dlast = dev(*scan_inputs(rows, hidden, len(lens), torch.float32, seed=31))

    def run(gate):
        h, last, carry = ops.gated_scan(gate, cand, seq, h0=h0, last=True, carry=True)
        return (h, last) + ops.gated_scan_backward(dh, gate, cand, carry, seq, h0=h0, dlast=dlast)
    want = run(gate)
    rest = torch.arange(hidden) != feature
    for r in range(7, rows, 128):
        bad = gate.clone()
        bad[r, feature] = NAN
        got = run(bad)
        assert all(same_bits(p[:, rest], q[:, rest]) for p, q in zip(got, want)), r
        s = next(k for k in range(len(lens)) if o[k] <= r < o[k + 1])
        hit = torch.zeros(rows, dtype=torch.bool)
        hit[r:o[s + 1]] = True
        assert got[0][hit, feature].isnan().all() and same_bits(got[0][~hit, feature], want[0][~hit, feature]), r
        other = torch.arange(len(lens)) != s
        assert got[1][s, feature].isnan() and got[4][s, feature].isnan(), r
        assert same_bits(got[1][other, feature], want[1][other, feature]) and same_bits(got[4][other, feature], want[4][other, feature]), r


def test_scan_bounds_outside_the_rows():
    """Bounds in front of the first row and behind the last are the nearest row's; descending ones touch nothing outside the arrays."""
    rows, hidden = 300, 33
    gate, cand, h0, _, _ = scan_inputs(rows, hidden, 3, torch.float32)
    h, last, _ = ops.gated_scan(*dev(gate, cand), torch.tensor([0, 100, 200, 300]).cuda(), h0=h0.cuda(), last=True)
    for kind in (torch.int32, torch.int64):
        h2, last2, _ = ops.gated_scan(*dev(gate, cand), torch.tensor([-50, 100, 200, 2 ** 31 - 1], dtype=kind).cuda(), h0=h0.cuda(), last=True)
        assert same_bits(h2, h) and same_bits(last2, last)
    ops.gated_scan(*dev(gate, cand), torch.tensor([250, 10, 290, -4]).cuda(), h0=h0.cuda(), last=True)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tanh", [False, True])
@pytest.mark.parametrize("rows,hidden", [(1, 1), (3, 37), (48, 2048), (130, 515)])
def test_scan_step(dtype, tanh, rows, hidden):
    gate, cand, state, _, _ = scan_inputs(rows, hidden, rows, dtype)
    pool, buf = strided(state, hidden + 5, 3)
    h = ops.gated_scan_step(*dev(gate, cand), pool, activation="tanh" if tanh else "none")
    want = ref.step(gate, cand, state, tanh)
    ref.check("state", pool, want)
    ref.check("h", h, want)
    assert holes(buf, pool).isnan().all()


def test_scan_steps_are_the_scan():
    """Prefill by the scan, then single rows: the states of the whole sequence."""
    rows, hidden, n = 40, 96, 5
    gate, cand, h0, _, _ = scan_inputs(rows * n, hidden, n, torch.float32)
    seq = torch.arange(n + 1) * rows
    want, _, _ = ref.scan(gate, cand, seq, h0, True)
    cut = 31
    state = ops.gated_scan(*dev(gate, cand), (seq[:-1].cuda(), (seq[:-1] + cut).cuda()), h0=h0.cuda(), activation="tanh", last=True)[1]
    for t in range(cut, rows):
        at = seq[:-1] + t
        h = ops.gated_scan_step(gate[at].cuda(), cand[at].cuda(), state, activation="tanh")
        ref.check("h", h, (want[0][at], want[1][at] + 8 * rows))   # a rounded state between the rows: 8 more roundings a row


# ------------------------------------------------------------------ distillation
DISTILLS = [(1, 1, 1), (3, 2, 5), (5, 37, 4), (64, 1000, 16), (2, 20000, 16), (4, 50257, 33), (1, 131072, 128), (3, 160001, 7), (17, 4099, 300),
            (300, 640, 8), (2, 32000, 1024)]


def distill_inputs(rows, classes, top, dtype, seed=0, twice=True):
    x = rand(rows, classes, seed=seed, scale=2.0, dtype=dtype)
    g = torch.Generator().manual_seed(seed + 1)
    index = torch.randint(0, classes, (rows, top), generator=g) if twice else torch.argsort(torch.rand(rows, classes, generator=g), 1)[:, :top]
    return x, rand(rows, top, seed=seed + 2, scale=2.0), index


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,classes,top", DISTILLS)
def test_distill(dtype, rows, classes, top):
    x, t, i = distill_inputs(rows, classes, top, dtype)
    w = torch.linspace(0.5, 1.5, rows)
    for T in (1.0, 2.5):
        loss, grad = ops.distill_loss(*dev(x, t, i), T, w.cuda())
        rl, rg = ref.distill(x, t, i, T, w)
        ref.check("loss", loss, rl)
        ref.check("dlogits", grad, rg)
        alone, none = ops.distill_loss(*dev(x, t, i), T, w.cuda(), grad=False)
        assert none is None
        ref.check("loss alone", alone, rl)
        again = ops.distill_loss(*dev(x, t, i), T, w.cuda())
        assert same_bits(again[0], loss) and same_bits(again[1], grad)
        z = x.cuda()
        inplace = ops.distill_loss(z, *dev(t, i), T, w.cuda(), out=z)
        assert inplace[1] is z and same_bits(z, grad) and same_bits(inplace[0], loss)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [100, 20000, 140000])
def test_distill_entries_left_out(dtype, classes):
    """Unused entries, classes outside the row, the same class twice, masked students, rows of weight 0 full of NaN, and rows of no entry."""
    x, t, i = distill_inputs(8, classes, 6, dtype, twice=False)
    i[0, 2], t[0, 4] = -1, -INF
    i[1, 1], i[1, 3] = classes, -2 ** 40
    i[2, 5] = i[2, 0]
    i[3, :] = -1
    t[4, :] = -INF
    w = torch.ones(8)
    w[5] = 0.0
    x[6, ::3] = -INF
    x[7, ::2] = torch.finfo(dtype).min
    i[6], i[7] = torch.tensor([1, 2, 4, 5, 7, 8]), torch.tensor([1, 3, 5, 7, 9, 11])
    clean = x.clone()
    x[5] = NAN
    rl, rg = ref.distill(clean, t, i, 1.5, w)
    for index, teacher in ((i, t), (i.clamp(min=-7).int(), t), (i, t.bfloat16())):
        if teacher.dtype != t.dtype:
            rl, rg = ref.distill(clean, teacher, i, 1.5, w)
        loss, grad = ops.distill_loss(*dev(x, teacher, index), 1.5, w.cuda())
        ref.check("loss", loss, rl)
        ref.check("dlogits", grad, rg)
        assert not loss[3:6].any() and not grad[3:6].any()
        ref.check("loss alone", ops.distill_loss(*dev(x, teacher, index), 1.5, w.cuda(), grad=False)[0], rl)


@pytest.mark.parametrize("classes", [50, 30000, 140000])
def test_distill_values_that_are_no_numbers(classes):
    x, t, i = distill_inputs(6, classes, 4, torch.float32, twice=False)
    want = ops.distill_loss(*dev(x, t, i), 1.0)
    x[1, classes // 2], x[2, 7], t[3, 1] = NAN, INF, NAN
    x[4, i[4, 2]] = -INF   # the teacher has mass where the student has none
    loss, grad = ops.distill_loss(*dev(x, t, i), 1.0)
    for r in (1, 2, 3):
        assert loss[r].isnan() and grad[r].isnan().any()
    assert loss[4] == INF and not grad[4].isnan().any()
    for r in (0, 5):
        assert same_bits(loss[r], want[0][r]) and same_bits(grad[r], want[1][r])
    # every logit the type's lowest: a student that knows nothing
    x = torch.full((2, classes), torch.finfo(torch.float32).min)
    loss, grad = ops.distill_loss(*dev(x, t[:2], i[:2]), 1.0)
    rl, rg = ref.distill(torch.zeros(2, classes), t[:2], i[:2], 1.0, None)
    ref.check("loss", loss, rl)
    ref.check("dlogits", grad, rg)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [1001, 50001])
def test_distill_strides(dtype, classes):
    rows, top = 5, 9
    x, t, i = distill_inputs(rows, classes, top, dtype)
    loss, grad = ops.distill_loss(*dev(x, t, i), 2.0)
    vx, _ = strided(x, classes + 4, 3)
    vt, _ = strided(t, top + 2, 1)
    vi = torch.full((rows, top + 3), -1, device="cuda")
    vi[:, 2:2 + top] = i.cuda()
    vo, bo = strided(torch.zeros_like(x), classes + 7, 1)
    loss2, grad2 = ops.distill_loss(vx, vt, vi[:, 2:2 + top], 2.0, out=vo)
    assert holes(bo, vo).isnan().all()
    rl, rg = ref.distill(x, t, i, 2.0, None)
    ref.check("loss", loss2, rl)
    ref.check("dlogits", grad2, rg)
    shared, _ = ops.distill_loss(x.cuda(), t[:1].cuda().expand(rows, top), i[:1].cuda().expand(rows, top), 2.0)
    ref.check("one teacher for all", shared, ref.distill(x, t[:1].expand(rows, top), i[:1].expand(rows, top), 2.0, None)[0])


# ------------------------------------------------------------------ refusals of the wrappers
def test_wrappers_refuse():
    x, w = torch.zeros(4, 8, device="cuda"), torch.ones(8, device="cuda")
    i = torch.zeros(4, 3, dtype=torch.int64, device="cuda")
    bad = [lambda: ops.layer_norm(x.double()), lambda: ops.layer_norm(x, w.bfloat16()), lambda: ops.layer_norm(x, w[:7]),
           lambda: ops.layer_norm(x, w.cpu()), lambda: ops.layer_norm(x.t()), lambda: ops.layer_norm(x, eps=-1.0),
           lambda: ops.layer_norm(x, out=torch.zeros(4, 7, device="cuda")), lambda: ops.layer_norm(x, out=x.half()),
           lambda: ops.layer_norm(x, out=x[:1].expand(4, 8)), lambda: ops.layer_norm_backward(x, x, w, None, None),
           lambda: ops.layer_norm_backward(x.half(), x, w, x[:, 0].contiguous(), x[:, 0].contiguous()),
           lambda: ops.gated_scan(x, x[:3]), lambda: ops.gated_scan(x, x.half()), lambda: ops.gated_scan(x, x, activation="relu"),
           lambda: ops.gated_scan(x, x, torch.zeros(3, device="cuda")), lambda: ops.gated_scan(x, x, torch.zeros(3, dtype=torch.int64)),
           lambda: ops.gated_scan(x, x, i[0][:0]), lambda: ops.gated_scan(x, x, (i[0], i[0][:2])), lambda: ops.gated_scan(x, x, (i[0],)),
           lambda: ops.gated_scan(x, x, (i[0], i[0].int())), lambda: ops.gated_scan(x, x, i[0], h0=x), lambda: ops.gated_scan(x, x, out=x),
           lambda: ops.gated_scan_backward(x, x, x, None), lambda: ops.gated_scan_backward(x, x, x, x),
           lambda: ops.gated_scan_step(x, x, x.half()), lambda: ops.gated_scan_step(x, x, x[:1].expand(4, 8)),
           lambda: ops.gated_scan_step(x, x, x), lambda: ops.distill_loss(x, x[:, :3], i[:, :2]), lambda: ops.distill_loss(x, x[:, :3], i.float()),
           lambda: ops.distill_loss(x, x[:, :3], i, 0.0), lambda: ops.distill_loss(x, x[:, :0], i[:, :0]),
           lambda: ops.distill_loss(x, x[:, :3], i, 1.0, w), lambda: ops.distill_loss(x, x[:, :3].clone(), i, grad=False, out=x)]
    for k, call in enumerate(bad):
        with pytest.raises(B.AmpError):
            call()
            pytest.fail("call %d was taken" % k)


def test_wrappers_refuse_arguments_of_other_kinds():
    """What is no tensor, number or name where one is due is a refused call as well."""
    x, st = torch.zeros(4, 8, device="cuda"), torch.zeros(4, device="cuda")
    i, s = torch.zeros(4, 3, dtype=torch.int64, device="cuda"), torch.zeros(1, 8, device="cuda")
    for call in (lambda: ops.layer_norm(x, eps="1"), lambda: ops.layer_norm(x, eps=None), lambda: ops.layer_norm(x, eps=st),
                 lambda: ops.distill_loss(x, x[:, :3], i, st[0]), lambda: ops.distill_loss(x, x[:, :3], i, None),
                 lambda: ops.gated_scan(x, x, activation=None), lambda: ops.gated_scan(x, x, activation=[]), lambda: ops.gated_scan(x, x, out=3),
                 lambda: ops.gated_scan_backward(x, x, x, s, out=(x,)), lambda: ops.gated_scan_backward(x, x, x, s, out=torch.zeros(2, 4, 8, device="cuda")),
                 lambda: ops.gated_scan_backward(x, x, x, s, out=5), lambda: ops.gated_scan(x, x, 4), lambda: ops.layer_norm(x, 2.0)):
        with pytest.raises(B.AmpError) as e:
            call()
        assert e.value.code == B.AMP_EINVAL


def test_wrappers_and_autograd():
    """Whatever requires grad is refused in grad mode, each argument of each call; without it the calls run, also inside a Function."""
    def leaf(*shape):
        return torch.rand(*shape, device="cuda", requires_grad=True)
    x, w, st = torch.rand(4, 8, device="cuda"), torch.rand(8, device="cuda"), torch.rand(4, device="cuda")
    i = torch.zeros(4, 3, dtype=torch.int64, device="cuda")
    s, t = torch.rand(1, 8, device="cuda"), torch.rand(4, 3, device="cuda")
    calls = [lambda: ops.layer_norm(leaf(4, 8)), lambda: ops.layer_norm(x, leaf(8)), lambda: ops.layer_norm(x, w, leaf(8)),
             lambda: ops.layer_norm(x, out=leaf(4, 8)), lambda: ops.layer_norm_backward(leaf(4, 8), x, w, st, st),
             lambda: ops.layer_norm_backward(x, leaf(4, 8), w, st, st), lambda: ops.layer_norm_backward(x, x, leaf(8), st, st),
             lambda: ops.layer_norm_backward(x, x, w, leaf(4), st), lambda: ops.gated_scan(leaf(4, 8), x), lambda: ops.gated_scan(x, leaf(4, 8)),
             lambda: ops.gated_scan(x, x, h0=leaf(1, 8)), lambda: ops.gated_scan_backward(leaf(4, 8), x, x, s),
             lambda: ops.gated_scan_backward(x, x, leaf(4, 8), s), lambda: ops.gated_scan_backward(x, x, x, s, dlast=leaf(1, 8)),
             lambda: ops.gated_scan_step(x, leaf(4, 8), x.clone()), lambda: ops.gated_scan_step(x, x, leaf(4, 8)),
             lambda: ops.distill_loss(leaf(4, 8), t, i), lambda: ops.distill_loss(x, leaf(4, 3), i), lambda: ops.distill_loss(x, t, i, 1.0, leaf(4))]
    for k, call in enumerate(calls):
        with pytest.raises(B.AmpError, match="requires grad"):
            call()
            pytest.fail("call %d was taken" % k)
        with torch.no_grad():
            call()
    # a tensor that is written to counts as changed: torch's own backward pass then says that it cannot use it
    a, b, c = (torch.rand(4, 8, device="cuda") for _ in range(3))
    for write in (lambda: ops.layer_norm(x, out=a), lambda: ops.layer_norm_backward(x, x, w, st, st, out=a),
                  lambda: ops.gated_scan(x, x, out=a), lambda: ops.gated_scan_backward(x, x, x, s, out=(b, a)),
                  lambda: ops.gated_scan_step(x, x, a), lambda: ops.gated_scan_step(x, x, c, out=a), lambda: ops.distill_loss(x, t, i, out=a)):
        p = leaf(4, 8)
        y = (p * a).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, mean, rstd = ops.layer_norm(x, w, b, stats=True)
            ctx.save_for_backward(x, w, mean, rstd)
            return y

        @staticmethod
        def backward(ctx, dy):
            return ops.layer_norm_backward(dy, *ctx.saved_tensors)
    p, q, r, dy = leaf(5, 40), leaf(40), leaf(40), torch.rand(5, 40, device="cuda")
    Norm.apply(p, q, r).backward(dy)
    with torch.no_grad():
        y, mean, rstd = ops.layer_norm(p, q, r, stats=True)
        want = ops.layer_norm_backward(dy, p, q, mean, rstd)
    assert all(same_bits(g.grad, v) for g, v in zip((p, q, r), want))
    with torch.inference_mode():
        z = torch.rand(4, 8, device="cuda")
        ops.gated_scan_step(z, z, z.clone(), out=torch.empty_like(z))


# ------------------------------------------------------------------ long and many
def test_offsets_past_32_bits():
    """Rows so far apart that the last ones begin behind 2^32 elements: the bits of the same rows next to each other."""
    rows, cols, step = 1100, 40, 4000000
    big = torch.empty(rows * step, dtype=torch.bfloat16, device="cuda")
    at = [big.as_strided((rows, cols), (step, 1), 64 * k) for k in range(5)]
    x = [dev(rand(rows, cols, seed=200 + k, dtype=torch.bfloat16)) for k in range(3)]
    for a, v in zip(at, x):
        a.copy_(v)
    w = dev(rand(cols, seed=203, shift=1.0))
    y, mean, rstd = ops.layer_norm(x[0], w, stats=True)
    assert same_bits(ops.layer_norm(at[0], w, out=at[3]), y)
    want = ops.layer_norm_backward(x[1], x[0], w, mean, rstd)
    got = ops.layer_norm_backward(at[1], at[0], w, mean, rstd, out=at[3])
    assert all(same_bits(p, q) for p, q in zip(got, want))
    seq = dev(torch.tensor([0, 300, 301, 1097]))
    want = ops.gated_scan(x[0], x[1], seq, activation="tanh", last=True, carry=True, out=dev(torch.zeros_like(x[0])))
    at[3].zero_()
    got = ops.gated_scan(at[0], at[1], seq, activation="tanh", last=True, carry=True, out=at[3])
    assert all(same_bits(p, q) for p, q in zip(got, want))
    carry = want[2]
    want = ops.gated_scan_backward(x[2], x[0], x[1], carry, seq, activation="tanh", out=(dev(torch.zeros_like(x[0])), dev(torch.zeros_like(x[0]))))
    at[3].zero_(), at[4].zero_()
    got = ops.gated_scan_backward(at[2], at[0], at[1], carry, seq, activation="tanh", out=(at[3], at[4]))
    assert all(same_bits(p, q) for p, q in zip(got, want))
    state = dev(rand(rows, cols, seed=204))
    other = state.clone()
    assert same_bits(ops.gated_scan_step(at[0], at[1], other, out=at[3]), ops.gated_scan_step(x[0], x[1], state)) and same_bits(other, state)
    index = dev(torch.arange(rows)[:, None] % cols + torch.zeros(1, 3, dtype=torch.long))
    want = ops.distill_loss(x[0], x[1][:, :3], index, 2.0)
    got = ops.distill_loss(at[0], at[1][:, :3], index, 2.0, out=at[3])
    assert all(same_bits(p, q) for p, q in zip(got, want))


def test_more_rows_than_workgroups():
    """Every row of a call with millions of them is that of a call with a few."""
    n, c = (1 << 21) + 1500, 5
    x, index = dev(rand(n, c, seed=210)), dev(torch.arange(n)[:, None] % c)
    w, dy = dev(rand(c, seed=211)), dev(rand(n, c, seed=212))
    loss, grad = ops.distill_loss(x, dy[:, :1], index)
    y, mean, rstd = ops.layer_norm(x, w, stats=True)
    dx = ops.layer_norm_backward(dy, x, w, mean, rstd)[0]
    state = x.clone()
    h = ops.gated_scan_step(dy, x, state)
    for s in (slice(0, 700), slice(n - 1600, n)):
        few = [t[s].contiguous() for t in (x, dy, index, mean, rstd)]
        assert all(same_bits(p[s], q) for p, q in zip((loss, grad), ops.distill_loss(few[0], few[1][:, :1], few[2])))
        assert same_bits(y[s], ops.layer_norm(few[0], w)) and same_bits(dx[s], ops.layer_norm_backward(few[1], few[0], w, *few[3:])[0])
        assert same_bits(h[s], ops.gated_scan_step(few[1], few[0], few[0].clone())) and same_bits(state[s], h[s])


@pytest.mark.parametrize("rows", [1, 128, 1000])
def test_scan_more_sequences_than_rows(rows):
    """Thousands of empty sequences before, between and behind the others hand their states through, in both directions."""
    n, hidden = 20000, 70
    begin = torch.cat([torch.zeros(n // 2, dtype=torch.long), torch.full((n - n // 2,), rows)])
    end = begin.clone()
    end[n // 2 - 1] = rows   # the one with rows
    h0, gate, cand, dh = (rand(n, hidden, seed=220), *(rand(rows, hidden, seed=221 + k) for k in range(3)))
    dlast = rand(n, hidden, seed=224)
    seq = (dev(begin), dev(end))
    h, last, carry = ops.gated_scan(*dev(gate, cand), seq, h0=dev(h0), last=True, carry=True)
    k = n // 2 - 1
    alone = ops.gated_scan(*dev(gate, cand), h0=dev(h0[k:k + 1]), last=True, carry=True)
    assert same_bits(h, alone[0]) and same_bits(last[k], alone[1][0])
    empty = torch.arange(n) != k
    assert same_bits(last.cpu()[empty], h0[empty])
    got = ops.gated_scan_backward(*dev(dh, gate, cand), carry, seq, h0=dev(h0), dlast=dev(dlast))
    want = ops.gated_scan_backward(*dev(dh, gate, cand), alone[2], h0=dev(h0[k:k + 1]), dlast=dev(dlast[k:k + 1]))
    assert same_bits(got[0], want[0]) and same_bits(got[1], want[1]) and same_bits(got[2][k], want[2][0])
    assert same_bits(got[2].cpu()[empty], dlast[empty])


# ------------------------------------------------------------------ together
def everything(s):
    """One pass through every operator: norm, recurrence, logits, loss, and all the way back."""
    y, mean, rstd = ops.layer_norm(s["x"], s["w"], s["b"], stats=True)
    h, last, carry = ops.gated_scan(y, s["cand"], s["seq"], h0=s["h0"], activation="tanh", last=True, carry=True)
    loss, dlogits = ops.distill_loss(h @ s["embed"], s["teacher"], s["index"], 2.0, s["row"])
    dh = dlogits @ s["embed_t"]
    dy, dcand, dh0 = ops.gated_scan_backward(dh, y, s["cand"], carry, s["seq"], h0=s["h0"], activation="tanh")
    dx, dw, db = ops.layer_norm_backward(dy, s["x"], s["w"], mean, rstd)
    step = ops.gated_scan_step(y[:2], s["cand"][:2], last[:2].clone())
    return [y, h, last, loss, dlogits, dx, dw, db, dcand, dh0, step]


def model(rows=700, hidden=64, classes=500, top=8, seed=0):
    g = torch.Generator().manual_seed(seed)
    embed = 0.3 * torch.randn(hidden, classes, generator=g)
    s = dict(x=torch.randn(rows, hidden, generator=g), w=1 + 0.1 * torch.randn(hidden, generator=g), b=torch.randn(hidden, generator=g),
             cand=torch.randn(rows, hidden, generator=g), seq=torch.tensor([0, 1, 130, 130, 500, rows]), h0=torch.randn(5, hidden, generator=g),
             embed=embed, embed_t=embed.t().contiguous(), teacher=torch.randn(rows, top, generator=g),
             index=torch.argsort(torch.rand(rows, classes, generator=g), 1)[:, :top], row=torch.full((rows,), 1.0 / rows))
    return s


def test_a_student_from_norm_to_loss_and_back():
    """The operators as a layer and its loss use them, against the whole computation in 64 bits by torch's own derivatives."""
    s = model()
    got = everything({k: v.cuda() for k, v in s.items()})
    d = {k: v.double() if v.is_floating_point() else v for k, v in s.items()}
    leaves = [d[k].requires_grad_() for k in ("x", "w", "b", "cand", "h0")]
    mean = d["x"].mean(1, keepdim=True)
    var = ((d["x"] - mean) ** 2).mean(1, keepdim=True)
    y = (d["x"] - mean) / (var + 1e-5).sqrt() * d["w"] + d["b"]
    z, v, hs = torch.sigmoid(y), torch.tanh(d["cand"]), []
    o = s["seq"].tolist()
    for k in range(5):
        h = d["h0"][k]
        for t in range(o[k], o[k + 1]):
            h = (1 - z[t]) * h + z[t] * v[t]
            hs.append(h)
    h = torch.stack(hs)
    lp, lq = torch.log_softmax(d["teacher"] / 2, 1), torch.log_softmax(h @ d["embed"] / 2, 1)
    loss = d["row"] * 4 * (lp.exp() * (lp - lq.gather(1, s["index"]))).sum(1)
    grads = torch.autograd.grad(loss.sum(), leaves)
    want = dict(y=(y, got[0]), h=(h, got[1]), loss=(loss, got[3]), dx=(grads[0], got[5]), dw=(grads[1], got[6]), db=(grads[2], got[7]),
                dcand=(grads[3], got[8]), dh0=(grads[4], got[9]))
    for name, (w, g) in want.items():
        # 32-bit products and sums over 64 .. 700 terms between the operators: some 2^-24 * 700 of the largest term
        assert (g.cpu().double() - w.detach()).abs().max() <= 2.0 ** -24 * 700 * max(1.0, 4 * float(w.detach().abs().max())), name
