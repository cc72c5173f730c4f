"""GPU: the gated delta rule, the policy loss and clipping against their formulas in 64 bits, within the bounds that more_reference derives
from 32-bit arithmetic; what they do with strides, rows of no sequence and values that are no numbers; and a training step of them."""
import math

import pytest
import torch
import torch.nn.functional as F

import more_reference as more
from ops_reference import check
from paper_1705_09786_amd import binding as B
from paper_1705_09786_amd import operators as ops
from test_gpu_operators import dev, holes, rand, same_bits, strided

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]
NAN, INF = float("nan"), float("inf")


# ------------------------------------------------------------------ gated delta rule
def layer(rows, n, heads, key_heads, dk, dv, dtype=torch.float32, seed=0, decay=0.1):
    """Inputs on the CPU: keys and queries of length one, n states in front and gradients behind."""
    q, k = (F.normalize(rand(rows, key_heads, dk, seed=seed + i) + 0.3 * rand(key_heads, dk, seed=seed + 9), dim=2).reshape(rows, -1).to(dtype)
            for i in (1, 2))
    return dict(q=q, k=k, v=rand(rows, heads * dv, seed=seed + 3, dtype=dtype), decay=-decay * rand(rows, heads, seed=seed + 4).abs(),
                beta=torch.sigmoid(rand(rows, heads, seed=seed + 5))), dict(
                    h0=rand(n, heads, dk, dv, seed=seed + 6, scale=0.2), do=rand(rows, heads * dv, seed=seed + 7, dtype=dtype, scale=0.3),
                    dlast=rand(n, heads, dk, dv, seed=seed + 8, scale=0.2))


NAMES = ("dq", "dk", "dv", "ddecay", "dbeta", "dh0")


def both(x, y, sequences, key_heads, scale=None):
    """Forward and backward pass on the GPU."""
    x = {k: v.cuda() for k, v in x.items()}
    where = sequences if sequences is None else tuple(t.cuda() for t in sequences) if isinstance(sequences, tuple) else sequences.cuda()
    o, last, carry = ops.gated_delta(*x.values(), where, key_heads=key_heads, scale=scale, h0=dev(y["h0"]), last=True, carry=True)
    grads = ops.gated_delta_backward(dev(y["do"]), *x.values(), carry, where, key_heads=key_heads, scale=scale, dlast=dev(y["dlast"]))
    return (o, last) + grads


def against(x, y, sequences, key_heads, got, scale=None):
    dtype = x["q"].dtype
    want = more.delta(*x.values(), sequences, key_heads, scale, y["h0"], dtype)[:2] + more.delta_backward(
        y["do"], *x.values(), sequences, key_heads, scale, y["h0"], y["dlast"], dtype)
    for name, g, w in zip(("o", "last") + NAMES, got, want):
        check(name, g, w)
        more.check_norm(name, g, w[0])


def offsets(*lengths, dtype=torch.int64):
    return torch.cumsum(torch.tensor((0,) + lengths), 0).to(dtype)


DELTA = [  # lengths, heads, key heads, dk, dv
    ((1,), 1, 1, 1, 1),
    ((31, 0, 32, 33, 1), 2, 2, 16, 16),
    ((63, 64, 65), 2, 1, 33, 40),
    ((130,), 3, 3, 50, 75),
    ((2, 97, 0, 0, 60), 4, 2, 64, 17),
    ((70, 40), 2, 2, 128, 128),
    ((66,), 1, 1, 65, 200),
    ((40,), 1, 1, 127, 129),
    ((1,) * 20 + (3,) * 20, 2, 1, 24, 36),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv", DELTA)
def test_delta(dtype, lengths, heads, key_heads, dk, dv):
    x, y = layer(sum(lengths), len(lengths), heads, key_heads, dk, dv, dtype)
    got = both(x, y, offsets(*lengths), key_heads)
    against(x, y, offsets(*lengths), key_heads, got)
    assert all(same_bits(p, q) for p, q in zip(got, both(x, y, offsets(*lengths, dtype=torch.int32), key_heads)))


@pytest.mark.parametrize("dtype", TYPES)
def test_delta_one_long_sequence(dtype):
    """Many chunks, no offsets, a scale of its own, states kept almost whole."""
    x, y = layer(1100, 1, 2, 2, 32, 24, dtype, decay=0.002)
    against(x, y, None, 2, both(x, y, None, 2, 0.7), 0.7)


@pytest.mark.parametrize("case", ["reset", "strong", "none", "growth", "beta", "zero_keys"])
def test_delta_decays_and_rates(case):
    x, y = layer(100, 1, 2, 2, 20, 20)
    if case == "reset":      # rows that forget everything
        x["decay"][[0, 17, 40, 64, 99]] = -INF
    elif case == "strong":   # sums far below what differences of floats would resolve
        x["decay"] = x["decay"] * 900
        x["decay"][50:] = -1e-4
    elif case == "none":
        x["decay"] *= 0
    elif case == "growth":
        x["decay"] = x["decay"].abs() * 0.1
    elif case == "beta":
        x["beta"] = 2 * x["beta"]
        x["beta"][::3] = 0
    else:
        x["k"][20:60] = 0
    got = both(x, y, None, 2)
    against(x, y, None, 2, got)


def test_delta_parts_of_wider_arrays_and_rows_of_no_sequence():
    lengths, heads, key_heads, dk, dv = (40, 33), 2, 1, 30, 21
    rows = 100
    x, y = layer(rows, 2, heads, key_heads, dk, dv)
    begin, end = torch.tensor([5, 60]), torch.tensor([45, 93])
    outside = torch.ones(rows, dtype=torch.bool)
    for b, e in zip(begin, end):
        outside[b:e] = False
    for t in (x["q"], x["k"], x["v"], x["decay"], x["beta"], y["do"]):
        t[outside] = NAN
    clean = {k: torch.nan_to_num(v) for k, v in x.items()}
    cy = {k: torch.nan_to_num(v) for k, v in y.items()}
    got = both(x, y, (begin, end), key_heads)
    for g in got[:1] + got[2:7]:
        assert (g[outside.cuda()] == 0).all()
    against(clean, cy, (begin, end), key_heads, got)
    # q, k and v as columns of one array, gates as columns of another, outputs into columns: the same bits, the rest untouched
    widths = [key_heads * dk, key_heads * dk, heads * dv]
    packed = torch.cat([x["q"], x["k"], x["v"], rand(rows, 3)], 1).cuda()
    q, k, v = packed[:, :-3].split(widths, 1)
    gates = torch.cat([x["decay"], rand(rows, 1), x["beta"]], 1).cuda()
    args = q, k, v, gates[:, :heads], gates[:, heads + 1:]
    where = begin.cuda(), end.cuda()
    o_buf = torch.full((rows, heads * dv + 5), 7.0, device="cuda")
    o, last, carry = ops.gated_delta(*args, where, key_heads=key_heads, h0=dev(y["h0"]), last=True, carry=True, out=o_buf[:, 2:-3])
    assert (o_buf[outside.cuda()] == 7).all() and (o_buf[:, :2] == 7).all() and (o_buf[:, -3:] == 7).all()
    assert same_bits(o[~outside.cuda()], got[0][~outside.cuda()]) and same_bits(last, got[1])
    d_packed, d_gates = torch.full_like(packed, 7.0), torch.full_like(gates, 7.0)
    out = tuple(d_packed[:, :-3].split(widths, 1)) + (d_gates[:, :heads], d_gates[:, heads + 1:])
    grads = ops.gated_delta_backward(dev(y["do"]), *args, carry, where, key_heads=key_heads, dlast=dev(y["dlast"]), out=out)
    assert (d_packed[outside.cuda()] == 7).all() and (d_packed[:, -3:] == 7).all() and (d_gates[:, heads] == 7).all() and (d_gates[outside.cuda()] == 7).all()
    for g, w in zip(grads[:5], got[2:7]):
        assert same_bits(g[~outside.cuda()], w[~outside.cuda()])
    assert same_bits(grads[5], got[7])


def test_delta_one_row_of_any_stride():
    x, y = layer(1, 1, 2, 1, 8, 12)
    want = both(x, y, None, 1)
    on = {k: torch.empty_strided(v.shape, (1 << 30, 1), device="cuda").copy_(v) for k, v in x.items()}
    o, last, carry = ops.gated_delta(*on.values(), key_heads=1, h0=dev(y["h0"]), last=True, carry=True)
    do = torch.empty_strided(y["do"].shape, (1 << 30, 1), device="cuda").copy_(y["do"])
    grads = ops.gated_delta_backward(do, *on.values(), carry, key_heads=1, dlast=dev(y["dlast"]))
    assert all(same_bits(p, q) for p, q in zip((o, last) + grads, want))


def test_delta_without_rows_or_sequences():
    x, y = layer(6, 3, 2, 2, 8, 8)
    empty = torch.zeros(4, dtype=torch.int64)
    got = both(x, y, empty, 2)
    assert (got[0] == 0).all() and same_bits(got[1].cpu(), y["h0"]) and same_bits(got[7].cpu(), y["dlast"]) and all((g == 0).all() for g in got[2:7])
    none = {k: v[:0] for k, v in x.items()}
    got = both(none, dict(y, do=y["do"][:0]), empty, 2)
    assert got[0].shape == (0, 16) and same_bits(got[1].cpu(), y["h0"]) and same_bits(got[7].cpu(), y["dlast"])
    got = both(x, dict(y, h0=y["h0"][:0], dlast=y["dlast"][:0]), torch.zeros(1, dtype=torch.int64), 2)
    assert (got[0] == 0).all() and all((g == 0).all() for g in got[2:7]) and got[1].shape == (0, 2, 8, 8)


def test_delta_bounds_outside_the_rows():
    """Bounds beyond the array are taken for its ends; sequences out of order harm nothing but their own outputs."""
    x, y = layer(90, 2, 2, 2, 16, 16)
    got = both(x, y, torch.tensor([-5, 50, 1 << 40]), 2)
    want = both(x, y, torch.tensor([0, 50, 90]), 2)
    assert all(same_bits(p, q) for p, q in zip(got, want))
    both(x, y, (torch.tensor([80, 0]), torch.tensor([20, 90])), 2)
    both(x, y, (torch.tensor([0, 0]), torch.tensor([90, 90])), 2)
    torch.cuda.synchronize()


def test_delta_thousands_of_sequences():
    """More than the plan keeps near: the same bits as in two calls for half of them each."""
    n = 6001
    lengths = torch.randint(0, 4, (n,), generator=torch.Generator().manual_seed(1))
    lengths[3000] = 200
    where = offsets(*lengths.tolist())
    rows, half = int(where[-1]), 3000
    x, y = layer(rows, n, 1, 1, 8, 8)
    got = both(x, y, where, 1)
    cut = int(where[half])
    parts = [both({k: v[:cut] for k, v in x.items()}, dict(h0=y["h0"][:half], do=y["do"][:cut], dlast=y["dlast"][:half]), where[:half + 1], 1),
             both({k: v[cut:] for k, v in x.items()}, dict(h0=y["h0"][half:], do=y["do"][cut:], dlast=y["dlast"][half:]), where[half:] - cut, 1)]
    for i, g in enumerate(got):
        assert same_bits(g, torch.cat([p[i] for p in parts]))
    some = slice(int(where[2990]), int(where[3010]))
    want = more.delta(*(t[some] for t in x.values()), where[2990:3011] - where[2990], 1, None, y["h0"][2990:3010], torch.float32)
    check("o", got[0][some], want[0])
    check("last", got[1][2990:3010], want[1])


def test_delta_numbers_that_are_none_stay_in_their_sequence_and_head():
    lengths = (50, 45)
    x, y = layer(95, 2, 2, 2, 16, 16)
    want = both(x, y, offsets(*lengths), 2)
    for name, row in (("q", 60), ("k", 61), ("v", 62), ("decay", 63), ("beta", 64)):
        bad = {k: v.clone() for k, v in x.items()}
        bad[name][row, bad[name].shape[1] // 2:] = NAN   # head 1 of sequence 1
        got = both(bad, y, offsets(*lengths), 2)
        for g, w in zip(got, want):
            if g.dim() == 4:
                assert same_bits(g[0], w[0]) and same_bits(g[1, 0], w[1, 0])
            else:
                half = g.shape[1] // 2
                assert same_bits(g[:50], w[:50]) and same_bits(g[:, :half], w[:, :half])
        assert not all(g.isfinite().all() for g in got)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,heads,key_heads,dk,dv", [(1, 1, 1, 1, 1), (3, 4, 2, 50, 75), (48, 2, 2, 128, 128), (5, 6, 1, 33, 130), (2, 1, 1, 64, 31)])
def test_delta_step(dtype, rows, heads, key_heads, dk, dv):
    x, y = layer(rows, rows, heads, key_heads, dk, dv, dtype)
    buf = torch.full((rows, heads * dk * dv + 7), 5.0, device="cuda")
    state = buf[:, 3:-4].unflatten(1, (heads, dk, dv))
    state.copy_(y["h0"])
    args = [t.cuda() for t in x.values()]
    o = ops.gated_delta_step(*args, state, key_heads=key_heads)
    want = more.delta_step(*x.values(), y["h0"], key_heads, None)
    check("o", o, want[0])
    check("state", state, want[1])
    assert (buf[:, :3] == 5).all() and (buf[:, -4:] == 5).all()
    # one row at a time is what the whole sequence gives, from the same states
    whole, last, _ = ops.gated_delta(*args, torch.arange(rows + 1, device="cuda"), key_heads=key_heads, h0=dev(y["h0"]), last=True)
    want = more.delta(*x.values(), torch.arange(rows + 1), key_heads, None, y["h0"], dtype)
    check("o", whole, want[0])
    check("last", last, want[1])


def test_delta_offsets_past_32_bits():
    """Rows of an array of more than 2^31 elements: sequences at its two ends."""
    n, stride = 700, (1 << 22) - 8
    x, y = layer(n, 2, 1, 1, 8, 8, torch.bfloat16)
    begin, end = torch.tensor([0, 660]), torch.tensor([35, 700])
    wide = torch.empty(n * stride, dtype=torch.bfloat16, device="cuda")
    args = [t.cuda() for t in x.values()]
    for i in (0, 1, 2):
        view = wide.as_strided((n, 8), (stride, 1), 16 * i)
        view.copy_(args[i])
        args[i] = view
    o, do = (wide.as_strided((n, 8), (stride, 1), at) for at in (48, 64))
    do.copy_(y["do"])
    got = ops.gated_delta(*args, (begin.cuda(), end.cuda()), h0=dev(y["h0"]), last=True, carry=True, out=o)
    inside = torch.zeros(n, dtype=torch.bool)
    inside[:35] = inside[660:] = True
    want = more.delta(*x.values(), (begin, end), 1, None, y["h0"], torch.bfloat16)
    check("o", got[0][inside.cuda()], tuple(t[inside] for t in want[0]))
    check("last", got[1], want[1])
    back = tuple(wide.as_strided((n, 8), (stride, 1), at) for at in (80, 96, 112)) + tuple(torch.zeros(n, 1, device="cuda") for _ in range(2))
    grads = ops.gated_delta_backward(do, *args, got[2], (begin.cuda(), end.cuda()), dlast=dev(y["dlast"]), out=back)
    want = more.delta_backward(y["do"], *x.values(), (begin, end), 1, None, y["h0"], y["dlast"], torch.bfloat16)
    for name, g, w in zip(NAMES, grads, want):
        if g.dim() == 2:
            g, w = g[inside.cuda()], tuple(t[inside] for t in w)
        check(name, g, w)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sequences", [None, (2000, 0, 3, 2300), (5, 1700, 1800, 64)])
def test_delta_sequences_cut_into_segments(dtype, sequences):
    """One head and long sequences: segments side by side, joined from their maps. States that hardly fade carry errors far."""
    rows = 3000 if sequences is None else sum(sequences)
    n = 1 if sequences is None else len(sequences)
    x, y = layer(rows, n, 1, 1, 24, 20, dtype, decay=0.001)
    x["decay"][rows // 2] = -INF
    where = None if sequences is None else offsets(*sequences)
    got = both(x, y, where, 1)
    against(x, y, where, 1, got)
    assert all(same_bits(p, q) for p, q in zip(got, both(x, y, where, 1)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,heads", [(1536, 1), (2048, 2), (4096, 1)])
def test_delta_without_bounds_in_whole_segments(dtype, rows, heads):
    """Rows that whole blocks and whole segments make up: one sequence is what its offsets say it is, to the last segment."""
    x, y = layer(rows, 1, heads, 1, 24, 20, dtype, decay=0.001)
    got = both(x, y, None, 1)
    assert all(same_bits(p, q) for p, q in zip(got, both(x, y, offsets(rows), 1)))
    against(x, y, None, 1, got)


@pytest.mark.parametrize("rows,heads,dk,dv", [(2048, 16, 128, 128), (8192, 4, 64, 64), (16384, 2, 50, 75), (32768, 8, 16, 16)])
def test_delta_without_bounds_is_one_sequence_of_all_rows(rows, heads, dk, dv):
    x, y = layer(rows, 1, heads, heads, dk, dv, torch.bfloat16, decay=0.001)
    x, y = ({k: v.cuda() for k, v in t.items()} for t in (x, y))
    got, want = both(x, y, None, heads), both(x, y, offsets(rows), heads)
    assert all(same_bits(p, q) for p, q in zip(got, want)) and all(g.isfinite().all() for g in got)


def some_lengths(n, most, seed):
    return torch.randint(0, most + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,heads,key_heads,dk,dv", [(70, 2, 2, 20, 70), (33, 4, 2, 50, 75), (12, 16, 16, 128, 66), (36, 4, 1, 100, 130)])
def test_delta_more_than_128_chains(dtype, n, heads, key_heads, dk, dv):
    """Sequences and heads enough for every type's workgroups of eight waves, at each size of a key."""
    assert n * heads * ((dv + 127) // 128) > 128 and dv > 64
    lengths = some_lengths(n, 70, n)
    x, y = layer(sum(lengths), n, heads, key_heads, dk, dv, dtype)
    against(x, y, offsets(*lengths), key_heads, both(x, y, offsets(*lengths), key_heads))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv", [((100, 33), 4, 1, 128, 40), ((70,), 3, 1, 50, 75), ((66, 5), 6, 2, 24, 20), ((65,), 5, 1, 3, 5),
                                                           ((40,), 2, 1, 128, 3), ((90,), 1, 1, 8, 1024)])
def test_delta_several_heads_to_a_key(dtype, lengths, heads, key_heads, dk, dv):
    """A head between the first and the last both takes its key's sums and leaves them; rows narrower than four; the widest."""
    x, y = layer(sum(lengths), len(lengths), heads, key_heads, dk, dv, dtype)
    against(x, y, offsets(*lengths), key_heads, both(x, y, offsets(*lengths), key_heads))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lengths,heads,key_heads,dk,dv", [((1600,), 2, 1, 128, 130), ((1700, 100), 2, 2, 128, 128), ((1600, 300, 0, 40), 2, 2, 50, 75),
                                                           ((1599,), 3, 1, 64, 64)])
def test_delta_segments_of_wide_states(dtype, lengths, heads, key_heads, dk, dv):
    """Maps and their join at every size of a key, for several heads and more columns than a workgroup has."""
    x, y = layer(sum(lengths), len(lengths), heads, key_heads, dk, dv, dtype, decay=0.001)
    where = None if len(lengths) == 1 else offsets(*lengths)
    got = both(x, y, where, key_heads)
    against(x, y, where, key_heads, got)
    assert all(same_bits(p, q) for p, q in zip(got, both(x, y, where, key_heads)))


# ------------------------------------------------------------------ policy loss
def tokens(rows, classes, dtype=torch.float32, seed=0, temperature=1.0):
    logits = rand(rows, classes, seed=seed, scale=1.5)
    index = torch.randint(0, classes, (rows,), generator=torch.Generator().manual_seed(seed + 1))
    logits.scatter_add_(1, index[:, None], 4 + 2 * rand(rows, 1, seed=seed + 2))
    logits = logits.to(dtype)
    lp = torch.log_softmax(logits.double() / temperature, 1).gather(1, index[:, None])[:, 0]
    return dict(logits=logits, index=index, old=(lp + 0.25 * rand(rows, seed=seed + 3)).float(), advantage=rand(rows, seed=seed + 4)), dict(
        reference=(lp + 0.4 * rand(rows, seed=seed + 5)).float(), weight=rand(rows, seed=seed + 6).abs() / rows)


def policy_against(x, y, kl=0.1, clip=(0.2, 0.3), temperature=1.0, **kw):
    on = {k: dev(v) for k, v in {**x, **y}.items()}
    got = ops.policy_loss(on["logits"], on["index"], on["old"], on["advantage"], reference=on["reference"], kl=kl, clip=clip, temperature=temperature,
                          weight=on["weight"], **kw)
    want = more.policy(x["logits"], x["index"], x["old"], x["advantage"], y["reference"], kl, *clip, temperature, y["weight"])
    for name, g, w in zip(("loss", "logprob", "dlogits"), got, want):
        if g is not None:
            check(name, g, w)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("classes", [1, 2, 3, 5, 8, 9, 257, 1000, 2049, 8200, 20000, 33001, 70001, 140003])
def test_policy(dtype, classes):
    rows = 9 if classes < 30000 else 3
    x, y = tokens(rows, classes, dtype)
    got = policy_against(x, y)
    again = policy_against(x, y, grad=False)
    assert again[2] is None
    temperature = 0.7
    x, y = tokens(rows, classes, dtype, 5, temperature)
    policy_against(x, y, 0.0, (0.2, 0.2), temperature)
    lp = ops.token_logprob(x["logits"].cuda(), x["index"].int().cuda(), temperature)
    check("logprob", lp, more.policy(x["logits"], x["index"], None, None, None, 0, 0, 0, temperature, None)[1])
    assert all(same_bits(p, q) for p, q in zip(got, policy_against(*tokens(rows, classes, dtype))))


def test_policy_many_rows_and_what_may_be_missing():
    x, y = tokens(3000, 130, torch.bfloat16)
    policy_against(x, y)
    for missing in ("old", "reference", "weight"):
        a, b = dict(x), dict(y)
        (a if missing == "old" else b)[missing] = None
        policy_against(a, b)


def test_policy_strides_in_place_and_left_out_rows():
    x, y = tokens(12, 333, torch.float16)
    x["index"][2], x["index"][5] = -100, 333
    y["weight"][[0, 7]] = 0
    x["logits"][2], x["logits"][7] = NAN, NAN   # rows that have no gradient, whatever they hold
    y["weight"][2] = NAN
    clean = dict(x, logits=torch.nan_to_num(x["logits"]))
    want = more.policy(clean["logits"], x["index"], x["old"], x["advantage"], y["reference"], 0.1, 0.2, 0.3, 1.0, torch.nan_to_num(y["weight"]))
    view, buf = strided(x["logits"], 337, 3)
    out, obuf = strided(torch.zeros_like(x["logits"]), 335, 1)
    args = [x["index"].cuda(), x["old"].cuda(), x["advantage"].cuda()]
    kw = dict(reference=y["reference"].cuda(), kl=0.1, clip=(0.2, 0.3), weight=y["weight"].cuda())
    loss, lp, grad = ops.policy_loss(view, *args, out=out, **kw)
    assert grad is out and holes(obuf, out).isnan().all()
    assert lp[7].isnan() and (grad[[0, 2, 5, 7]] == 0).all() and (loss[[0, 2, 5, 7]] == 0).all() and (lp[[2, 5]] == 0).all()
    keep = torch.ones(12, dtype=torch.bool)
    keep[7] = False
    for name, g, w in zip(("loss", "logprob", "dlogits"), (loss, lp, grad), want):
        check(name, g[keep.cuda()], tuple(t[keep] for t in w))
    place = ops.policy_loss(view, *args, out=view, **kw)
    assert place[2] is view and same_bits(view, out) and same_bits(place[0], loss) and holes(buf, view).isnan().all()


@pytest.mark.parametrize("classes", [40, 5000, 140003])
def test_policy_logits_at_the_edges(classes):
    x, y = tokens(6, classes)
    x["logits"][0, ::2] = -INF                            # classes that are masked
    x["logits"][1, 1:] = torch.finfo(torch.float32).min   # nothing but one left
    x["logits"][2] += 3e4
    x["logits"][3] = 0.0
    x["logits"][4] *= 1e3
    x["index"][:5] = torch.tensor([1, 0, 3, 4, int(x["logits"][4].argmax())])
    lp = torch.log_softmax(x["logits"].double(), 1).gather(1, x["index"][:, None])[:, 0]
    x["old"], y["reference"] = (lp + 0.1).float(), (lp - 0.1).float()
    policy_against(x, y)
    x["logits"][1], x["logits"][3, 2], x["logits"][4, 5] = -INF, NAN, INF
    got = policy_against_rows(x, y, [0, 2, 5])
    for g in got:
        assert g[[1, 3, 4]].reshape(3, -1).isnan().any(1).all()


def policy_against_rows(x, y, rows):
    on = {k: dev(v) for k, v in {**x, **y}.items()}
    got = ops.policy_loss(on["logits"], on["index"], on["old"], on["advantage"], reference=on["reference"], kl=0.1, clip=(0.2, 0.3), weight=on["weight"])
    want = more.policy(*(x[k][rows] for k in ("logits", "index", "old", "advantage")), y["reference"][rows], 0.1, 0.2, 0.3, 1.0, y["weight"][rows])
    for name, g, w in zip(("loss", "logprob", "dlogits"), got, want):
        check(name, g[rows], w)
    return got


def test_policy_next_to_the_limits():
    """Two equal classes: lp is log(1/2) to the last bit; ratios one step of `old` to either side of both limits."""
    steps = []
    for limit in (1.2, 0.8):
        at = torch.tensor(math.log(0.5) - math.log(limit), dtype=torch.float32)
        steps += [torch.nextafter(at, torch.tensor(-INF)), at, torch.nextafter(at, torch.tensor(INF))]
    old = torch.stack(steps).repeat(2)
    n = old.numel()
    x = dict(logits=torch.zeros(n, 2), index=torch.zeros(n, dtype=torch.int64), old=old, advantage=torch.cat([torch.ones(n // 2), -torch.ones(n // 2)]))
    y = dict(reference=None, weight=None)
    _, _, grad = policy_against(x, y, 0.0, (0.2, 0.2))
    free = (grad != 0).any(1).cpu()
    r = math.log(0.5) - old.double()
    assert torch.equal(free, torch.where(x["advantage"] > 0, r <= math.log1p(0.2), r >= math.log1p(-0.2)))
    assert free.any() and not free.all()


def test_policy_far_ratios_and_open_limits():
    x, y = tokens(8, 50)
    x["old"][0], x["old"][1], x["advantage"][0], x["advantage"][1] = -200.0, -200.0, 1.0, 0.0
    policy_against(x, y)
    x, y = tokens(8, 50)
    policy_against(x, y, 0.1, (1.0, INF))


@pytest.mark.parametrize("classes", [40, 5000, 140003])
def test_policy_class_without_probability(classes):
    """Without `old` the ratio is 1 whatever the class's probability is: 0, a part of a bit, or all there is."""
    x, y = tokens(4, classes)
    x["logits"][0, int(x["index"][0])] = -INF
    x["logits"][1, int(x["index"][1])] = -1e4
    x["logits"][2] = -INF
    x["logits"][2, int(x["index"][2])] = 0.0
    x["old"], y["reference"] = None, None
    got = policy_against(x, y)
    assert got[1][0] == -INF and got[0][0] == -(x["advantage"] * y["weight"])[0]
    x["logits"][3, 0] = NAN   # a log-probability that is no number leaves no loss and no gradient
    x["index"][3] = 1
    got = ops.policy_loss(x["logits"].cuda(), x["index"].cuda(), None, x["advantage"].cuda())
    assert all(g[3].isnan().any() for g in got) and all(g[:3].isfinite().all() for g in (got[0], got[2]))


def test_policy_advantage_that_is_no_number():
    """On neither side of a limit: loss and gradient are no numbers, however far the ratio is."""
    x, y = tokens(3, 50)
    x["advantage"][:] = NAN
    lp = torch.log_softmax(x["logits"].double(), 1).gather(1, x["index"][:, None])[:, 0]
    x["old"] = (lp + torch.tensor([-2.0, 0.0, 2.0])).float()
    loss, _, grad = ops.policy_loss(*(x[k].cuda() for k in ("logits", "index", "old", "advantage")))
    assert loss.isnan().all() and grad.isnan().all()


def test_policy_very_long_row():
    """2^24 classes, all but the first 0.3 below those: a thread's sum has thousands of equal terms, whose roundings in 32 bits would all point the
    same way. Allowed: a term's own units (more_reference.policy), eight additions of them in 32 bits, and the result's rounding."""
    classes, high, advantage, far = 1 << 24, 1 << 14, 2.0, 0.3
    x = torch.full((1, classes), -far)
    x[0, :high] = 0.0
    index = torch.tensor([classes - 5])
    far = -float(x[0, -1])   # as 32 bits have it
    lp = -far - math.log((classes - high) * math.exp(-far) + high)
    units = 4 + 3 * far + 8
    want = torch.tensor([lp], dtype=torch.float64), torch.tensor([units], dtype=torch.float64)
    on = x.cuda(), index.cuda()
    check("logprob", ops.token_logprob(*on), want)
    _, got, grad = ops.policy_loss(*on, None, torch.tensor([advantage], device="cuda"))
    check("logprob", got, want)
    value = advantage * torch.exp(x.double() + far + lp)
    value[0, -5] = -advantage * (1 - math.exp(lp))
    check("dlogits", grad, (value, (2 * units + 4) * value.abs()))


# ------------------------------------------------------------------ clipping
def some_tensors(sizes, dtype, seed=0, scale=1.0):
    return [rand(math.prod(s) if isinstance(s, tuple) else s, seed=seed + i, dtype=dtype, scale=scale).reshape(s) for i, s in enumerate(sizes)]


SIZES = [(1,), (0, 5, (3, 7), ()), ((150, 300), 150, 1, (2, 3, 4), 4099), (70001,) * 3, tuple(range(1, 300)), (1 << 21, (1 << 21) + 3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes", SIZES)
def test_clip(dtype, sizes):
    host = some_tensors(sizes, dtype)
    grads = dev(*host) if len(host) > 1 else [dev(*host)]
    norm, _ = more.clip(host, None)
    alone = ops.clip_gradients(grads)
    check("norm", alone, norm)
    for max_norm in (0.5 * float(norm[0]), 2.0 * float(norm[0]), 0.0):
        want = more.clip(host, max_norm)[1]
        out = [torch.empty_like(g) for g in grads]
        assert same_bits(ops.clip_gradients(grads, max_norm, out=out), alone)
        for o, w in zip(out, want):
            check("out", o, w)
        place = [g.clone() for g in grads]
        assert same_bits(ops.clip_gradients(place, max_norm), alone)
        assert all(same_bits(p, o) for p, o in zip(place, out))
        assert all(same_bits(g.cpu(), h) for g, h in zip(grads, host))


def test_clip_mixed_types_and_parts_of_a_buffer():
    host = some_tensors((100, 33, 7), torch.float32) + some_tensors((50, 9), torch.bfloat16, 5) + some_tensors((77,), torch.float16, 9)
    grads = dev(*host)
    flat = torch.full((150,), 3.0, dtype=torch.float32, device="cuda")
    out = [flat[1:101], flat[101:134], flat[134:141]] + [torch.empty_like(g) for g in grads[3:]]
    ops.clip_gradients(grads, 1.0, out=out)
    for o, w in zip(out, more.clip(host, 1.0)[1]):
        check("out", o, w)
    assert flat[0] == 3 and (flat[141:] == 3).all()


def test_clip_norms_that_floats_do_not_hold_on_the_way():
    big = [torch.full((1000,), 1e30, device="cuda"), torch.full((7,), 1e-30, device="cuda")]
    check("norm", ops.clip_gradients(big), more.clip([b.cpu() for b in big], None)[0])
    small = [torch.full((1000,), 1e-30, device="cuda")]
    check("norm", ops.clip_gradients(small), more.clip([b.cpu() for b in small], None)[0])
    for bad in (INF, NAN):
        t = [torch.ones(10, device="cuda"), torch.tensor([1.0, bad], device="cuda")]
        keep = [x.clone() for x in t]
        norm = ops.clip_gradients(t, 0.1)
        assert not norm.isfinite() and all(same_bits(p, q) for p, q in zip(t, keep))
    zero = [torch.zeros(10, device="cuda")]
    assert ops.clip_gradients(zero, 1.0) == 0 and (zero[0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-6, 1e-8])
def test_clip_by_factors_below_the_smallest_normal_float(dtype, max_norm):
    """Norms of 1e38 and small limits: the factor is below 2^-126, the results are not."""
    host = some_tensors((100, 7, 4099), dtype, scale=1.5e36)
    grads = dev(*host)
    norm = ops.clip_gradients(grads)
    assert 5e37 < float(norm) < 2e38
    out = [torch.empty_like(g) for g in grads]
    ops.clip_gradients(grads, max_norm, out=out)
    for o, w in zip(out, more.clip(host, max_norm)[1]):
        check("out", o, w)
    ops.clip_gradients(grads, max_norm)
    assert all(same_bits(p, o) for p, o in zip(grads, out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_clip_leaves_a_norm_beyond_floats(dtype):
    """Finite numbers whose norm is not: as with any norm that is not finite, the elements stay."""
    grads = [torch.full((10,), 3e38, dtype=dtype, device="cuda"), torch.ones(5, dtype=dtype, device="cuda")]
    keep, out = [g.clone() for g in grads], [torch.zeros_like(g) for g in grads]
    assert ops.clip_gradients(grads, 1.0, out=out) == INF
    assert all(same_bits(p, q) for p, q in zip(out, keep))
    assert ops.clip_gradients(grads, 1.0) == INF
    assert all(same_bits(p, q) for p, q in zip(grads, keep))


# ------------------------------------------------------------------ together
def problem(seed, dtype=torch.bfloat16):
    """A layer over packed sequences, with the classes that were drawn: every input of a training step."""
    lengths, heads, key_heads, dk, dv, classes, hidden = (70, 1, 0, 45), 2, 1, 24, 20, 97, 32
    rows = sum(lengths)
    w = dict(wx=rand(hidden, 2 * key_heads * dk + heads * dv, seed=seed, scale=hidden ** -0.5), wn=rand(heads * dv, seed=seed + 1, scale=0.1, shift=1.0),
             wo=rand(heads * dv, classes, seed=seed + 2, scale=0.2))
    s = dict(x=rand(rows, hidden, seed=seed + 3), decay=-0.1 * rand(rows, heads, seed=seed + 4).abs(), beta=torch.sigmoid(rand(rows, heads, seed=seed + 5)),
             index=torch.randint(0, classes, (rows,), generator=torch.Generator().manual_seed(seed + 6)), old=-4.5 + 0.1 * rand(rows, seed=seed + 7),
             reference=-4.5 + 0.1 * rand(rows, seed=seed + 8), advantage=rand(rows, seed=seed + 9), weight=torch.full((rows,), 1.0 / rows),
             offsets=offsets(*lengths))
    return {**w, **s}, dict(heads=heads, key_heads=key_heads, dk=dk, dv=dv, dtype=dtype)


def train_step(s, c, max_norm=0.05):
    """Loss, the norm and the clipped gradients of the weights, through the operators; matrix products in 32 bits."""
    kh, dk, t = c["key_heads"], c["dk"], c["dtype"]
    widths = [kh * dk, kh * dk, c["heads"] * c["dv"]]
    p = s["x"] @ s["wx"]
    raw = p.split(widths, 1)
    # keys and queries of length one, and the derivative of that
    scale = [1.0 / raw[i].reshape(-1, kh, dk).norm(dim=2, keepdim=True) for i in (0, 1)]
    unit = [raw[i].reshape(-1, kh, dk) * scale[i] for i in (0, 1)]
    args = [unit[0].reshape(-1, kh * dk).to(t), unit[1].reshape(-1, kh * dk).to(t), raw[2].to(t), s["decay"], s["beta"]]
    o, _, carry = ops.gated_delta(*args, s["offsets"], key_heads=kh, carry=True)
    y, mean, rstd = ops.layer_norm(o, s["wn"], stats=True)
    logits = y.float() @ s["wo"]
    loss, lp, dlogits = ops.policy_loss(logits, s["index"], s["old"], s["advantage"], reference=s["reference"], kl=0.1, weight=s["weight"])
    dwo, dy = y.float().T.contiguous() @ dlogits, dlogits @ s["wo"].T.contiguous()
    do, dwn, _ = ops.layer_norm_backward(dy.to(t), o, s["wn"], mean, rstd)
    grads = ops.gated_delta_backward(do, *args, carry, s["offsets"], key_heads=kh)
    back = []
    for i in (0, 1):
        g = grads[i].float().reshape(-1, kh, dk)
        back.append((scale[i] * (g - unit[i] * (g * unit[i]).sum(2, keepdim=True))).reshape(-1, kh * dk))
    dwx = s["x"].T.contiguous() @ torch.cat(back + [grads[2].float()], 1)
    out = [dwx, dwn, dwo]
    norm = ops.clip_gradients(out, max_norm)
    return [loss, lp, norm] + out + list(grads[3:5])


def plain_step(s, c, max_norm=0.05):
    """The same in 64 bits with torch's own derivatives, on the CPU."""
    kh, dk, heads = c["key_heads"], c["dk"], c["heads"]
    w = {k: s[k].double().requires_grad_() for k in ("wx", "wn", "wo", "decay", "beta")}
    p = s["x"].double() @ w["wx"]
    q, k, v = p.split([kh * dk, kh * dk, heads * c["dv"]], 1)
    q, k = (F.normalize(x.reshape(-1, kh, dk), dim=2).repeat_interleave(heads // kh, 1) for x in (q, k))
    v = v.reshape(-1, heads, c["dv"])
    rows = []
    for b, e in zip(s["offsets"][:-1].tolist(), s["offsets"][1:].tolist()):
        S = torch.zeros(heads, dk, c["dv"], dtype=torch.float64)
        for t in range(b, e):
            S = torch.exp(w["decay"][t])[:, None, None] * S
            err = v[t] - (k[t][..., None] * S).sum(1)
            S = S + w["beta"][t][:, None, None] * k[t][..., None] * err[:, None]
            rows.append((dk ** -0.5 * (q[t][..., None] * S).sum(1)).reshape(-1))
    o = torch.stack(rows)
    y = F.layer_norm(o, (o.shape[1],), w["wn"], None, 1e-5)
    lp = torch.log_softmax(y @ w["wo"], 1).gather(1, s["index"][:, None])[:, 0]
    r, d, A = torch.exp(lp - s["old"].double()), s["reference"].double() - lp, s["advantage"].double()
    loss = s["weight"].double() * (-torch.minimum(r * A, r.clamp(0.8, 1.2) * A) + 0.1 * (torch.exp(d) - d - 1))
    loss.sum().backward()
    grads = [w[k].grad for k in ("wx", "wn", "wo")]
    norm = torch.stack([(g ** 2).sum() for g in grads]).sum().sqrt()
    f = min(1.0, max_norm / float(norm))
    return [loss.detach(), lp.detach(), norm] + [g * f for g in grads] + [w["decay"].grad, w["beta"].grad]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_step(dtype):
    """The operators' gradients joined by hand are those of the formulas. In 32 bits the chain of some ten operations is off by some units
    of the sizes that meet, sums of 1e-7 of them; in bf16 each of eight roundings of the activations and their gradients is half a step
    of 2^-8, as often up as down: sqrt(8) / 2 steps, twice that where a norm divides by a spread of its own."""
    s, c = problem(1, dtype)
    got = train_step({k: v.cuda() for k, v in s.items()}, c)
    for name, g, w in zip(("loss", "logprob", "norm", "dwx", "dwn", "dwo", "ddecay", "dbeta"), got, plain_step(s, c)):
        off = float((g.cpu().double() - w).norm() / w.norm())
        assert off <= (2e-5 if dtype == torch.float32 else math.sqrt(8) * 2.0 ** -8), (name, off)


def test_steps_after_a_prefix():
    """A sequence read as a whole and then row by row, from the state that was left, is the sequence read as a whole."""
    x, y = layer(80, 1, 3, 3, 40, 24)
    args = {k: v.cuda() for k, v in x.items()}
    want = more.delta(*x.values(), None, 3, None, None, torch.float32)
    o, state, _ = ops.gated_delta(*(t[:61] for t in args.values()), last=True)
    out = [o]
    for t in range(61, 80):
        out.append(ops.gated_delta_step(*(a[t:t + 1] for a in args.values()), state))
    check("o", torch.cat(out), want[0])
    check("state", state, want[1])


def test_refusals_on_tensors():
    x, y = layer(10, 1, 2, 1, 8, 8)
    a = {k: v.cuda() for k, v in x.items()}

    def refused(part, f, *args, **kw):
        with pytest.raises(B.AmpError) as e:
            f(*args, **kw)
        assert part in str(e.value), str(e.value)

    def with_(**kw):
        return {**a, **kw}.values()

    refused("k is", ops.gated_delta, *with_(k=a["k"][:, :4]), key_heads=1)
    refused("type", ops.gated_delta, *with_(v=a["v"].half()), key_heads=1)
    refused("decay is of type", ops.gated_delta, *with_(decay=a["decay"].half()), key_heads=1)
    refused("rows", ops.gated_delta, *with_(v=a["v"][:5]), key_heads=1)
    refused("key heads", ops.gated_delta, *a.values(), key_heads=3)
    refused("divide", ops.gated_delta, *a.values(), key_heads=4)
    refused("not on a GPU", ops.gated_delta, *with_(q=x["q"]), key_heads=1)
    refused("h0", ops.gated_delta, *a.values(), key_heads=1, h0=torch.zeros(1, 2, 8, 7, device="cuda"))
    refused("dk", ops.gated_delta, *with_(q=torch.zeros(10, 129, device="cuda"), k=torch.zeros(10, 129, device="cuda")), key_heads=1)
    refused("overlaps", ops.gated_delta, *a.values(), key_heads=1, out=a["v"])
    refused("requires grad", ops.gated_delta, *with_(q=a["q"].clone().requires_grad_()), key_heads=1)
    o, _, carry = ops.gated_delta(*a.values(), key_heads=1, carry=True)
    refused("carry", ops.gated_delta_backward, o, *a.values(), None, key_heads=1)
    refused("carry", ops.gated_delta_backward, o, *a.values(), carry[:-1], key_heads=1)
    refused("five", ops.gated_delta_backward, o, *a.values(), carry, key_heads=1, out=(o, o))
    refused("state", ops.gated_delta_step, *a.values(), torch.zeros(10, 2, 8, 9, device="cuda"), key_heads=1)
    refused("state", ops.gated_delta_step, *a.values(), torch.zeros(10, 2, 8, 8, device="cuda").transpose(2, 3), key_heads=1)
    refused("state", ops.gated_delta_step, *a.values(), torch.zeros(1, 2, 8, 8, device="cuda").expand(10, 2, 8, 8), key_heads=1)
    p, r = tokens(4, 9)
    p = {k: v.cuda() for k, v in p.items()}
    refused("index", ops.policy_loss, p["logits"], p["index"].float(), p["old"], p["advantage"])
    refused("advantage", ops.policy_loss, p["logits"], p["index"], p["old"], None)
    refused("old", ops.policy_loss, p["logits"], p["index"], p["old"][:3], p["advantage"])
    refused("clip_low", ops.policy_loss, p["logits"], p["index"], p["old"], p["advantage"], clip=(1.5, 0.2))
    refused("clip", ops.policy_loss, p["logits"], p["index"], p["old"], p["advantage"], clip=(1, 2, 3))
    refused("temperature", ops.policy_loss, p["logits"], p["index"], p["old"], p["advantage"], temperature=0.0)
    refused("kl", ops.policy_loss, p["logits"], p["index"], p["old"], p["advantage"], kl=NAN)
    refused("grad", ops.policy_loss, p["logits"], p["index"], p["old"], p["advantage"], grad=False, out=p["logits"])
    refused("index", ops.token_logprob, p["logits"], p["index"][:2])
    g = [torch.ones(5, device="cuda"), torch.ones(4, 4, device="cuda")]
    refused("no gradients", ops.clip_gradients, [])
    refused("contiguous", ops.clip_gradients, [g[1].T[1:]])
    refused("contiguous", ops.clip_gradients, [g[0], torch.ones(3)])
    refused("contiguous", ops.clip_gradients, [g[0].double()])
    refused("max_norm", ops.clip_gradients, g, -1.0)
    refused("out", ops.clip_gradients, g, out=g)
    refused("sizes", ops.clip_gradients, g, 1.0, out=g[:1])
    refused("types", ops.clip_gradients, g, 1.0, out=[torch.ones_like(t, dtype=torch.half) for t in g])
    refused("not a tensor", ops.clip_gradients, [g[0], 1.0])
    refused("overlaps", ops.clip_gradients, [g[0], g[0]], 1.0)
    refused("overlaps", ops.clip_gradients, [g[0][:3], g[0][2:]], 1.0)
    refused("requires grad", ops.clip_gradients, [g[0].clone().requires_grad_()])
    assert ops.clip_gradients([g[0], g[0]]) == math.sqrt(10)   # without results the same tensor counts twice
