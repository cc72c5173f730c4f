"""GPU: a training step and single rows of the operators on streams of their own and in HIP graphs.  Behind the other tests, as
test_zz_operator_streams is."""
import pytest
import torch

from paper_1705_09786_amd import operators as ops
from test_gpu_operators import same_bits
from test_gpu_operators_more import problem, train_step

pytestmark = pytest.mark.gpu


def everything(s, c):
    """A training step, the log-probabilities alone, and a row for every sequence."""
    kh, dk, heads, dv = c["key_heads"], c["dk"], c["heads"], c["dv"]
    got = train_step(s, c)
    p = (s["x"][:4] @ s["wx"]).to(c["dtype"]).split([kh * dk, kh * dk, heads * dv], 1)
    state = torch.ones(4, heads, dk, dv, device="cuda")
    o = ops.gated_delta_step(p[0] * 0.2, p[1] * 0.2, p[2], s["decay"][:4], s["beta"][:4], state, key_heads=kh)
    return got + [o, state, ops.token_logprob(s["x"], s["index"] % 32)]


def test_other_streams_and_two_calls_at_once():
    s = [{k: v.cuda() for k, v in problem(k)[0].items()} for k in range(2)]
    c = problem(0)[1]
    want = [everything(m, c) for m in s]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = everything(s[k], c)
    torch.cuda.synchronize()
    for k in range(2):
        assert all(same_bits(p, q) for p, q in zip(got[k], want[k]))


def test_captured_and_replayed():
    """Captured once, replayed with other inputs, eager work between the replays; two graphs side by side."""
    s = [{k: v.cuda() for k, v in problem(k)[0].items()} for k in range(3)]
    c = problem(0)[1]
    want = [everything(m, c) for m in s]
    buffers = [{k: v.clone() for k, v in s[0].items()} for _ in range(2)]
    graphs, outs = [], []
    for b in buffers:
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            everything(b, c)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            outs.append(everything(b, c))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(4):
        use = (turn % 3, (turn + 1) % 3)
        for b, u in zip(buffers, use):
            for k in b:
                b[k].copy_(s[u][k])
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for o, u in zip(outs, use):
            assert all(same_bits(p, q) for p, q in zip(o, want[u])), turn
        again = everything(s[turn % 3], c)
        assert all(same_bits(p, q) for p, q in zip(again, want[turn % 3]))
