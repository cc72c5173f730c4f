"""GPU: the operators on whole arrays on streams of their own and in HIP graphs.  Behind the other tests, which ask for the dies that the
first hardware queue starts at: once there are streams, the default one may be served by another queue."""
import pytest
import torch

from test_gpu_operators import everything, model, same_bits

pytestmark = pytest.mark.gpu


def test_other_streams_and_two_calls_at_once():
    s = [{k: v.cuda() for k, v in model(seed=k).items()} for k in range(2)]
    want = [everything(m) for m in s]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(3):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = everything(s[k])
    torch.cuda.synchronize()
    for k in range(2):
        assert all(same_bits(p, q) for p, q in zip(got[k], want[k]))


def test_captured_and_replayed():
    """Captured once, replayed with other inputs, eager work between the replays; two graphs side by side."""
    s = [{k: v.cuda() for k, v in model(seed=k).items()} for k in range(3)]
    want = [everything(m) for m in s]
    buffers = [{k: v.clone() for k, v in s[0].items()} for _ in range(2)]
    graphs, outs = [], []
    for b in buffers:
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            everything(b)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            outs.append(everything(b))
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
        again = everything(s[turn % 3])
        assert all(same_bits(p, q) for p, q in zip(again, want[turn % 3]))
