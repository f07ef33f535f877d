"""The smallest feed-forward blocks and linear layers, whose h or partial sums are a few bytes: many calls on one object under way at the same time, on
two streams and in graphs, each with what it computes alone."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import FeedForward, Linear

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CALLS = 64


def ffn(rows, hidden, dtype, C=1536):
    op = FeedForward(1, rows, C, hidden, dtype, "silu")
    g = torch.Generator(device="cuda").manual_seed(hidden)
    r = lambda *s, by=1.0: (torch.randn(s, generator=g, device="cuda") * by).to(DT[dtype])
    w1, w2, xs = r(hidden, C, by=C ** -0.5), r(C, hidden), [r(1, rows, C) for _ in range(2)]
    return (lambda i, out: op.forward(xs[i], w1, w2, out)), (lambda: torch.empty_like(xs[0]))


def linear(K):
    op = Linear(vb.make_linear_shape(1, 1, K, 8, "f32"))
    g = torch.Generator(device="cuda").manual_seed(K)
    w, xs = torch.randn((8, K), generator=g, device="cuda"), [torch.randn((1, 1, K), generator=g, device="cuda") for _ in range(2)]
    return (lambda i, out: op.forward(xs[i], w, out)), (lambda: torch.empty((1, 1, 8), device="cuda"))


@pytest.mark.parametrize("make", [lambda: ffn(1, 128, "bf16"), lambda: ffn(16, 8, "bf16"), lambda: ffn(1, 64, "f32"), lambda: linear(1024), lambda: linear(256)],
                         ids=["ffn 1 x 128", "ffn 16 x 8", "ffn 1 x 64 fp32", "linear 1024", "linear 256"])
def test_calls_at_the_same_time(make):
    call, new = make()
    want = [new(), new()]
    for i in range(2):
        call(i, want[i])
    torch.cuda.synchronize()
    assert not torch.equal(*want)
    # two streams
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[new() for _ in range(CALLS)] for _ in range(2)]
    torch.cuda.synchronize()
    for k in range(CALLS):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                call(i, outs[i][k])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])
    # two graphs of one object, replayed together with eager calls
    graphs = []
    for i, st in enumerate(streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            for o in outs[i]:
                call(i, o)
        graphs.append(graph)
    for i in range(2):
        for o in outs[i]:
            o.zero_()
    eager = [new() for _ in range(CALLS)]
    torch.cuda.synchronize()
    for graph, st in zip(graphs, streams):
        with torch.cuda.stream(st):
            graph.replay()
    for o in eager:
        call(0, o)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in outs[i])
    assert all(torch.equal(o, want[0]) for o in eager)
