"""A Rotary serves every layer of a model: its backward calls on several streams, in captured graphs and of several numbers of tensors do not
meet in one scratch buffer.  (A result repeats bit for bit, so that each is compared with the call alone.)"""
import pytest
import torch

from tests.test_gpu_rotary import case

pytestmark = pytest.mark.gpu


def _make(n, norm="row", seed=40):
    shape, op, x, dy, w, *_ = case(1, 12, 128, (4, 24, 32), (1, 24, 32), "bf16", (22, 21, 21), norm, "interleaved", seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    mk = lambda: torch.randn(x[0].shape, generator=g, device="cuda").bfloat16()
    return op, [mk() for _ in range(n)], [mk() for _ in range(n)], [1 + 0.1 * torch.randn(op.n_weights, generator=g, device="cuda") for _ in range(n)]


@pytest.mark.parametrize("norm", ["row", "head"])
def test_backward_calls_on_several_streams(norm):
    op, x, dy, w = _make(8, norm)
    dx = [torch.empty_like(t) for t in x]
    pair = lambda i: (dy[2 * i : 2 * i + 2], x[2 * i : 2 * i + 2], dx[2 * i : 2 * i + 2], w[2 * i : 2 * i + 2])
    want = [op.backward(*pair(i)) for i in range(4)]
    keep = [t.clone() for t in dx]
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    got = [[] for _ in range(4)]
    for _ in range(10):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(op.backward(*pair(i)))
    torch.cuda.synchronize()
    for i in range(4):
        for dw in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(dw, want[i]))
    assert all(torch.equal(a, b) for a, b in zip(dx, keep))


def test_captured_backward_and_calls_of_more_tensors():
    """Two graphs of two tensors each, calls of one, three and four tensors ahead of their replays, and what the allocator hands out then
    filled: each gives what it gave alone, and nothing of what it does not own changes."""
    op, x, dy, w = _make(4)
    dx = [torch.empty_like(t) for t in x]
    want = [op.backward(dy[2 * i : 2 * i + 2], x[2 * i : 2 * i + 2], dx[2 * i : 2 * i + 2], w[2 * i : 2 * i + 2]) for i in range(2)]
    keep = [t.clone() for t in dx]
    # (a row of tokens is cut into as many sums as there are CTAs for a tensor, which follows from the number of tensors)
    alone = {n: op.backward(dy[:n], x[:n], [torch.empty_like(t) for t in x[:n]], w[:n]) for n in (1, 4, 3)}
    torch.cuda.synchronize()
    graphs, dws = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            dws.append(op.backward(dy[2 * i : 2 * i + 2], x[2 * i : 2 * i + 2], dx[2 * i : 2 * i + 2], w[2 * i : 2 * i + 2]))
        graphs.append(g)
    for n in (1, 4, 3):
        out = [torch.empty_like(t) for t in x[:n]]
        again = op.backward(dy[:n], x[:n], out, w[:n])
        assert all(torch.equal(a, b) for a, b in zip(again, alone[n])) and all(torch.equal(a, b) for a, b in zip(out, keep))
        del out, again
        others = [torch.full((1 << 20,), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
        for t in dx + dws[0] + dws[1]:
            t.fill_(3.0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert all(torch.equal(a, b) for a, b in zip(dws[i], want[i]))
        assert all(torch.equal(a, b) for a, b in zip(dx, keep))
        assert all(bool((t == 7).all()) for t in others)
