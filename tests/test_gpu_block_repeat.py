"""Calls one behind another give the same bits, at sizes where a CTA takes many tiles: what a CTA reads of a box while the next one is on its way
would differ from call to call."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm, FeedForward, Linear

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
CALLS = 8


def rnd(g, *s, by=1.0, dt=BF):
    return (torch.randn(s, generator=g, device="cuda") * by).to(dt)


def same(call, what):
    """`call` gives new tensors; eight in a row, then eight with the device idle between them."""
    torch.cuda.synchronize()
    got = [call() for _ in range(CALLS)]
    torch.cuda.synchronize()
    for i in range(CALLS):
        got.append(call())
        torch.cuda.synchronize()
    for i, g in enumerate(got):
        for k, (a, b) in enumerate(zip(got[-1], g)):
            assert torch.equal(a, b), f"{what}: result {k} of call {i} differs at {(a != b).nonzero()[:4].tolist()}"


@pytest.mark.parametrize("seed", [0, 1, 2])
@pytest.mark.parametrize("gated", [True, False])
def test_feed_forward_gradients(gated, seed):
    B, S, C, H = 1, 13440, 1536, 4104
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = 2 * H if gated else H
    x, d, w1, w2 = rnd(g, B, S, C), rnd(g, B, S, C), rnd(g, wide, C, by=C ** -0.5), rnd(g, C, H, by=H ** -0.5)
    up = rnd(g, B, S, wide)
    op = FeedForward(B, S, C, H, "bf16", "silu" if gated else "gelu", gated, 0)

    def call():
        dx = torch.empty_like(x)
        return (dx, *[t for t in op.backward(d, x, w1, w2, (up, None), dx, with_bias=True) if t is not None])

    same(call, "gradients")
    op.check_status()


@pytest.mark.parametrize("act,gated,gt,residual", [("none", False, -1, False), ("gelu", False, -1, False), ("silu", True, -1, False), ("none", False, 640, True)])
def test_linear(act, gated, gt, residual):
    B, S, K, N = 1, 13440, 1536, 2312
    g = torch.Generator(device="cuda").manual_seed(N)
    wide = 2 * N if gated else N
    x, w, d = rnd(g, B, S, K), rnd(g, wide, K, by=K ** -0.5), rnd(g, B, S, N)
    res = rnd(g, B, S, N) if residual else None
    gate = rnd(g, B, -(-S // gt), N, dt=torch.float32) if gt >= 0 else None
    op = Linear(vb.make_linear_shape(B, S, K, N, "bf16", act, gated, 0, max(gt, 0)))

    def call():
        out, kept = torch.empty_like(d), torch.empty((B, S, wide), dtype=BF, device="cuda")
        op.forward(x, w, out, gate=gate, residual=res, kept=kept)
        return out, kept

    def back():
        dx = torch.empty_like(x)
        return (dx, *[t for t in op.backward(d, x, w, dx, kept=kept if act != "none" or gate is not None else None, gate=gate) if t is not None])

    same(call, "linear")
    kept = call()[1]
    same(back, "its gradients")
    op.check_status()


@pytest.mark.parametrize("post", ["none", "rms"])
def test_block_norm(post):
    B, S, C = 1, 13440, 1536
    op = BlockNorm(vb.make_norm_shape(B, S, C, "bf16", post_norm=post))
    g = torch.Generator(device="cuda").manual_seed(1)
    h, y, d = rnd(g, B, S, C), rnd(g, B, S, C), rnd(g, B, S, C)
    gate = rnd(g, B, 1, C, dt=torch.float32)

    def call():
        out, total = torch.empty_like(h), torch.empty_like(h)
        op.forward(h, out, y=y, h_out=total, gate=gate)
        return out, total

    def back():
        dx, dy = torch.empty_like(h), torch.empty_like(h)
        return dx, dy, op.backward(d, h, dx, y=y, dy_out=dy, gate=gate)["dgate"]

    same(call, "norm")
    same(back, "its gradients")
    op.check_status()
