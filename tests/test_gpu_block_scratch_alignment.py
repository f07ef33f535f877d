"""Linear layers, feed-forward blocks and block norms with scratch that begins on 16 bytes and on no more: what the interface asks of every pointer.  Results
as with scratch on 256 bytes, nothing written behind its stated size."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm, FeedForward, Linear

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class At:
    """Scratch that begins `off` bytes behind a 256-byte boundary, with bytes of a pattern behind it."""

    def __init__(self, op, off):
        self.off, self.given = off, []
        op._scratch = self

    def __call__(self, n):
        big = torch.full((self.off + n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        self.given.append((big, n))
        ws = big[self.off: self.off + n]
        assert ws.data_ptr() % 256 == self.off
        return ws

    def clean(self):
        return all(bool((big[self.off + n:] == 0xA5).all()) for big, n in self.given)


def same(make, run):
    res = []
    for off in (0, 16, 48):
        op = make()
        at = At(op, off)
        res.append(run(op))
        torch.cuda.synchronize()
        op.check_status()
        assert at.given and at.clean()
    for r in res[1:]:
        assert all(a is b or torch.equal(a, b) for a, b in zip(r, res[0]))


def rnd(dtype, *s, by=1.0):
    return (torch.randn(s, generator=torch.Generator().manual_seed(sum(s))) * by).to(DT[dtype]).cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,S,K,N,act,gated,heads,gt", [
    (1, 64, 5120, 520, "none", False, 0, -1),          # forward cut into slices
    (1, 300, 4104, 264, "silu", True, 0, 0),
    (2, 700, 128, 264, "none", False, 2, 100),         # weight gradients cut into slices, du in scratch
    (1, 40, 128, 72, "gelu", False, 0, 7),             # two planes
    (1, 2000, 1536, 1536, "none", False, 0, 0),
    (1, 1, 1024, 8, "none", False, 0, -1),
])
def test_linear(dtype, B, S, K, N, act, gated, heads, gt):
    shape = vb.make_linear_shape(B, S, K, N, dtype, act, gated, heads, max(gt, 0))
    x = rnd(dtype, B, heads, S, K // heads) if heads else rnd(dtype, B, S, K)
    w, d, kept = rnd(dtype, shape.wide, K, by=K ** -0.5), rnd(dtype, B, S, N), rnd(dtype, B, S, shape.wide)
    gate = rnd("f32", B, shape.groups, N) if gt >= 0 else None
    perm = torch.randperm(S, generator=torch.Generator().manual_seed(S)).to(torch.int32).cuda() if heads else None

    def run(op):
        out, dx = torch.empty_like(d), torch.empty_like(x)
        op.forward(x, w, out, gate=gate, perm=perm)
        return [out, dx, *op.backward(d, x, w, dx, kept=kept, gate=gate, perm=perm, with_bias=True)]

    same(lambda: Linear(shape), run)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,C,H,gated,gt", [(1, 64, 72, False, 0), (200, 264, 1544, True, 30), (1000, 1536, 520, False, -1)])
def test_feed_forward(dtype, S, C, H, gated, gt):
    make = lambda: FeedForward(1, S, C, H, dtype, "silu", gated, max(gt, 0))
    op = make()
    x, d, w1, w2 = rnd(dtype, 1, S, C), rnd(dtype, 1, S, C, by=2.0), rnd(dtype, op.shape.wide, C, by=C ** -0.5), rnd(dtype, C, H, by=H ** -0.5)
    gate = rnd("f32", 1, op.shape.groups, C) if gt >= 0 else None

    def run(op):
        out, dx, kept = torch.empty_like(x), torch.empty_like(x), op.keep()
        op.forward(x, w1, w2, out, gate=gate, kept=kept)
        return [out, dx, *op.backward(d, x, w1, w2, kept, dx, gate=gate, with_bias=True)]

    same(make, run)


@pytest.mark.parametrize("dtype,C", [("bf16", 72), ("f32", 1544)])
def test_block_norm(dtype, C):
    h, y, d, gate, weight = rnd(dtype, 1, 90, C), rnd(dtype, 1, 90, C, by=2.0), rnd(dtype, 1, 90, C, by=0.5), rnd("f32", 1, 9, C), rnd("f32", C)

    def run(op):
        dx, dy = torch.empty_like(h), torch.empty_like(y)
        return [dx, dy, *(g for g in op.backward(d, h, dx, y=y, dy_out=dy, gate=gate, weight=weight).values() if g is not None)]

    same(lambda: BlockNorm(vb.make_norm_shape(1, 90, C, dtype, mod_tokens=10)), run)
