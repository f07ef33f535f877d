"""Gradients of linear layers in bf16 on both sides of the bounds up to which what the rounding of du leaves goes on with it.  Below them du is held to
2^-16, above to half a step; results are rounded once more.  (A rounding is half a step of a number at most, evenly spread below that: its root mean
square is 2^-8 / sqrt(3) of a power of two at or below the number.)"""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import Linear
from tests import _block64 as P

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def run(S, K, N, act, gated, rounding):
    g = torch.Generator(device="cuda").manual_seed(S + K + N)
    r = lambda *s, by=1.0, dt=BF: (torch.randn(s, generator=g, device="cuda") * by).to(dt)
    wide = 2 * N if gated else N
    x, w, d, kept, gate = r(1, S, K), r(wide, K, by=K ** -0.5), r(1, S, N), r(1, S, wide), r(1, 1, N, dt=torch.float32)
    op, dx = Linear(vb.make_linear_shape(1, S, K, N, "bf16", act, gated, 0, 0)), torch.empty_like(x)
    dw = op.backward(d, x, w, dx, kept=kept, gate=gate)[0]
    (du, due), _ = P.du_of(d.double(), kept.double(), act, gated, gate.double(), 0, False)
    rounded = due + rounding * (du.abs() + due)
    for what, got, (ref, err) in (("dx", dx, P.input_grad(du, rounded, w.double())), ("dweight", dw, P.weight_grad(du, rounded, x.double()))):
        off, half = (got.double() - ref).abs(), 2.0 ** -8
        assert bool((off <= half * ref.abs() + (1 + half) * err + torch.finfo(BF).tiny).all()), what
        # one rounding, or two independent ones; a mean over 2,048 squares is a few hundredths off (1 / sqrt(2048) of their spread)
        times = 1 if rounding < 2.0 ** -10 else 2
        if got.numel() >= 2048:
            assert off.square().mean() <= times * 1.1 * (half ** 2 / 3) * ref.square().mean(), what
    op.check_status()


@pytest.mark.parametrize("S,K,N,act,gated", [
    (128, 256, 256, "none", False), (1, 2048, 2048, "none", False), (7, 1024, 4096, "silu", False), (8, 8, 8184, "none", False), (5, 512, 4096, "silu", True),
    (4096, 8, 8, "gelu", False), (64, 512, 256, "silu", True),
])
def test_within(S, K, N, act, gated):
    wide = 2 * N if gated else N
    assert S * (K + wide) <= 2 ** 16 and K * wide <= 2 ** 22 and wide <= 2 ** 13
    run(S, K, N, act, gated, 2.0 ** -16)


@pytest.mark.parametrize("S,K,N,act,gated", [
    (129, 256, 256, "none", False), (1, 2056, 2048, "none", False), (7, 1032, 4096, "silu", False), (4, 8, 8200, "none", False), (5, 520, 4096, "silu", True),
    (4097, 8, 8, "gelu", False), (65, 512, 256, "silu", True),
])
def test_beyond(S, K, N, act, gated):
    wide = 2 * N if gated else N
    assert S * (K + wide) > 2 ** 16 or K * wide > 2 ** 22 or wide > 2 ** 13
    run(S, K, N, act, gated, 2.0 ** -8)


def test_scratch_goes_by_the_same_bounds():
    du = lambda S, K, N: vb.linear_workspace_bytes(vb.make_linear_shape(1, S, K, N, "bf16"), True)
    # (one plane of 129 rows is smaller than two of 128; sums of slices and of columns are the same but for a few rows)
    assert du(128, 256, 256) - du(129, 256, 256) > 100 * 256 * 2
