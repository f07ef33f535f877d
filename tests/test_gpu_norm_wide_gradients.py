"""Gradients of block norms at every number of channels, in fp32 with a branch and a gradient of h: the largest rows that the kernel's ring in shared
memory has to hold beside the threads' parts of sums.  Against the 64-bit statement, whose bounds of 32-bit arithmetic stand there."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm
from tests import _block64 as P

pytestmark = pytest.mark.gpu


def gradients(C, dtype, stream, post, S=5):
    g = torch.Generator(device="cuda").manual_seed(C)
    T = {"bf16": torch.bfloat16, "f32": torch.float32}
    r = lambda dt, *s: torch.randn(s, generator=g, device="cuda").to(dt)
    h, d_h, y, d = r(T[stream], 1, S, C), r(T[stream], 1, S, C), r(T[dtype], 1, S, C), r(T[dtype], 1, S, C)
    gate = r(torch.float32, 1, 1, C)
    op = BlockNorm(vb.make_norm_shape(1, S, C, dtype, stream, "layer", post))
    dx, dy = torch.empty_like(h), torch.empty_like(y)
    got = op.backward(d, h, dx, d_h, y, dy, gate=gate)
    p = {n: None for n in ("scale", "shift", "weight", "bias", "post_weight")} | {"gate": gate.double()}
    want = P.block_norm_grad(d.double(), h.double(), d_h.double(), y.double(), "layer", post, p, 0)
    for what, a in (("dx", dx), ("dy", dy), ("dgate", got["dgate"])):
        ref, err = want[what]
        half = torch.finfo(a.dtype).eps / 2
        off = (a.double() - ref).abs()
        assert bool((off <= half * ref.abs() + (1 + half) * err + torch.finfo(a.dtype).tiny).all()), f"{what} of {C} channels: {off.max():.3e}"
    op.check_status()


@pytest.mark.parametrize("C", [6872, 6880, 6888, 6896, 7000, 7096, 7104, 7112, 7120, 8184, 8192])
@pytest.mark.parametrize("dtype,stream,post", [("f32", "f32", "none"), ("f32", "f32", "layer"), ("bf16", "f32", "rms"), ("bf16", "bf16", "none")])
def test_wide_rows(C, dtype, stream, post):
    gradients(C, dtype, stream, post)


def test_every_width_in_fp32():
    for C in range(8, 8193, 8):
        gradients(C, "f32", "f32", "none", 3)
