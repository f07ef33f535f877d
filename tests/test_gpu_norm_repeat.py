"""Gradients of block norms call after call with the same bits, in the forms whose rows stay longest in the ring in shared memory: a gradient of h beside the
branch, two pieces of channels per thread, fp32 rows, d_h that does not go through the ring.  A row that the next batch replaced too early would
differ from call to call."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("S,C,dtype,stream,post,mod", [
    (20000, 1536, "bf16", "bf16", "none", 640), (20000, 1536, "bf16", "f32", "layer", 0), (6000, 5128, "bf16", "bf16", "none", 0),
    (4000, 8192, "bf16", "f32", "rms", 500), (3000, 7112, "f32", "f32", "none", 0), (60000, 72, "f32", "f32", "none", 1000),
])
def test_gradients(S, C, dtype, stream, post, mod):
    g = torch.Generator(device="cuda").manual_seed(C)
    r = lambda dt, *s: torch.randn(s, generator=g, device="cuda").to(dt)
    h, d_h, y, d = r(DT[stream], 1, S, C), r(DT[stream], 1, S, C), r(DT[dtype], 1, S, C), r(DT[dtype], 1, S, C)
    op = BlockNorm(vb.make_norm_shape(1, S, C, dtype, stream, "layer", post, mod))
    p = {n: r(torch.float32, 1, op.shape.groups, C) for n in ("gate", "scale", "shift")}

    def call():
        dx, dy = torch.empty_like(h), torch.empty_like(y)
        got = op.backward(d, h, dx, d_h, y, dy, **p)
        out, total = torch.empty_like(d), torch.empty_like(h)
        op.forward(h, out, y, total, **p)
        return [dx, dy, out, total, *(t for t in got.values() if t is not None)]

    want = call()
    for i in range(6):
        for a, b in zip(call(), want):
            assert torch.equal(a, b)
        if i % 2:
            torch.cuda.synchronize()
    op.check_status()
