"""Norms without an eps: the gradients stay finite where no real row or head is zero.  Tolerances: test_gpu_rotary.py."""
import pytest
import torch

from paper_2506_23858_b200.layer import Rotary
from tests import _plain64 as P
from tests.test_gpu_rotary import case, check

pytestmark = pytest.mark.gpu

# rows that do not fill the vectors of their warps: all pairs, a part of them, halves that are not whole vectors; more vectors than the
# registers of a CTA hold
SHAPES = [
    dict(heads=5, d=128, dtype="bf16", pairs=(22, 21, 21), layout="interleaved"),
    dict(heads=3, d=64, dtype="f32", pairs=(32,), layout="half"),
    dict(heads=9, d=64, dtype="bf16", pairs=(5,), layout="half"),
    dict(heads=50, d=128, dtype="bf16", pairs=(16,), layout="half"),
    dict(heads=61, d=64, dtype="f32", pairs=(7, 6), layout="half"),
    dict(heads=100, d=64, dtype="f32", pairs=(32,), layout="interleaved"),
]


@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_gradients_without_eps(i, norm):
    c = SHAPES[i]
    shape, _, x, dy, w, pos, f, axis, m = case(B=2, grid=(2, 3, 5), block=(2, 3, 5), norm=norm, seed=30 + i, **c)
    op = Rotary(shape, pos.cuda(), f.cuda(), axis.cuda(), layout=c["layout"], norm=norm, mscale=m, eps=0.0, with_backward=True)
    xs, dys, ws = [t.cuda() for t in x], [t.cuda() for t in dy], [t.cuda() for t in w]
    out, dx = [torch.empty_like(t) for t in xs], [torch.empty_like(t) for t in xs]
    op.forward(xs, out, ws)
    dw = op.backward(dys, xs, dx, ws)
    for k in range(2):
        check(out[k], *P.norm_rotate(x[k], w[k], pos, f, axis, c["layout"], norm, m, 0.0), 5e-6, f"y {k}")
        (ref, mag), wref = P.norm_rotate_grad(dy[k], x[k], w[k], pos, f, axis, c["layout"], norm, m, 0.0)
        check(dx[k], ref, mag, 5e-6, f"dx {k}")
        check(dw[k], *wref, 1.3e-5, f"dw {k}")
