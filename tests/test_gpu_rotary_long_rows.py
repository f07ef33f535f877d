"""Rows whose sums of the weights' gradient have no room in shared memory (more than 51,200 channels), and the longest that have.  Tolerances:
test_gpu_rotary.py."""
import pytest
import torch

from tests import _plain64 as P
from tests.test_gpu_rotary import case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,d,dtype,layout,pairs", [(400, 128, "bf16", "interleaved", (64,)), (401, 128, "bf16", "half", (22, 21, 21)),
                                                        (403, 128, "f32", "half", (64,)), (810, 64, "f32", "interleaved", (13,))])
def test_backward_of_long_rows(heads, d, dtype, layout, pairs):
    shape, op, x, dy, w, pos, f, axis, m = case(2, heads, d, (2, 3, 5), (1, 3, 5), dtype, pairs, "row", layout, seed=heads)
    xs, dys, ws = [t.cuda() for t in x], [t.cuda() for t in dy], [t.cuda() for t in w]
    out, dx = [torch.empty_like(t) for t in xs], [torch.empty_like(t) for t in xs]
    op.forward(xs, out, ws)
    dw = op.backward(dys, xs, dx, ws)
    for k in range(2):
        check(out[k], *P.norm_rotate(x[k], w[k], pos, f, axis, layout, "row", m), 5e-6, f"y {k}")
        (ref, mag), wref = P.norm_rotate_grad(dy[k], x[k], w[k], pos, f, axis, layout, "row", m)
        check(dx[k], ref, mag, 5e-6, f"dx {k}")
        check(dw[k], *wref, 1.3e-5, f"dw {k}")
    again = op.backward(dys, xs, dys, ws)
    assert all(torch.equal(a, b) for a, b in zip(again + dys, dw + dx))
