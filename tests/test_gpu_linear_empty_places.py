"""Places of a linear layer's input that no token leads to (padding of a block order): what forward() left in kept there may be anything, and has no part in any
gradient."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import Linear
from tests.test_gpu_linear import DT, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act,gated,gt", [("none", False, 0), ("gelu", False, -1), ("silu", True, 0), ("silu", True, 16), ("gelu", False, 7)])
def test_kept_of_places_without_a_token(dtype, act, gated, gt):
    B, S, heads, N, tokens = 2, 70, 1, 72, max(gt, 0)
    shape = vb.make_linear_shape(B, S, 128, N, dtype, act, gated, heads, tokens)
    op = Linear(shape)
    g = torch.Generator().manual_seed(N)
    x, w, d = (make(g, dtype, *s).cuda() for s in ((B, heads, S, 128), (shape.wide, 128), (B, S, N)))
    kept = make(g, dtype, B, S, shape.wide).cuda()
    gate = torch.randn((B, shape.groups, N), generator=g).cuda() if gt >= 0 else None
    perm = torch.randperm(S, generator=g).to(torch.int32)
    empty = torch.zeros(S, dtype=torch.bool)
    empty[[3, 9, 20, 64]] = True
    perm[empty] = torch.tensor([-5, S, 2 ** 30, -1], dtype=torch.int32)
    res = []
    for junk in (0.0, float("nan"), float("inf"), -float("inf"), 3e38):
        k = kept.clone()
        k[:, empty.cuda()] = junk
        dx = torch.full_like(x, 7.0)
        res.append((dx, *op.backward(d, x, w, dx, kept=k, gate=gate, perm=perm.cuda(), with_bias=True)))
        assert not bool(dx[:, :, empty.cuda()].any())
    for r in res:
        for a, b in zip(r, res[0]):
            assert a is b or (bool(a.isfinite().all()) and torch.equal(a, b))
    op.check_status()
    assert DT[dtype] is x.dtype
