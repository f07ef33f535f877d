"""One Rotary for layers of several block shapes over the same tokens: the block order is the layer's."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import Rotary, SteppedAttention, VmobaLayer, default_capacity, rotary_frequencies

pytestmark = pytest.mark.gpu
GRID = (4, 8, 8)


def _rotary(heads, d, dtype, grid, block, norm, batch=1):
    shape = vb.make_shape(batch, heads, d, grid, block, dtype)
    f, axis, _ = rotary_frequencies((d // 2 - 2 * (d // 6), d // 6, d // 6))
    at = torch.arange(shape.S)
    pos = torch.stack([at // 64, at // 8 % 8, at % 8], 1).to(torch.int32)
    return Rotary(shape, pos.cuda(), f.cuda(), axis.cuda(), norm=norm, with_backward=True)


@pytest.mark.parametrize("dtype,d,norm", [("bf16", 128, "row"), ("f32", 64, "head")])
@pytest.mark.parametrize("block", [(1, 8, 8), (4, 4, 4), (2, 8, 2)])
def test_layers_of_other_block_shapes(block, dtype, d, norm):
    g = torch.Generator().manual_seed(7)
    rot = _rotary(3, d, dtype, GRID, (4, 8, 8), norm)
    mk = lambda: torch.randn((1, 256, 3, d), generator=g).cuda().to(rot.dtype)
    q, k, v, do = mk(), mk(), mk(), mk()
    ws = [1 + 0.2 * torch.randn(rot.n_weights, generator=g).cuda() for _ in range(2)]
    shape = vb.make_shape(1, 3, d, GRID, block, dtype)
    A, Bl = (VmobaLayer(shape, default_capacity(shape, 0.4), with_backward=True) for _ in range(2))
    o1, o2 = torch.empty_like(q), torch.empty_like(q)
    g1, g2 = [[torch.empty_like(q) for _ in range(3)] for _ in range(2)]
    A.forward(q, k, v, 0.4, o1, rotary=rot, weights=ws)
    A.check_status()
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    rot.forward((q, k), (qr, kr), ws)
    Bl.forward(qr, kr, v, 0.4, o2)
    assert torch.equal(A.perm, Bl.perm) and torch.equal(A.q_bm, Bl.q_bm) and torch.equal(A.k_bm, Bl.k_bm) and torch.equal(A.v_bm, Bl.v_bm)
    assert torch.equal(o1, o2)
    dw1 = A.backward(do, *g1, rotary=rot, qk=(q, k), weights=ws)
    Bl.backward(do, *g2)
    dw2 = rot.backward(g2[:2], (q, k), g2[:2], ws)
    assert torch.equal(g1[1], g2[1]) and torch.equal(g1[2], g2[2]) and torch.equal(dw1[1], dw2[1])
    for a, b in ((g1[0], g2[0]), (dw1[0], dw2[0])):       # (dq is added up in any order: equal to rounding)
        assert (a.float() - b.float()).norm() <= 2e-2 * b.float().norm()
    # the dense steps of a sampler over the same layer
    o3, o4 = torch.empty_like(q), torch.empty_like(q)
    step = SteppedAttention(A, 0.4, 4)
    assert step.forward(0, q, k, v, o3, rotary=rot, weights=ws) == step.forward(0, qr, kr, v, o4) == "dense"
    assert torch.equal(o3, o4)


def test_a_shape_of_other_sizes_is_refused():
    rot = _rotary(3, 64, "f32", GRID, (1, 8, 8), "row")
    x, out = torch.randn((1, 256, 3, 64), device="cuda"), torch.full((1, 3, 256, 64), 2.0, device="cuda")
    before = vb.kernel_launches()
    for args in ((1, 3, 64, (8, 8, 8), (1, 8, 8), "f32"), (2, 3, 64, GRID, (1, 8, 8), "f32"), (1, 4, 64, GRID, (1, 8, 8), "f32"),
                 (1, 3, 128, GRID, (1, 8, 8), "f32"), (1, 3, 64, GRID, (1, 8, 8), "bf16")):
        shape = vb.make_shape(*args)
        for order, dst in ((True, out), (False, torch.empty_like(x))):
            with pytest.raises(ValueError):
                rot.forward((x,), (dst,), block_order=order, shape=shape)
        with pytest.raises(ValueError):
            rot.backward((out,), (x,), (torch.empty_like(x),), block_order=True, shape=shape)
        if shape.B == 1 and shape.S == 256:
            layer = VmobaLayer(shape, default_capacity(shape, 0.4))
            y = torch.empty((1, 256, shape.heads, shape.head_dim), dtype=layer.q_bm.dtype, device="cuda")
            with pytest.raises(ValueError):
                layer.forward(y, y, y, 0.4, torch.empty_like(y), rotary=rot)
    assert vb.kernel_launches() == before and bool((out == 2).all())


def test_a_permutation_table_that_does_not_hold_the_tokens_is_refused():
    rot = _rotary(3, 64, "f32", GRID, (1, 8, 8), "row")
    x, out = torch.randn((1, 256, 3, 64), device="cuda"), torch.empty((1, 3, 256, 64), device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    before = vb.kernel_launches()
    for bad in (torch.empty(255, **i32), torch.empty(256, dtype=torch.int64, device="cuda"), torch.empty(512, **i32)[::2],
                torch.empty(256, dtype=torch.int32)):
        with pytest.raises(ValueError):
            rot.forward((x,), (out,), block_order=True, perm=bad)
    assert vb.kernel_launches() == before
    for shape in ((256,), (1, 256), (300,)):
        perm = torch.full(shape, -1, **i32)
        rot.forward((x,), (torch.empty_like(x),), perm=perm)             # (raster order: the table alone)
        perm = perm.flatten()
        assert torch.equal(perm[:256].sort().values, torch.arange(256, **i32)) and bool((perm[256:] == -1).all())
