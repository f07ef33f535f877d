"""Rotary positions with norm on the GPU against the 64-bit statement.

Tolerances.  A result is rounded once to its type: half a step, finfo.eps / 2 of it.  Ahead of that stands 32-bit arithmetic.  An angle is exact
to 2^-24 pi (its reduction is rounded to 32 bits) plus what sincosf adds (2 units in the last place): 4e-7 of the magnitudes turned.  A mean of
squares, or of products, is a sum of at most 64 terms per thread and a tree of at most 8 more additions: 72 x 2^-24 = 4.3e-6 relative to the
magnitudes added, half of that through the square root; five more roundings 3e-7.  5e-6 of the magnitudes covers each.  dw adds at most 128
tokens per thread in 32 bits ahead of the 64-bit sum: 128 x 2^-24 = 7.6e-6 on top, 1.3e-5 of the magnitudes."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import Rotary, SteppedAttention, VmobaLayer, default_capacity, rotary_frequencies
from tests import _plain64 as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(got, ref, mag, rel, what):
    half = torch.finfo(got.dtype).eps / 2
    err = (got.detach().double().cpu() - ref).abs()
    tol = half * ref.abs() + rel * (1 + half) * mag
    assert bool((err <= tol).all()), f"{what}: {err.max():.3e}, worst over its tolerance {(err / tol.clamp(min=1e-300)).max():.2f}"


def case(B, heads, d, grid, block, dtype, pairs, norm, layout, batch_pos=False, seed=0, big=False, weight=True, scaling="none"):
    g = torch.Generator().manual_seed(seed)
    S = grid[0] * grid[1] * grid[2]
    shape = vb.make_shape(B, heads, d, grid, block, dtype)
    f, axis, m = rotary_frequencies(pairs, scaling=scaling, factor=1.0 if scaling == "none" else 4.0)
    hi = 2 ** 31 - 1 if big else 4000
    pos = torch.randint(-3 if not big else 2 ** 30, hi, ((B, S, len(pairs)) if batch_pos else (S, len(pairs))), generator=g, dtype=torch.int64).to(torch.int32)
    n = {"none": 0, "head": d, "row": heads * d}[norm]
    mk = lambda: torch.randn((B, S, heads, d), generator=g).to(DT[dtype])
    x, dy = [mk(), mk()], [mk(), mk()]
    w = [1 + 0.2 * torch.randn(n, generator=g) if n and (weight or i == 0) else None for i in range(2)]
    op = Rotary(shape, pos.cuda(), f.cuda(), axis.cuda(), layout=layout, norm=norm, mscale=m, with_backward=True)
    return shape, op, x, dy, w, pos, f, axis, m


CASES = [
    # one token; a few; odd heads, grids and head parts; vectors that are not whole pairs; every norm, layout and type
    dict(B=1, heads=1, d=128, grid=(1, 1, 1), block=(1, 1, 1), dtype="bf16", pairs=(64,), norm="row", layout="half"),
    dict(B=1, heads=12, d=128, grid=(1, 1, 1), block=(1, 1, 1), dtype="bf16", pairs=(22, 21, 21), norm="row", layout="interleaved"),
    dict(B=2, heads=5, d=64, grid=(2, 3, 5), block=(1, 3, 5), dtype="f32", pairs=(5,), norm="none", layout="half"),
    dict(B=2, heads=5, d=64, grid=(2, 3, 5), block=(2, 3, 1), dtype="bf16", pairs=(7, 6), norm="head", layout="half"),
    dict(B=3, heads=3, d=64, grid=(3, 4, 5), block=(3, 2, 5), dtype="bf16", pairs=(32,), norm="row", layout="half", batch_pos=True),
    dict(B=1, heads=7, d=128, grid=(4, 6, 9), block=(2, 3, 3), dtype="f32", pairs=(10, 11, 11), norm="head", layout="interleaved"),
    dict(B=1, heads=13, d=128, grid=(3, 7, 11), block=(1, 7, 11), dtype="bf16", pairs=(16,), norm="row", layout="interleaved", scaling="parts"),
    dict(B=1, heads=40, d=128, grid=(3, 5, 8), block=(3, 5, 4), dtype="bf16", pairs=(22, 21, 21), norm="row", layout="interleaved"),
    dict(B=1, heads=40, d=128, grid=(2, 5, 8), block=(1, 5, 8), dtype="f32", pairs=(64,), norm="row", layout="half"),
    # a row of more vectors than the warps of a CTA hold at a time (the row is read twice)
    dict(B=1, heads=70, d=128, grid=(2, 2, 3), block=(2, 2, 3), dtype="f32", pairs=(64,), norm="row", layout="half"),
    dict(B=1, heads=3, d=128, grid=(5, 30, 40), block=(5, 6, 8), dtype="bf16", pairs=(0,), norm="head", layout="half"),
    dict(B=1, heads=2, d=64, grid=(1, 9, 9), block=(1, 3, 9), dtype="f32", pairs=(32,), norm="none", layout="interleaved", big=True),
    dict(B=1, heads=4, d=64, grid=(1, 9, 9), block=(1, 3, 9), dtype="f32", pairs=(1, 1, 1, 1), norm="row", layout="half", weight=False),
    # rows too long for the registers of a thread: of the backward, of both
    dict(B=2, heads=60, d=128, grid=(1, 2, 9), block=(1, 2, 3), dtype="bf16", pairs=(22, 21, 21), norm="row", layout="interleaved"),
    dict(B=1, heads=101, d=128, grid=(1, 5, 3), block=(1, 5, 3), dtype="bf16", pairs=(20, 21), norm="row", layout="interleaved"),
    dict(B=2, heads=100, d=128, grid=(1, 2, 9), block=(1, 2, 3), dtype="bf16", pairs=(13,), norm="head", layout="half", batch_pos=True),
    dict(B=1, heads=130, d=128, grid=(2, 3, 3), block=(1, 3, 3), dtype="bf16", pairs=(64,), norm="none", layout="half"),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_and_backward(i):
    c = CASES[i]
    shape, op, x, dy, w, pos, f, axis, m = case(**c, seed=i)
    xs, dys = [t.cuda() for t in x], [t.cuda() for t in dy]
    ws = [None if t is None else t.cuda() for t in w]
    ref = [P.norm_rotate(x[k], w[k], pos, f, axis, c["layout"], c["norm"], m) for k in range(2)]
    # raster order, strided output with space between the rows, which stays as it was
    out = [torch.full((shape.B, shape.S, shape.heads + 1, 2 * shape.head_dim), 7.0, dtype=xs[0].dtype, device="cuda") for _ in range(2)]
    view = [t[:, :, 1:, : shape.head_dim] for t in out]
    op.forward(xs, view, ws)
    for k in range(2):
        check(view[k], *ref[k], 5e-6, f"raster {k}")
        assert bool((out[k][:, :, 0] == 7).all()) and bool((out[k][..., shape.head_dim:] == 7).all())
    # block order, with a third tensor that only moves, and the permutation
    bm = [torch.empty((shape.B, shape.heads, shape.S, shape.head_dim), dtype=xs[0].dtype, device="cuda") for _ in range(3)]
    perm = torch.empty(shape.S, dtype=torch.int32, device="cuda")
    op.forward(xs, bm[:2], ws, block_order=True, moved=(dys[0],), moved_outs=(bm[2],), perm=perm)
    for k in range(2):
        assert torch.equal(bm[k].cpu(), P.block_order(view[k].cpu(), c["grid"], c["block"]))
    assert torch.equal(bm[2].cpu(), P.block_order(dy[0], c["grid"], c["block"]))
    assert torch.equal(dys[0][:, perm.long()].transpose(1, 2), bm[2])
    # gradients: from raster order, in place, and from block order
    got = [torch.empty_like(t) for t in xs]
    dw = op.backward(dys, xs, got, ws)
    for k in range(2):
        (dx, mag), wref = P.norm_rotate_grad(dy[k], x[k], w[k], pos, f, axis, c["layout"], c["norm"], m)
        check(got[k], dx, mag, 5e-6, f"dx {k}")
        if wref is None:
            assert dw is None
        else:
            check(dw[k], *wref, 1.3e-5, f"dw {k}")
    again = [t.clone() for t in dys]
    dw2 = op.backward(again, xs, again, ws)
    gbm = [P.block_order(t, c["grid"], c["block"]).cuda().contiguous() for t in dy]
    third = [torch.empty_like(t) for t in xs]
    op.backward(gbm, xs, third, ws, block_order=True)
    for k in range(2):
        assert torch.equal(again[k], got[k]) and torch.equal(third[k], got[k])
        assert dw is None or torch.equal(dw[k], dw2[k])
    # forward in place
    op.forward(xs, xs, ws)
    for k in range(2):
        assert torch.equal(xs[k], view[k])


def test_expanded_inputs_and_qkv_slices():
    """Heads that share memory (stride 0) as input, and q, k as slices of one projection."""
    shape, op, x, dy, w, pos, f, axis, m = case(2, 4, 64, (2, 4, 4), (1, 4, 4), "bf16", (32,), "row", "half", seed=5)
    one = x[0][:, :, :1].cuda().expand(-1, -1, 4, -1)
    qkv = torch.stack([x[0], x[1], dy[0]], 2).cuda()
    outs = [torch.empty_like(x[0], device="cuda") for _ in range(2)]
    op.forward((one, qkv[:, :, 1]), outs, [t.cuda() for t in w])
    check(outs[0], *P.norm_rotate(x[0][:, :, :1].expand(-1, -1, 4, -1), w[0], pos, f, axis, "half", "row"), 5e-6, "expanded")
    check(outs[1], *P.norm_rotate(x[1], w[1], pos, f, axis, "half", "row"), 5e-6, "slice")


def test_refused_calls_launch_nothing():
    shape, op, x, dy, w, *_ = case(1, 2, 64, (2, 2, 2), (1, 2, 2), "f32", (32,), "row", "half")
    xs = [t.cuda() for t in x]
    before = vb.kernel_launches()
    for bad in (xs[0].bfloat16(), xs[0][:, :4], x[0], xs[0].transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(ValueError):
            op.forward((bad,), (xs[0],))
        with pytest.raises(ValueError):
            op.forward((xs[0],), (bad,))
    with pytest.raises(ValueError):
        op.forward(xs, xs, [torch.ones(5, device="cuda"), None])
    with pytest.raises(ValueError):
        op.backward(xs, None, xs)
    with pytest.raises(vb.VmobaError):
        op.forward((xs[0],), (xs[1][:, :, :1].expand(-1, -1, 2, -1),))       # an output whose heads share memory
    with pytest.raises(ValueError):
        Rotary(shape, torch.zeros((8, 1), device="cuda"), torch.ones(4, dtype=torch.float64, device="cuda"),
               torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert vb.kernel_launches() == before


def test_layer_with_rotary_equals_rotary_ahead_of_the_layer():
    """VmobaLayer.forward / backward with a Rotary against the operators called one by one, bf16 and fp32, and the dense step."""
    for dtype, d, norm in (("bf16", 128, "row"), ("f32", 64, "head")):
        shape, op, x, dy, w, *_ = case(1, 3, d, (4, 8, 8), (2, 4, 4), dtype, (12, 10, 10), norm, "interleaved", seed=3)
        q, k, v, do = x[0].cuda(), x[1].cuda(), dy[0].cuda(), dy[1].cuda()
        ws = [t.cuda() for t in w]
        mk = lambda: VmobaLayer(shape, default_capacity(shape, 0.4), with_backward=True)
        A, Bl = mk(), mk()
        o1, o2 = torch.empty_like(q), torch.empty_like(q)
        g1, g2 = [[torch.empty_like(q) for _ in range(3)] for _ in range(2)]
        A.forward(q, k, v, 0.4, o1, rotary=op, weights=ws)
        dw1 = A.backward(do, *g1, rotary=op, qk=(q, k), weights=ws)
        qr, kr = torch.empty_like(q), torch.empty_like(k)
        op.forward((q, k), (qr, kr), ws)
        Bl.forward(qr, kr, v, 0.4, o2)
        Bl.backward(do, *g2)
        half = [torch.empty_like(q) for _ in range(2)]
        dw2 = op.backward(g2[:2], (q, k), half, ws)
        assert torch.equal(o1, o2) and torch.equal(g1[2], g2[2])
        A.check_status()
        for a, b in zip(g1[:2] + dw1, half + dw2):       # (dq is added up in the order of the CTAs: equal to rounding)
            assert (a.float() - b.float()).norm() <= 2e-2 * b.float().norm()
        assert torch.equal(g1[1], half[1]) and torch.equal(dw1[1], dw2[1])
        o3, o4 = torch.empty_like(q), torch.empty_like(q)
        step = SteppedAttention(A, 0.4, 4)
        assert step.forward(0, q, k, v, o3, rotary=op, weights=ws) == step.forward(0, qr, kr, v, o4) == "dense"
        assert torch.equal(o3, o4)
        assert step.forward(3, q, k, v, o3, rotary=op, weights=ws) == "sparse" and torch.equal(o3, o1)


def test_captured_and_on_another_stream():
    shape, op, x, dy, w, pos, f, axis, m = case(1, 6, 128, (3, 5, 7), (1, 5, 7), "bf16", (22, 21, 21), "row", "interleaved", seed=9)
    xs, dys, ws = [t.cuda() for t in x], [t.cuda() for t in dy], [t.cuda() for t in w]
    out, dx = [torch.empty_like(t) for t in xs], [torch.empty_like(t) for t in xs]
    op.forward(xs, out, ws)
    dw = op.backward(dys, xs, dx, ws)
    want = [t.clone() for t in out + dx + dw]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in out + dx:
            t.zero_()
        op.forward(xs, out, ws)
        dw = op.backward(dys, xs, dx, ws)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out + dx + dw, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(xs, out, ws)
        dw = op.backward(dys, xs, dx, ws)
    for t in out + dx + dw:
        t.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out + dx + dw, want))


@pytest.mark.parametrize("norm", ["none", "head", "row"])
@pytest.mark.parametrize("layout", ["interleaved", "half"])
def test_what_is_not_finite_stays_where_it_is(layout, norm):
    """Channels that no pair holds pass through whatever stands beside them; a row (norm per head: a head) that holds no such value keeps its
    bits."""
    shape, op, x, dy, w, *_ = case(1, 3, 64, (1, 4, 4), (1, 4, 4), "bf16", (10,), norm, layout, seed=8)
    xs, ws = [t.cuda() for t in x], [None if t is None else t.cuda() for t in w]
    outs = [torch.empty_like(t) for t in xs]
    op.forward(xs, outs, ws)
    bad = [t.clone() for t in xs]
    bad[0][0, 5, 1, 40] = float("inf")
    bad[0][0, 9, 2, 41] = float("nan")
    got = [torch.empty_like(t) for t in xs]
    op.forward(bad, got, ws)
    same = torch.ones_like(outs[0], dtype=torch.bool)
    if norm == "none":
        same[0, 5, 1, 40] = same[0, 9, 2, 41] = False
        assert got[0][0, 5, 1, 40] == float("inf") and got[0][0, 9, 2, 41].isnan()
    elif norm == "head":
        same[0, 5, 1] = same[0, 9, 2] = False
    else:
        same[0, 5] = same[0, 9] = False
    assert torch.equal(got[0][same], outs[0][same]) and torch.equal(got[1], outs[1])


@pytest.mark.parametrize("B,S,token,sample", [(1, 2200, 2 ** 20, 0), (2, 5, 2 ** 28, 2 ** 31)])
def test_offsets_beyond_32_bits(B, S, token, sample):
    """The last token more than 2^31 elements behind the first; samples that do not follow one another at the tokens' distance."""
    shape, op, x, dy, w, pos, f, axis, m = case(B, 2, 64, (1, 1, S), (1, 1, S), "bf16", (32,), "row", "half", seed=2)
    big = torch.empty((B - 1) * sample + S * token, dtype=torch.bfloat16, device="cuda")
    far = [big.as_strided((B, S, 2, 64), (sample or S * token, token, 64, 1), 128 * i) for i in range(4)]
    for a, b in zip(far, x):
        a.copy_(b)
    ws = [t.cuda() for t in w]
    op.forward(far[:2], far[2:], ws)
    got = [torch.empty((B, S, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    op.backward([t.cuda() for t in dy], far[:2], got, ws)
    for k in range(2):
        check(far[2 + k], *P.norm_rotate(x[k], w[k], pos, f, axis, "half", "row", m), 5e-6, f"far {k}")
        (dx, mag), _ = P.norm_rotate_grad(dy[k], x[k], w[k], pos, f, axis, "half", "row", m)
        check(got[k], dx, mag, 5e-6, f"dx {k}")
