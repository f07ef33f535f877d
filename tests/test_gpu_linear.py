"""Linear layers and feed-forward blocks on the GPU against the 64-bit statements, whose bounds of 32-bit arithmetic stand there; a result is rounded once
more to its type, half a step of it.  Gradients of products behind an activation, a gate or a reordering (du), and h of a feed-forward block, are rounded
once in between: half a step of each of them in the sums they go into.  That worst case is far from what roundings add up to, so that the root of the
mean square of a bf16 result's error is held to 2^-8 of the result's too: one rounding is 2^-8 / sqrt(12) of a number's power of two at most, and three
independent ones of a sum's terms or of the sum stay below 2^-8."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import FeedForward, Linear
from tests import _block64 as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(got, want, what):
    ref, err = want
    got, half = got.detach().cpu(), torch.finfo(got.dtype).eps / 2
    off = (got.double() - ref).abs()
    tol = half * ref.abs() + (1 + half) * err + torch.finfo(got.dtype).tiny
    assert bool((off <= tol).all()), f"{what}: {off.max():.3e}, worst over its tolerance {(off / tol).nan_to_num(posinf=9e9).max():.2f}"
    if got.dtype is torch.bfloat16 and ref.numel() >= 256:
        assert off.square().mean().sqrt() <= 2.0 ** -8 * ref.square().mean().sqrt(), f"{what}: root mean square"


def make(gen, dtype, *shape, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(DT[dtype])


def half_of(dtype):
    return torch.finfo(DT[dtype]).eps / 2 if dtype == "bf16" else 0.0


# B, S, n_in, n_out, dtype, act, gated, heads, gate_tokens (-1: no gate), residual, bias
CASES = [
    (1, 1, 8, 8, "bf16", "none", False, 0, -1, False, False),
    (1, 1, 1536, 1000, "bf16", "silu", False, 0, -1, False, True),
    (3, 1, 72, 40, "bf16", "gelu", True, 0, 0, True, True),
    (1, 5, 64, 264, "bf16", "gelu", False, 0, 0, True, True),
    (2, 130, 200, 136, "bf16", "none", False, 0, -1, False, True),
    (1, 255, 128, 520, "bf16", "silu", True, 0, 100, True, True),
    (2, 257, 264, 256, "bf16", "gelu", False, 0, 64, True, False),
    (1, 700, 1000, 520, "bf16", "none", False, 0, 1, True, True),
    (3, 60, 256, 192, "bf16", "none", False, 2, 7, True, True),
    (2, 300, 320, 328, "bf16", "silu", False, 5, 0, True, True),
    (1, 513, 128, 1032, "bf16", "gelu", True, 1, 200, False, True),
    (1, 64, 4104, 128, "bf16", "none", False, 0, -1, False, False),
    (1, 2000, 64, 64, "bf16", "none", False, 0, 0, True, True),
    (1, 1, 16, 24, "f32", "gelu", False, 0, -1, True, True),
    (2, 77, 72, 136, "f32", "silu", True, 0, 10, True, True),
    (2, 90, 128, 200, "f32", "none", False, 2, 0, True, True),
    (1, 1300, 264, 1544, "f32", "gelu", False, 0, -1, False, True),
]


def data(i, strided=False):
    B, S, K, N, dtype, act, gated, heads, gt, residual, bias = CASES[i]
    g = torch.Generator().manual_seed(i)
    rows = 2 * N if gated else N
    t = {"x": make(g, dtype, B, S, K), "w": make(g, dtype, rows, K, scale=K ** -0.5), "b": make(g, dtype, rows, scale=0.3) if bias else None,
         "res": make(g, dtype, B, S, N) if residual else None, "d": make(g, dtype, B, S, N), "tokens": max(gt, 0),
         "order": torch.randperm(S, generator=g) if heads else None}
    t["gate"] = torch.randn((B, -(-S // gt) if gt else 1, N), generator=g) if gt >= 0 else None
    shape = vb.make_linear_shape(B, S, K, N, dtype, act, gated, heads, max(gt, 0))
    return CASES[i], t, shape


def cuda(t):
    return None if t is None else t.cuda()


def by_heads(x, heads):
    B, S, K = x.shape
    return x.view(B, S, heads, K // heads).transpose(1, 2).contiguous() if heads else x


def wide(x, pad):
    """x as a view of a tensor with `pad` channels of something else behind every row."""
    if x is None:
        return None
    big = torch.full((*x.shape[:-1], x.shape[-1] + pad), 7.0, dtype=x.dtype, device=x.device)
    big[..., : x.shape[-1]] = x
    return big[..., : x.shape[-1]]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_linear_forward_and_backward(i):
    (B, S, K, N, dtype, act, gated, heads, gt, residual, bias), t, shape = data(i)
    dbl = lambda n: None if t[n] is None else t[n].double()
    f32 = dtype == "f32"
    (out, oe), (kept, ke) = P.linear(dbl("x"), dbl("w"), dbl("b"), act, gated, dbl("gate"), t["tokens"], dbl("res"), f32, t["order"])
    op = Linear(shape)
    x, w, perm = by_heads(t["x"].cuda(), heads), t["w"].cuda(), None if t["order"] is None else t["order"].to(torch.int32).cuda()
    got_kept = torch.empty((B, S, shape.wide), dtype=DT[dtype], device="cuda")
    got = torch.full((B, S, N + 8), 7.0, dtype=DT[dtype], device="cuda")
    op.forward(x, w, got[..., :N], bias=cuda(t["b"]), gate=cuda(t["gate"]), residual=wide(cuda(t["res"]), 16), perm=perm, kept=got_kept)
    check(got[..., :N], (out, oe), "out")
    assert bool((got[..., N:] == 7).all())
    check(got_kept, (kept, ke), "kept")
    # onto the residual itself, without kept, from strided rows
    onto = torch.zeros((B, S, N), dtype=DT[dtype], device="cuda") if t["res"] is None else t["res"].cuda()
    op.forward(x if heads else wide(x, 24), w, onto, bias=cuda(t["b"]), gate=cuda(t["gate"]), residual=None if t["res"] is None else onto, perm=perm)
    assert torch.equal(onto, got[..., :N].contiguous())
    op.check_status()

    # gradients, from what the forward left
    k64 = got_kept.cpu().double()
    (du, due), dg = P.du_of(dbl("d"), k64, act, gated, dbl("gate"), t["tokens"], f32, t["order"])
    apart = act != "none" or gated or t["gate"] is not None
    half = half_of(dtype) if apart else 0.0
    rounded = due + half * (du.abs() + due)
    dx = torch.empty_like(x)
    res = op.backward(t["d"].cuda(), x, w, dx, kept=got_kept if apart else None, gate=cuda(t["gate"]), perm=perm, with_bias=True)
    want_dx, dxe = P.input_grad(du, rounded, dbl("w"))
    check(dx.transpose(1, 2).reshape(B, S, K) if heads else dx, (want_dx, dxe), "dx")
    check(res[0], P.weight_grad(du, rounded, dbl("x")), "dweight")
    check(res[1], P.column_sums(du, due), "dbias")
    assert (res[2] is None) == (dg is None)
    if dg is not None:
        check(res[2], dg, "dgate")
    # the same again bit for bit, from strided rows; parts of it alone
    dx2 = torch.empty_like(x) if heads else wide(torch.zeros_like(x), 8)
    again = op.backward(wide(t["d"].cuda(), 8), x if heads else wide(x, 8), w, dx2, kept=got_kept if apart else None, gate=cuda(t["gate"]), perm=perm, with_bias=True)
    assert torch.equal(dx, dx2)
    for a, b in zip(res, again):
        assert a is None or torch.equal(a, b)
    only = op.backward(t["d"].cuda(), x, w, None, kept=got_kept if apart else None, gate=cuda(t["gate"]), perm=perm, with_weight=False, with_bias=True)
    assert only[0] is None and torch.equal(only[1], res[1])
    op.check_status()


FFN = [
    # B, S, channels, hidden, dtype, act, gated, gate_tokens, residual, bias
    (1, 1, 64, 136, "bf16", "gelu", False, 0, True, True),
    (2, 9, 72, 200, "bf16", "silu", True, 4, True, False),
    (1, 300, 264, 520, "bf16", "gelu", False, -1, False, True),
    (2, 200, 128, 328, "bf16", "silu", True, 0, True, True),
    (1, 65, 48, 104, "f32", "gelu", False, 20, True, True),
    (2, 40, 64, 72, "f32", "silu", True, -1, True, True),
    (1, 40, 64, 72, "bf16", "none", True, -1, False, True),
]


@pytest.mark.parametrize("i", range(len(FFN)))
def test_feed_forward_forward_and_backward(i):
    B, S, C, H, dtype, act, gated, gt, residual, bias = FFN[i]
    g, f32, tokens = torch.Generator().manual_seed(100 + i), dtype == "f32", max(gt, 0)
    rows = 2 * H if gated else H
    x, w1, w2, d = make(g, dtype, B, S, C), make(g, dtype, rows, C, scale=C ** -0.5), make(g, dtype, C, H, scale=H ** -0.5), make(g, dtype, B, S, C)
    b1, b2 = (make(g, dtype, rows, scale=0.3), make(g, dtype, C, scale=0.3)) if bias else (None, None)
    res = make(g, dtype, B, S, C) if residual else None
    gate = torch.randn((B, -(-S // gt) if gt else 1, C), generator=g) if gt >= 0 else None
    D = lambda t: None if t is None else t.double()
    half = half_of(dtype)
    (h, he), (up, upe) = P.linear(D(x), D(w1), D(b1), act, gated, f32=f32)
    hr = he + half * (h.abs() + he)
    (out, oe), (down, de) = P.linear(h, D(w2), D(b2), gate=D(gate), tokens=tokens, residual=D(res), f32=f32, xe=hr)
    op = FeedForward(B, S, C, H, dtype, act, gated, tokens)
    kept, got = op.keep(), torch.empty((B, S, C), dtype=DT[dtype], device="cuda")
    c = [cuda(t) for t in (x, w1, w2)]
    op.forward(*c, got, cuda(b1), cuda(b2), cuda(gate), cuda(res), kept)
    check(got, (out, oe), "out")
    check(kept[0], (up, upe), "kept up")
    check(kept[1], (down, de), "kept down")
    again = torch.empty_like(got)
    op.forward(*c, again, cuda(b1), cuda(b2), cuda(gate), cuda(res))
    assert torch.equal(got, again)

    up, down = D(kept[0].cpu()), D(kept[1].cpu())
    (dd, dde), dg = P.du_of(D(d), down, "none", False, D(gate), tokens, f32)
    ddr = dde + (half * (dd.abs() + dde) if gate is not None else 0.0)
    dh, dhe = P.input_grad(dd, ddr, D(w2))
    dhr = dhe + half * (dh.abs() + dhe)
    (du, due), _ = P.du_of(dh, up, act, gated, None, 0, f32, de=dhr)
    dur = due + half * (du.abs() + due)
    h, he = P.through(act, gated, up, torch.zeros_like(up), f32)
    hr = he + half * (h.abs() + he)
    dx = torch.empty_like(c[0])
    res_ = op.backward(d.cuda(), *c, kept if gate is not None else (kept[0], None), dx, cuda(gate), with_bias=True)
    want = {"dw_up": P.weight_grad(du, dur, D(x)), "dw_down": P.weight_grad(dd, ddr, h, hr), "db_up": P.column_sums(du, due),
            "db_down": P.column_sums(dd, dde), "dgate": dg}
    check(dx, P.input_grad(du, dur, D(w1)), "dx")
    for (n, v), r in zip(want.items(), res_):
        assert (v is None) == (r is None)
        if v is not None:
            check(r, v, n)
    dx2 = torch.empty_like(dx)
    for a, b in zip(res_, op.backward(d.cuda(), *c, kept, dx2, cuda(gate), with_bias=True)):
        assert a is None or torch.equal(a, b)
    assert torch.equal(dx, dx2)
    # weights' gradients without dx, and dx without them
    r = op.backward(d.cuda(), *c, kept, None, cuda(gate))
    assert torch.equal(r[0], res_[0]) and torch.equal(r[1], res_[1]) and r[2] is None
    dx2.zero_()
    op.backward(d.cuda(), *c, kept, dx2, cuda(gate), with_weights=False)
    assert torch.equal(dx, dx2)
    op.check_status()


def test_places_outside_leave_their_rows_out():
    shape = vb.make_linear_shape(1, 40, 128, 64, "bf16", heads=1)
    g = torch.Generator().manual_seed(3)
    x, w, d = (make(g, "bf16", *s).cuda() for s in ((1, 1, 40, 128), (64, 128), (1, 40, 64)))
    perm = torch.arange(40, dtype=torch.int32, device="cuda")
    want = torch.empty((1, 40, 64), dtype=torch.bfloat16, device="cuda")
    op = Linear(shape)
    op.forward(x, w, want, perm=perm)
    bad = perm.clone()
    bad[3], bad[7] = 40, -1
    out = torch.full_like(want, 5.0)
    op.forward(x, w, out, perm=bad)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[3] = keep[7] = False
    assert torch.equal(out[:, keep], want[:, keep]) and bool((out[:, ~keep] == 5).all())


def test_values_that_are_not_finite_stay_in_their_rows():
    for dtype in ("bf16", "f32"):
        shape = vb.make_linear_shape(1, 200, 64, 72, dtype, "gelu")
        g = torch.Generator().manual_seed(4)
        x, w = make(g, dtype, 1, 200, 64).cuda(), make(g, dtype, 72, 64).cuda()
        op, a, b = Linear(shape), *(torch.empty((1, 200, 72), dtype=DT[dtype], device="cuda") for _ in range(2))
        op.forward(x, w, a)
        x[0, 5, 3], x[0, 130, 9] = float("nan"), float("inf")
        op.forward(x, w, b)
        clean = torch.ones(200, dtype=torch.bool, device="cuda")
        clean[5] = clean[130] = False
        assert torch.equal(a[:, clean], b[:, clean]) and bool(b[0, 5].isnan().all()) and not bool(b[0, 130].isfinite().all())


def test_large_arguments_of_the_activations():
    u = torch.tensor([-1e30, -1e5, -200.0, -88.0, -30.0, -1e-30, 0.0, 1e-30, 30.0, 100.0, 1e5, 1e30], dtype=torch.float64)
    for dtype in ("bf16", "f32"):
        for name in ("gelu", "silu"):
            S = u.numel()
            kept = torch.zeros((1, S, 8), dtype=DT[dtype], device="cuda")
            kept[0] = u.to(DT[dtype])[:, None]
            op = Linear(vb.make_linear_shape(1, S, 8, 8, dtype, name))
            eye, d = torch.eye(8, dtype=DT[dtype], device="cuda"), torch.ones((1, S, 8), dtype=DT[dtype], device="cuda")
            dx, x = torch.empty_like(d), torch.zeros_like(d)
            x[0] = u.to(DT[dtype])[:, None] * torch.eye(8, dtype=DT[dtype])[:1]
            op.backward(d, x, eye, dx, kept=kept, with_weight=False)
            want = torch.where(u.abs() > 60, (u > 0).double(), P.slope(name, u))
            assert torch.allclose(dx[0, :, 0].double().cpu(), want, rtol=2.0 ** -7, atol=1e-5), name
            out = torch.empty_like(d)
            op.forward(x, eye, out)
            v = x[0, :, 0].double().cpu()
            want = torch.where(v.abs() > 60, v.clamp(min=0), P.act(name, v))
            assert torch.allclose(out[0, :, 0].double().cpu(), want, rtol=2.0 ** -7, atol=1e-5), name


def test_refusals():
    ok = vb.make_linear_shape(2, 16, 64, 32, "bf16")
    op = Linear(ok)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    x, w, out = z(2, 16, 64), z(32, 64), z(2, 16, 32)
    with pytest.raises(ValueError):
        Linear(vb.make_linear_shape(2, 16, 60, 32, "bf16"))
    with pytest.raises(ValueError):
        Linear(ok, device="cpu")
    for bad in (dict(x=z(2, 16, 72)), dict(x=z(2, 16, 64, dt=torch.float32)), dict(x=x.cpu()), dict(weight=z(32, 72)), dict(weight=z(64, 32).T), dict(out=z(2, 16, 40)),
                dict(out=z(2, 16, 33)[..., :32]), dict(out=z(1, 16, 32).expand(2, 16, 32)), dict(bias=z(64)), dict(bias=z(32, dt=torch.float32)),
                dict(gate=z(2, 2, 32, dt=torch.float32)), dict(gate=z(2, 1, 32)), dict(residual=z(2, 16, 64)), dict(perm=z(16, dt=torch.int32)), dict(kept=z(2, 16, 64))):
        with pytest.raises(ValueError):
            op.forward(**{"x": x, "weight": w, "out": out, **bad})
    with pytest.raises(ValueError):
        Linear(vb.make_linear_shape(2, 16, 64, 32, "bf16", "gelu")).backward(out, x, w, None)
    with pytest.raises(ValueError):
        op.backward(out, x, w, None, gate=z(2, 1, 32, dt=torch.float32))
    # inputs in whatever order are copied, rows that are shared too
    a, b = z(2, 16, 32), z(2, 16, 32)
    xx = torch.randn((16, 64), device="cuda").to(torch.bfloat16)
    ww = torch.randn((32, 64), device="cuda").to(torch.bfloat16)
    op.forward(xx.expand(2, 16, 64), ww, a)
    op.forward(xx.expand(2, 16, 64).contiguous().transpose(1, 2).contiguous().transpose(1, 2), ww, b)
    assert torch.equal(a, b) and bool(a.any())
    with pytest.raises(ValueError):
        FeedForward(1, 4, 60, 64)
    ff = FeedForward(1, 4, 64, 72)
    with pytest.raises(ValueError):
        ff.backward(z(1, 4, 64), z(1, 4, 64), z(72, 64), z(64, 72), (None, None), None)


@pytest.mark.parametrize("B,S,K,N,act,gated,heads,gt", [
    (2, 2, 240, 56, "silu", True, 0, -1), (1, 1, 8, 8, "gelu", False, 0, 0), (3, 17, 128, 72, "none", False, 2, 5),
    (1, 100, 128, 96, "gelu", True, 1, 0), (2, 40, 128, 264, "silu", False, 0, 7),
])
def test_few_results_without_the_roundings_between(B, S, K, N, act, gated, heads, gt):
    # of du there are two planes: what its rounding left is in the results, to 2^-17 of it
    g = torch.Generator(device="cuda").manual_seed(S + K)
    wide, tokens = 2 * N if gated else N, max(gt, 0)
    dev = lambda *s, by=1.0, dt=torch.bfloat16: (torch.randn(s, generator=g, device="cuda") * by).to(dt)
    x, w, d, kept = dev(B, S, K), dev(wide, K, by=K ** -0.5), dev(B, S, N), dev(B, S, wide)
    gate = dev(B, -(-S // gt) if gt else 1, N, dt=torch.float32) if gt >= 0 else None
    order = torch.randperm(S, device="cuda") if heads else None
    D = lambda t: None if t is None else t.double()
    op = Linear(vb.make_linear_shape(B, S, K, N, "bf16", act, gated, heads, tokens))
    xx = x.view(B, S, heads, K // heads).transpose(1, 2).contiguous() if heads else x
    dx = torch.empty_like(xx)
    dw, db, dgate = op.backward(d, xx, w, dx, kept=kept, gate=gate, perm=None if order is None else order.to(torch.int32), with_bias=True)
    (du, due), dg = P.du_of(D(d), D(kept), act, gated, D(gate), tokens, False, order)
    rounded = due + 2.0 ** -16 * du.abs()
    for got, (ref, err), what in ((dx.transpose(1, 2).reshape(B, S, K) if heads else dx, P.input_grad(du, rounded, D(w)), "dx"),
                                  (dw, P.weight_grad(du, rounded, D(x)), "dweight")):
        half = torch.finfo(got.dtype).eps / 2
        off = (got.double() - ref).abs()
        assert bool((off <= half * ref.abs() + (1 + half) * err + torch.finfo(got.dtype).tiny).all()), what
    op.check_status()
