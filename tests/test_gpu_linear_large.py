"""Linear layers and feed-forward blocks at sizes where a CTA pair takes several tiles, in every way that results leave: against the 64-bit
statement, on the GPU.  Tolerances as in the tests of small ones.  Offsets beyond 32 bits; rows that samples' ends cut."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm, FeedForward, Linear
from tests import _block64 as P

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HALF = 2.0 ** -8


def check(got, want, what):
    ref, err = want
    off = (got.double() - ref).abs()
    half = torch.finfo(got.dtype).eps / 2
    tol = half * ref.abs() + (1 + half) * err + torch.finfo(got.dtype).tiny
    assert bool((off <= tol).all()), f"{what}: {off.max():.3e}, worst over its tolerance {(off / tol).nan_to_num(posinf=9e9).max():.2f}"
    if got.dtype is BF:
        assert off.square().mean().sqrt() <= HALF * ref.square().mean().sqrt(), f"{what}: root mean square"


def rnd(g, *s, by=1.0, dt=BF):
    return (torch.randn(s, generator=g, device="cuda") * by).to(dt)


def cut(x, pad_rows):
    """x as a view in which samples do not follow one another at the tokens' distance."""
    B, S, C = x.shape
    big = torch.full((B, S + pad_rows, C), 3.0, dtype=x.dtype, device="cuda")
    big[:, :S] = x
    return big[:, :S]


@pytest.mark.parametrize("B,S,K,N,act,gated,heads,gt,residual,apart", [
    (1, 9000, 328, 2056, "none", False, 0, -1, False, False),          # boxes
    (3, 3001, 200, 1288, "gelu", False, 0, -1, False, True),           # boxes, samples apart
    (2, 5000, 256, 1544, "none", False, 2, 700, True, False),          # rows, another order
    (1, 7000, 136, 1032, "silu", True, 0, -1, False, False),           # gated
    (2, 2600, 136, 1160, "gelu", True, 0, 1300, True, True),           # gated, by rows, samples apart
])
def test_linear(B, S, K, N, act, gated, heads, gt, residual, apart):
    g = torch.Generator(device="cuda").manual_seed(S)
    wide, tokens = 2 * N if gated else N, max(gt, 0)
    x, w, b, d = rnd(g, B, S, K), rnd(g, wide, K, by=K ** -0.5), rnd(g, wide, by=0.2), rnd(g, B, S, N)
    res = rnd(g, B, S, N) if residual else None
    gate = rnd(g, B, -(-S // gt) if gt else 1, N, dt=torch.float32) if gt >= 0 else None
    order = torch.randperm(S, device="cuda") if heads else None
    D = lambda t: None if t is None else t.double()
    op = Linear(vb.make_linear_shape(B, S, K, N, "bf16", act, gated, heads, tokens))
    perm = None if order is None else order.to(torch.int32)
    xx = x.view(B, S, heads, K // heads).transpose(1, 2).contiguous() if heads else cut(x, 5) if apart else x
    out = cut(torch.zeros_like(d), 3) if apart else torch.empty_like(d)
    kept = torch.empty((B, S, wide), dtype=BF, device="cuda")
    op.forward(xx, w, out, bias=b, gate=gate, residual=res, perm=perm, kept=kept)
    want, kw = P.linear(D(x), D(w), D(b), act, gated, D(gate), tokens, D(res), False, order)
    check(out, want, "out")
    check(kept, kw, "kept")
    del want, kw
    needs = act != "none" or gated or gate is not None
    (du, due), dg = P.du_of(D(d), kept.double(), act, gated, D(gate), tokens, False, order)
    rounded = due + (HALF * (du.abs() + due) if needs else 0.0)
    dx = torch.empty_like(xx) if heads or not apart else cut(torch.zeros_like(x), 2)
    dw, db, dgate = op.backward(d, xx, w, dx, kept=kept if needs else None, gate=gate, perm=perm, with_bias=True)
    check(dx.transpose(1, 2).reshape(B, S, K) if heads else dx, P.input_grad(du, rounded, D(w)), "dx")
    check(dw, P.weight_grad(du, rounded, D(x)), "dweight")
    check(db, P.column_sums(du, due), "dbias")
    if dg is not None:
        check(dgate, dg, "dgate")
    op.check_status()


@pytest.mark.parametrize("B,S,C,H,act,gated,gt", [(1, 9000, 136, 1544, "gelu", False, -1), (2, 3300, 200, 1096, "silu", True, 500)])
def test_feed_forward_gradients(B, S, C, H, act, gated, gt):
    g = torch.Generator(device="cuda").manual_seed(S)
    wide, tokens = 2 * H if gated else H, max(gt, 0)
    x, d = rnd(g, B, S, C), rnd(g, B, S, C)
    w1, w2 = rnd(g, wide, C, by=C ** -0.5), rnd(g, C, H, by=H ** -0.5)
    gate = rnd(g, B, -(-S // gt), C, dt=torch.float32) if gt >= 0 else None
    up, down = rnd(g, B, S, wide), rnd(g, B, S, C)
    D = lambda t: None if t is None else t.double()
    op = FeedForward(B, S, C, H, "bf16", act, gated, tokens)
    dx = torch.empty_like(x)
    for dd in (d, cut(d, 4)):
        got = op.backward(dd, x, w1, w2, (up, down if gate is not None else None), dx, gate=gate, with_bias=True)
        (g1, g1e), dg = P.du_of(D(d), D(down), "none", False, D(gate), tokens, False)
        # (the gated gradient goes on in two planes: 2^-17 of it is left)
        g1r = g1e + (2.0 ** -16 * g1.abs() if gate is not None else 0.0)
        dh, dhe = P.input_grad(g1, g1r, D(w2))
        (du, due), _ = P.du_of(dh, D(up), act, gated, None, 0, False, de=dhe)
        dur = due + HALF * (du.abs() + due)
        h, he = P.through(act, gated, D(up), torch.zeros_like(up, dtype=torch.float64), False)
        check(dx, P.input_grad(du, dur, D(w1)), "dx")
        check(got[0], P.weight_grad(du, dur, D(x)), "dw_up")
        check(got[1], P.weight_grad(g1, g1r, h, he + HALF * (h.abs() + he)), "dw_down")
        check(got[2], P.column_sums(du, due), "db_up")
        check(got[3], P.column_sums(g1, g1e), "db_down")
        if dg is not None:
            check(got[4], dg, "dgate")
    op.check_status()


def test_samples_of_one_token_in_strided_rows():
    big = torch.randn((40, 9, 264), device="cuda").to(BF)
    w = torch.randn((72, 264), device="cuda").to(BF)
    for x in (big[:, 3:4], big[:20, 3:4]):                  # (by tiles; straight into registers)
        B = x.shape[0]
        op = Linear(vb.make_linear_shape(B, 1, 264, 72, "bf16"))
        out = torch.zeros((B, 5, 72), dtype=BF, device="cuda")
        op.forward(x, w, out[:, 2:3])
        want = torch.empty((1, B, 72), dtype=BF, device="cuda")
        Linear(vb.make_linear_shape(1, B, 264, 72, "bf16")).forward(x.reshape(1, B, 264).contiguous(), w, want)
        assert torch.equal(out[:, 2], want[0]) and not bool(out[:, :2].any()) and not bool(out[:, 3:].any())
    op = Linear(vb.make_linear_shape(10, 1, 264, 72, "bf16", gate_tokens=0))
    gate, out = torch.randn((10, 1, 72), device="cuda"), torch.empty((10, 1, 72), dtype=BF, device="cuda")
    op.forward(big[:10, :1], w, out, gate=gate)
    ref = (big[:10, 0].double() @ w.double().T) * gate[:, 0].double()
    assert ((out[:, 0].double() - ref).abs() <= HALF * ref.abs() + 1e-3).all()


def test_offsets_beyond_32_bits():
    # 2^31 elements lie between the first row and the last: of x, of out, of kept, of a stream
    S, C = 5, 64
    step = 2 ** 29 + 64
    x = torch.empty(4 * step + C, dtype=BF, device="cuda").as_strided((1, S, C), (0, step, 1))
    x.copy_(torch.randn((1, S, C), device="cuda"))
    w = torch.randn((72, C), device="cuda").to(BF)
    near = x.contiguous()
    for n in (S, 300):                                     # (few tokens; tiles)
        if n == 300:
            far = torch.empty(2 * 10 ** 9 + 2 ** 28, dtype=BF, device="cuda")
            row = (far.numel() - C) // 299 // 8 * 8
            x = far.as_strided((1, 300, C), (0, row, 1))
            x.copy_(torch.randn((1, 300, C), device="cuda"))
            near = x.contiguous()
        op = Linear(vb.make_linear_shape(1, n, C, 72, "bf16"))
        a, b = (torch.empty((1, n, 72), dtype=BF, device="cuda") for _ in range(2))
        op.forward(x, w, a)
        op.forward(near, w, b)
        assert torch.equal(a, b)
        d = torch.randn((1, n, 72), device="cuda").to(BF)
        dx = torch.empty_like(near)
        dw = op.backward(d, near, w, dx)[0]
        dw2 = op.backward(d, x, w, None)[0]
        assert torch.equal(dw, dw2)
        norm = BlockNorm(vb.make_norm_shape(1, n, C, "bf16"))
        p, q = torch.empty_like(near), torch.empty_like(near)
        norm.forward(x, p, h_out=x)
        norm.forward(near, q)
        assert torch.equal(p, q) and torch.equal(x.contiguous(), near)
        back, back2 = torch.empty_like(near), near.clone()
        norm.backward(p, x, back)
        norm.backward(q, near, back2)
        assert torch.equal(back, back2)


def test_norm_gradients_without_the_branchs_own():
    B, S, C = 2, 50, 264
    for post in ("none", "layer"):
        op = BlockNorm(vb.make_norm_shape(B, S, C, "bf16", post_norm=post))
        h, y, d = (torch.randn((B, S, C), device="cuda").to(BF) for _ in range(3))
        gate = torch.randn((B, 1, C), device="cuda")
        dx, dx2, dy = (torch.empty_like(h) for _ in range(3))
        a = op.backward(d, h, dx, y=y, dy_out=dy, gate=gate)
        b = op.backward(d, h, dx2, y=y, gate=gate)
        assert torch.equal(dx, dx2) and torch.equal(a["dgate"], b["dgate"])


def test_permutations_that_are_none():
    # places without a token and tokens with two: nothing is read that was not written, and what is sound comes out right
    B, S, heads, N = 2, 70, 1, 72
    for groups in (0, 16):
        op = Linear(vb.make_linear_shape(B, S, 128, N, "bf16", heads=heads, gate_tokens=groups))
        g = torch.Generator(device="cuda").manual_seed(1)
        x, w, d = rnd(g, B, heads, S, 128), rnd(g, N, 128), rnd(g, B, S, N)
        gate = rnd(g, B, 5 if groups else 1, N, dt=torch.float32)
        kept = rnd(g, B, S, N)
        perm = torch.arange(S, dtype=torch.int32, device="cuda")
        ref = torch.empty_like(x)
        op.backward(d, x, w, ref, kept=kept, gate=gate, perm=perm)
        perm[3], perm[9], perm[20] = -5, S, 2 ** 30
        for _ in range(2):
            junk = torch.full((64 << 20,), float("nan"), device="cuda")       # (what the next scratch may find)
            del junk
            dx = torch.full_like(x, 7.0)
            dw, _, dg = op.backward(d, x, w, dx, kept=kept, gate=gate, perm=perm)
            sound = torch.ones(S, dtype=torch.bool, device="cuda")
            sound[[3, 9, 20]] = False
            assert torch.equal(dx[:, :, sound], ref[:, :, sound]) and not bool(dx[:, :, ~sound].any())
            assert bool(dw.isfinite().all()) and bool(dg.isfinite().all())


@pytest.mark.parametrize("B,S,K,N,heads,gt", [(1, 5000, 256, 1544, 2, 700), (2, 1700, 1536, 1536, 0, 0), (3, 3, 136, 1032, 0, -1)])
def test_residual_that_is_the_output(B, S, K, N, heads, gt):
    g = torch.Generator(device="cuda").manual_seed(N)
    x, w, b, res = rnd(g, B, S, K), rnd(g, N, K, by=K ** -0.5), rnd(g, N, by=0.2), rnd(g, B, S, N)
    gate = rnd(g, B, -(-S // gt) if gt else 1, N, dt=torch.float32) if gt >= 0 else None
    perm = torch.randperm(S, device="cuda").to(torch.int32) if heads else None
    op = Linear(vb.make_linear_shape(B, S, K, N, "bf16", "none", False, heads, max(gt, 0)))
    xx = x.view(B, S, heads, K // heads).transpose(1, 2).contiguous() if heads else x
    apart, stream = torch.empty_like(res), res.clone()
    op.forward(xx, w, apart, bias=b, gate=gate, residual=res, perm=perm)
    op.forward(xx, w, stream, bias=b, gate=gate, residual=stream, perm=perm)
    assert torch.equal(apart, stream)
    block = FeedForward(B, S, K, 264, "bf16", "gelu", False, 0)
    w1, w2 = rnd(g, 264, K, by=K ** -0.5), rnd(g, K, 264, by=264 ** -0.5)
    apart, stream = torch.empty_like(x), x.clone()
    block.forward(x, w1, w2, apart, residual=x)
    block.forward(x, w1, w2, stream, residual=stream)
    assert torch.equal(apart, stream)
    op.check_status()
    block.check_status()
