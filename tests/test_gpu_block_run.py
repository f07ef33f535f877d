"""The operators of a transformer block as they are used together: norm and modulation, q, k and v from one linear layer, rotary positions, the
attention layer, its projection straight from block order onto the residual stream, norm, feed-forward block.  Forward and gradients in fp32
against automatic differentiation in 64 bits; the projection against the same layer with o in raster order; several streams; captured graphs.

Tolerance of the fp32 run: every operator's tests hold it to 5e-6 of the magnitudes it adds up or less (its sums have at most 600 terms, 600 x 2^-24 =
3.6e-5 at the worst and about its root, 1.5e-6, of independent roundings); ten of them one after another, each of whose errors the next
ones pass on about as they pass on the values: 2e-5 of the root of the mean square of a result covers them with a factor of four to spare over
ten independent ones (1.5e-6 x sqrt(10) = 5e-6)."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import (BlockNorm, FeedForward, Linear, Rotary, SteppedAttention, VmobaLayer, default_capacity,
                                         rotary_frequencies)
from tests import _block64 as P
from tests import _plain64 as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Block:
    """One block of a video transformer, from this package's operators."""

    def __init__(self, B, grid, blocks, heads, d, hidden, dtype, tau, gated=True, seed=0):
        self.B, self.grid, self.heads, self.d, self.tau, self.dtype = B, grid, heads, d, tau, DT[dtype]
        S, C = grid[0] * grid[1] * grid[2], heads * d
        self.S, self.C, frame = S, C, grid[1] * grid[2]
        self.frame = frame
        shape = vb.make_shape(B, heads, d, grid, blocks, dtype)
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, by=1.0, dt=self.dtype: (torch.randn(s, generator=g) * by).to(dt)
        up = 2 * hidden if gated else hidden
        self.w = {"qkv": r(3 * C, C, by=C ** -0.5), "b_qkv": r(3 * C, by=0.1), "out": r(C, C, by=C ** -0.5), "b_out": r(C, by=0.1),
                  "up": r(up, C, by=C ** -0.5), "b_up": r(up, by=0.1), "down": r(C, hidden, by=hidden ** -0.5), "b_down": r(C, by=0.1)}
        self.mod = r(B, 6, grid[0], C, by=0.3, dt=torch.float32)      # a row per frame
        f, axis, m = rotary_frequencies((d // 2 - 2 * (d // 6), d // 6, d // 6))
        pos = torch.stack(torch.meshgrid(*(torch.arange(n, dtype=torch.int32) for n in grid), indexing="ij"), -1).view(S, 3).contiguous()
        self.pos, self.freq, self.axis = pos, f, axis
        self.rotary = Rotary(shape, pos.cuda(), f.cuda(), axis.cuda())
        self.attn = VmobaLayer(shape, default_capacity(shape, tau) if tau < 1 else B * heads * S * shape.n_blocks, with_backward=True)
        self.norm1 = BlockNorm(vb.make_norm_shape(B, S, C, dtype, mod_tokens=frame))
        self.norm2 = BlockNorm(vb.make_norm_shape(B, S, C, dtype, mod_tokens=frame))
        self.qkv = Linear(vb.make_linear_shape(B, S, C, 3 * C, dtype))
        self.proj = Linear(vb.make_linear_shape(B, S, C, C, dtype, heads=heads, gate_tokens=frame))
        self.ffn = FeedForward(B, S, C, hidden, dtype, "silu" if gated else "gelu", gated, gate_tokens=frame)
        self.gated, self.hidden = gated, hidden
        self.x, self.d_out = r(B, S, C), r(B, S, C)
        self.cw = {n: t.cuda() for n, t in self.w.items()}
        self.cmod = self.mod.cuda()

    def new(self, *shape):
        return torch.empty(shape, dtype=self.dtype, device="cuda")

    def forward(self, x, kept=None):
        B, S, C, w, m = self.B, self.S, self.C, self.cw, self.cmod
        a, qkv, h, b, out = self.new(B, S, C), self.new(B, S, 3 * C), self.new(B, S, C), self.new(B, S, C), self.new(B, S, C)
        self.norm1.forward(x, a, scale=m[:, 1], shift=m[:, 0])
        self.qkv.forward(a, w["qkv"], qkv, bias=w["b_qkv"])
        q, k, v = qkv.view(B, S, 3, self.heads, self.d).unbind(2)
        keep = self.new(B, S, C) if kept is not None else None
        self.attn.forward(q, k, v, self.tau, h, rotary=self.rotary, projection=self.proj,
                          projected={"weight": w["out"], "bias": w["b_out"], "gate": m[:, 2], "residual": x, "kept": keep})
        self.norm2.forward(h, b, scale=m[:, 4], shift=m[:, 3])
        keep2 = self.ffn.keep() if kept is not None else None
        self.ffn.forward(b, w["up"], w["down"], out, w["b_up"], w["b_down"], gate=m[:, 5], residual=h, kept=keep2)
        if kept is not None:
            kept.update(x=x, a=a, q=q, k=k, h=h, b=b, proj=keep, ffn=keep2)
        return out

    def backward(self, d_out, kept):
        B, S, C, w, m, g = self.B, self.S, self.C, self.cw, self.cmod, {}
        db, dqkv, dx = self.new(B, S, C), self.new(B, S, 3 * C), self.new(B, S, C)
        g["up"], g["down"], g["b_up"], g["b_down"], dg5 = self.ffn.backward(d_out, kept["b"], w["up"], w["down"], kept["ffn"], db, gate=m[:, 5], with_bias=True)
        dh = self.new(B, S, C)
        n2 = self.norm2.backward(db, kept["h"], dh, d_h=d_out, scale=m[:, 4], shift=m[:, 3])
        dq, dk, dv = dqkv.view(B, S, 3, self.heads, self.d).unbind(2)
        _, (g["out"], g["b_out"], dg2) = self.attn.backward(dh, dq, dk, dv, rotary=self.rotary, qk=(kept["q"], kept["k"]), projection=self.proj,
                                                            projected={"weight": w["out"], "kept": kept["proj"], "gate": m[:, 2], "with_bias": True})
        da = self.new(B, S, C)
        g["qkv"], g["b_qkv"], _ = self.qkv.backward(dqkv, kept["a"], w["qkv"], da, with_bias=True)
        n1 = self.norm1.backward(da, kept["x"], dx, d_h=dh, scale=m[:, 1], shift=m[:, 0])
        g["mod"] = torch.stack([n1["dshift"], n1["dscale"], dg2, n2["dshift"], n2["dscale"], dg5], 1)
        g["x"] = dx
        return g

    def plain(self):
        """(out, gradients) in 64 bits: with tau = 1 the layer is dense attention."""
        B, S, C, h, d = self.B, self.S, self.C, self.heads, self.d
        w = {n: t.double().requires_grad_() for n, t in self.w.items()}
        m, x = self.mod.double().requires_grad_(), self.x.double().requires_grad_()
        row = lambda i: P.rows_of(m[:, i], S, self.frame)
        norm = lambda v: (v - v.mean(-1, keepdim=True)) / (v.var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
        a = norm(x) * (1 + row(1)) + row(0)
        q, k, v = (a @ w["qkv"].T + w["b_qkv"]).view(B, S, 3, h, d).unbind(2)
        ang = (self.pos.double()[:, self.axis.long()] * self.freq)[None, :, None]
        turn = lambda t: torch.stack([t[..., 0::2] * ang.cos() - t[..., 1::2] * ang.sin(), t[..., 1::2] * ang.cos() + t[..., 0::2] * ang.sin()], -1).flatten(-2)
        s = torch.einsum("bshd,bthd->bhst", turn(q), turn(k)) * d ** -0.5
        o = torch.einsum("bhst,bthd->bshd", s.softmax(-1), v).reshape(B, S, C)
        hh = x + row(2) * (o @ w["out"].T + w["b_out"])
        b = norm(hh) * (1 + row(4)) + row(3)
        u = b @ w["up"].T + w["b_up"]
        u = P.act("silu", u[..., : self.hidden]) * u[..., self.hidden:] if self.gated else P.act("gelu", u)
        out = hh + row(5) * (u @ w["down"].T + w["b_down"])
        names = list(w) + ["mod", "x"]
        grads = torch.autograd.grad(out, [*w.values(), m, x], self.d_out.double())
        return out.detach(), dict(zip(names, grads))


@pytest.mark.parametrize("gated", [True, False])
def test_block_in_fp32_against_automatic_differentiation(gated):
    blk = Block(2, (3, 4, 6), (1, 4, 6), 3, 64, 200, "f32", 1.0, gated)
    out, grads = blk.plain()
    kept = {}
    got = blk.forward(blk.x.cuda(), kept)
    g = blk.backward(blk.d_out.cuda(), kept)
    for name, a, b in [("out", got, out)] + [(n, g[n], t) for n, t in grads.items()]:
        off = (a.double().cpu() - b).square().mean().sqrt() / b.square().mean().sqrt()
        assert off <= 2e-5, f"{name}: {off:.2e}"
    for op in (blk.attn, blk.norm1, blk.norm2, blk.qkv, blk.proj, blk.ffn):
        op.check_status()


def test_block_in_bf16_is_near_the_fp32_one():
    # bf16 tensors between nine operators, each rounded by 2^-9 of it or so: 3 in a hundred is far from a wrong operator and from their sum
    blk = Block(1, (4, 8, 16), (2, 4, 8), 2, 128, 520, "bf16", 1.0)
    out, grads = blk.plain()
    kept = {}
    got = blk.forward(blk.x.cuda(), kept)
    g = blk.backward(blk.d_out.cuda(), kept)
    for name, a, b in [("out", got, out)] + [(n, g[n], t) for n, t in grads.items()]:
        off = (a.double().cpu() - b).square().mean().sqrt() / b.square().mean().sqrt()
        assert off <= 3e-2, f"{name}: {off:.2e}"


@pytest.mark.parametrize("dtype,heads,d", [("bf16", 3, 128), ("f32", 2, 64)])
def test_projection_of_the_layer_against_the_same_in_raster_order(dtype, heads, d):
    B, grid, blocks, tau = 2, (4, 6, 8), (2, 3, 4), 0.4
    S, C, N = 192, heads * d, 264
    g = torch.Generator().manual_seed(5)
    r = lambda *s, by=1.0, dt=DT[dtype]: (torch.randn(s, generator=g) * by).to(dt).cuda()
    q, k, v = (r(B, S, heads, d) for _ in range(3))
    w, bias, gate, res, do = r(N, C, by=C ** -0.5), r(N), r(B, 5, N, dt=torch.float32), r(B, S, N), r(B, S, N)
    shape = vb.make_shape(B, heads, d, grid, blocks, dtype)
    L = VmobaLayer(shape, default_capacity(shape, tau), with_backward=True)
    in_blocks = Linear(vb.make_linear_shape(B, S, C, N, dtype, heads=heads, gate_tokens=40))
    raster = Linear(vb.make_linear_shape(B, S, C, N, dtype, gate_tokens=40))
    new = lambda *s: torch.empty(s, dtype=DT[dtype], device="cuda")
    o, want, out, kept, kept_b = new(B, S, heads, d), new(B, S, N), new(B, S, N), new(B, S, N), new(B, S, N)
    args = dict(weight=w, bias=bias, gate=gate, residual=res)
    L.forward(q, k, v, tau, o)
    raster.forward(o.view(B, S, C), out=want, kept=kept, **args)
    dx, dq, dk, dv = new(B, S, C), *(new(B, S, heads, d) for _ in range(3))
    wgrads = raster.backward(do, o.view(B, S, C), w, dx, kept=kept, gate=gate, with_bias=True)
    L.backward(dx.view(B, S, heads, d), dq, dk, dv)
    L.forward(q, k, v, tau, out, projection=in_blocks, projected=dict(args, kept=kept_b))
    assert torch.equal(out, want)
    assert torch.equal(kept_b, kept[:, L.perm.long()])
    got = [new(B, S, heads, d) for _ in range(3)]
    grads = L.backward(do, *got, projection=in_blocks, projected=dict(weight=w, kept=kept_b, gate=gate, with_bias=True))
    # the tokens are added up in another order: 192 x 2 roundings of 2^-24, and one more of the type
    half = torch.finfo(DT[dtype]).eps
    for a, b in zip(grads, wgrads):
        assert (a.double() - b.double()).abs().max() <= (1e-4 if a.dtype is torch.float32 else half) * b.double().abs().max()
    # (a row of dq is a sum of parts in any order)
    for a, b in zip(got, (dq, dk, dv)):
        assert (a.double() - b.double()).abs().max() <= (1e-5 if dtype == "f32" else half) * b.double().abs().max()
    # the dense step of a sampler takes the projection too
    step = SteppedAttention(L, tau, 2, 0.5)
    out2, want2, o2 = new(B, S, N), new(B, S, N), new(B, S, heads, d)
    assert step.forward(0, q, k, v, o2) == "dense" and step.forward(0, q, k, v, out2, projection=in_blocks, projected=args) == "dense"
    raster.forward(o2.view(B, S, C), out=want2, **args)
    assert torch.equal(out2, want2)
    assert step.forward(1, q, k, v, out2, projection=in_blocks, projected=args) == "sparse" and torch.equal(out2, want)
    # refusals
    for bad in (dict(projection=raster, projected=args), dict(projection=in_blocks), dict(projection=in_blocks, projected={"bias": bias}),
                dict(projection=in_blocks, projected=args, fold_o=True)):
        with pytest.raises(ValueError):
            L.forward(q, k, v, tau, out, **bad)


def test_block_captured_and_on_two_streams():
    blk = Block(1, (2, 8, 16), (2, 4, 4), 2, 128, 264, "bf16", 0.5)
    x1, x2 = blk.x.cuda(), (blk.x * 0.5 + 0.25).cuda()
    want1, want2 = blk.forward(x1).clone(), blk.forward(x2).clone()
    static = x1.clone()
    blk.forward(static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = blk.forward(static)
    for x, want in ((x2, want2), (x1, want1), (x2, want2)):
        static.copy_(x)
        out.fill_(7)
        graph.replay()
        assert torch.equal(out, want)
    # operators of one object on two streams at the same time: their scratch is the call's own
    B, S, C = 1, 2000, 512
    lin = Linear(vb.make_linear_shape(B, S, C, 136, "bf16"))            # (few tiles: the summed index is cut, partial sums in scratch)
    ffn, norm = FeedForward(B, S, C, 520, gated=True), BlockNorm(vb.make_norm_shape(B, S, C, "bf16"))
    g = torch.Generator().manual_seed(1)
    r = lambda *s, by=1.0: (torch.randn(s, generator=g) * by).to(torch.bfloat16).cuda()
    w, w1, w2 = r(136, C, by=0.05), r(1040, C, by=0.05), r(C, 520, by=0.05)
    xs, ds = [r(B, S, C) for _ in range(2)], [r(B, S, 136) for _ in range(2)]

    def run(i):
        y, z, n, dx = torch.empty_like(ds[i]), torch.empty_like(xs[i]), torch.empty_like(xs[i]), torch.empty_like(xs[i])
        lin.forward(xs[i], w, y)
        dw, _, _ = lin.backward(ds[i], xs[i], w, dx)
        kept = ffn.keep()
        ffn.forward(xs[i], w1, w2, z, kept=kept)
        dx2 = torch.empty_like(xs[i])
        g1 = ffn.backward(z, xs[i], w1, w2, kept, dx2)
        norm.forward(z, n, y=xs[i])
        return [y, dw, dx, z, g1[0], g1[1], dx2, n]

    want = [run(0), run(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = [None, None]
        for i, st in enumerate(streams):
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                got[i] = run(i)
        torch.cuda.synchronize()
        for i in range(2):
            for a, b in zip(got[i], want[i]):
                assert torch.equal(a, b)


def test_backward_captured_and_replayed():
    B, S, C, H = 1, 300, 264, 328
    ffn, norm = FeedForward(B, S, C, H, gated=True), BlockNorm(vb.make_norm_shape(B, S, C, "bf16", post_norm="rms", mod_tokens=100))
    g = torch.Generator().manual_seed(2)
    r = lambda *s, by=1.0, dt=torch.bfloat16: (torch.randn(s, generator=g) * by).to(dt).cuda()
    w1, w2, gate = r(2 * H, C, by=0.06), r(C, H, by=0.06), r(B, 3, C, dt=torch.float32)
    x, d = r(B, S, C), r(B, S, C)

    def step():
        out, h, dx, dy, dxx = (torch.empty_like(x) for _ in range(5))
        kept = ffn.keep()
        ffn.forward(x, w1, w2, out, kept=kept)
        norm.forward(x, None, out, h, gate=gate)
        n = norm.backward(d, h, dx, y=out, dy_out=dy, gate=gate)
        return [out, dx, dy, n["dgate"], dxx, *ffn.backward(dy, x, w1, w2, kept, dxx)[:2]]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        graph.replay()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
