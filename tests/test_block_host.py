"""Linear layers, feed-forward blocks and block norms without a GPU: the 64-bit statements against gradients by automatic differentiation and
by differences, and the entry points' refusals (no kernel is launched)."""
import ctypes

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from tests import _block64 as P


def rnd(*s, seed=0):
    return torch.randn(s, generator=torch.Generator().manual_seed(seed + sum(s)), dtype=torch.float64)


@pytest.mark.parametrize("name,gated", [("none", False), ("gelu", False), ("silu", True), ("none", True)])
def test_statement_of_a_linear_layers_gradients(name, gated):
    B, S, K, N, tokens = 2, 7, 6, 5, 3
    rows = 2 * N if gated else N
    order = torch.randperm(S, generator=torch.Generator().manual_seed(1))
    x, w, b, gate, res, d = rnd(B, S, K), rnd(rows, K, seed=1), rnd(rows), rnd(B, 3, N), rnd(B, S, N, seed=2), rnd(B, S, N, seed=3)
    leaves = [t.clone().requires_grad_() for t in (x, w, b, gate)]
    out = P.linear(leaves[0], leaves[1], leaves[2], name, gated, leaves[3], tokens, res, order=order)[0][0]
    want = torch.autograd.grad(out, leaves, d)
    kept = P.linear(x, w, b, name, gated)[1][0]
    (du, due), dg = P.du_of(d, kept, name, gated, gate, tokens, True, order)
    got = (P.input_grad(du, due, w)[0], P.weight_grad(du, due, x)[0], P.column_sums(du, due)[0], dg[0])
    for a, c in zip(got, want):
        assert torch.allclose(a, c, rtol=1e-11, atol=1e-11)
    # and against a difference
    u, h = rnd(B, S, K, seed=9), 1e-5
    val = lambda t: (P.linear(t, w, b, name, gated, gate, tokens, res, order=order)[0][0] * d).sum()
    assert abs((val(x + h * u) - val(x - h * u)) / (2 * h) - (got[0] * u).sum()) < 1e-6 * (got[0] * u).abs().sum()


@pytest.mark.parametrize("kind,post,branch", [("layer", "none", True), ("rms", "rms", True), ("layer", "layer", True), ("rms", "none", False)])
def test_statement_of_the_norms_gradients(kind, post, branch):
    B, S, C, tokens = 2, 5, 8, 2
    x, y, d, d_h = rnd(B, S, C), rnd(B, S, C, seed=1) if branch else None, rnd(B, S, C, seed=2), rnd(B, S, C, seed=3)
    p = {"scale": rnd(B, 3, C), "shift": rnd(B, 3, C, seed=1), "weight": rnd(C), "bias": rnd(C, seed=1)}
    if branch:
        p |= {"gate": rnd(B, 3, C, seed=2), "post_weight": rnd(C, seed=2)}
    leaves = {n: t.clone().requires_grad_() for n, t in p.items()} | {"x": x.clone().requires_grad_()}
    if branch:
        leaves["y"] = y.clone().requires_grad_()
    (h, _), (out, _) = P.block_norm(leaves["x"], leaves.get("y"), kind, post, leaves, tokens)
    want = dict(zip(leaves, torch.autograd.grad([out, h], list(leaves.values()), [d, d_h])))
    got = P.block_norm_grad(d, h.detach(), d_h, y, kind, post, p, tokens)
    assert set(got) == {"d" + n for n in want}
    for n, g in want.items():
        assert torch.allclose(got["d" + n][0], g, rtol=1e-9, atol=1e-10), n


FAKE, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(None)          # aligned, never dereferenced: checks fail first
ODD = ctypes.c_void_p(0x1008)


def pair(*st):
    return (ctypes.c_int64 * 2)(*st)


def forward(s, x=FAKE, xs=pair(16 * 64, 64), w=FAKE, b=NULL, gate=NULL, gs=pair(0, 0), res=NULL, rs=pair(16 * 32, 32), out=FAKE,
            os_=pair(16 * 32, 32), kept=NULL, perm=NULL, ws=FAKE, n=1 << 40):
    return vb.lib().vmoba_linear(ctypes.byref(s), x, xs, w, b, gate, gs, res, rs, out, os_, kept, perm, NULL, ws, n, NULL)


def test_linear_refusals():
    L = vb.make_linear_shape
    good = L(2, 16, 64, 32, "bf16")
    assert vb.linear_workspace_bytes(good) > 0 and vb.linear_workspace_bytes(good, True) > 0
    for kw in (dict(x=NULL), dict(w=NULL), dict(out=NULL), dict(ws=NULL), dict(x=ODD), dict(b=ODD), dict(out=ODD), dict(kept=ODD), dict(res=ODD),
               dict(gate=ODD, gs=pair(32, 32)), dict(xs=None), dict(os_=None), dict(xs=pair(16 * 64, 63)), dict(xs=pair(16 * 64, 56)),
               dict(xs=pair(0, 64)), dict(os_=pair(16 * 32, 0)), dict(os_=pair(-512, 32)), dict(res=FAKE, rs=pair(16 * 32, 28)), dict(gate=FAKE, gs=pair(8, 0)),
               dict(gate=FAKE, gs=None), dict(perm=FAKE)):
        assert forward(good, **kw) == vb.ERR_ARG, kw
    assert forward(good, n=16) == vb.ERR_WORKSPACE
    for bad, code in ((L(2, 16, 60, 32, "bf16"), vb.ERR_SHAPE), (L(2, 16, 64, 36, "f32"), vb.ERR_SHAPE), (L(0, 16, 64, 32, "bf16"), vb.ERR_SHAPE),
                      (L(2, 0, 64, 32, "bf16"), vb.ERR_SHAPE), (L(1 << 16, 1 << 16, 64, 32, "bf16"), vb.ERR_SHAPE), (L(2, 16, 1 << 21, 32, "bf16"), vb.ERR_SHAPE),
                      (L(2, 16, 64, 32, 5), vb.ERR_ARG), (L(2, 16, 64, 32, "bf16", 9), vb.ERR_ARG), (L(2, 16, 64, 32, "bf16", gated=2), vb.ERR_ARG),
                      (L(2, 16, 64, 32, "bf16", heads=2), vb.ERR_SHAPE), (L(2, 16, 64, 32, "bf16", heads=-1), vb.ERR_ARG),
                      (L(2, 16, 64, 32, "bf16", gate_tokens=-1), vb.ERR_ARG)):
        assert forward(bad) == code
        assert vb.linear_workspace_bytes(bad) == 0 and vb.linear_workspace_bytes(bad, True) == 0 and vb.ffn_workspace_bytes(bad) == 0
    assert vb.lib().vmoba_linear(None, *[None] * 14, 0, None) == vb.ERR_ARG


def test_linear_backward_and_feed_forward_refusals():
    lib, L = vb.lib(), vb.make_linear_shape
    plain, acts = L(2, 16, 64, 32, "bf16"), L(2, 16, 64, 32, "bf16", "gelu")
    xs, os_ = pair(16 * 64, 64), pair(16 * 32, 32)

    def bwd(s, d=FAKE, x=FAKE, w=FAKE, kept=FAKE, gate=NULL, dx=FAKE, dxs=xs, dw=FAKE, db=NULL, dg=NULL, perm=NULL, ws=FAKE, n=1 << 40):
        return lib.vmoba_linear_bwd(ctypes.byref(s), d, os_, x, xs, w, kept, gate, pair(0, 0), dx, dxs, dw, db, dg, perm, NULL, ws, n, NULL)

    for s, kw in ((plain, dict(d=NULL)), (plain, dict(w=NULL)), (plain, dict(x=NULL)), (acts, dict(kept=NULL)), (plain, dict(dg=FAKE)),
                  (plain, dict(gate=FAKE, dg=FAKE, kept=NULL)), (plain, dict(perm=FAKE)), (plain, dict(dxs=pair(0, 64))), (plain, dict(db=ODD)), (plain, dict(ws=NULL))):
        assert bwd(s, **kw) == vb.ERR_ARG, kw
    assert bwd(plain, n=16) == vb.ERR_WORKSPACE

    def ffn(s, x=FAKE, wu=FAKE, wd=FAKE, gate=NULL, out=FAKE, os_=xs, ws=FAKE, n=1 << 40):
        return lib.vmoba_ffn(ctypes.byref(s), x, xs, wu, NULL, wd, NULL, gate, pair(0, 0), NULL, xs, out, os_, NULL, NULL, NULL, ws, n, NULL)

    for kw in (dict(x=NULL), dict(wu=NULL), dict(wd=NULL), dict(out=NULL), dict(out=ODD), dict(os_=pair(16 * 64, 32)), dict(ws=NULL)):
        assert ffn(acts, **kw) == vb.ERR_ARG, kw
    assert ffn(acts, n=16) == vb.ERR_WORKSPACE
    assert ffn(L(2, 16, 128, 32, "bf16", heads=1)) == vb.ERR_ARG and vb.ffn_workspace_bytes(L(2, 16, 128, 32, "bf16", heads=1)) == 0

    def ffn_bwd(s, x=FAKE, wu=FAKE, wd=FAKE, up=FAKE, down=NULL, gate=NULL, dx=FAKE, dg=NULL, n=1 << 40):
        return lib.vmoba_ffn_bwd(ctypes.byref(s), FAKE, xs, x, xs, wu, wd, up, down, gate, pair(0, 0), dx, xs, FAKE, NULL, FAKE, NULL, dg, NULL, FAKE, n, NULL)

    for kw in (dict(x=NULL), dict(wu=NULL), dict(wd=NULL), dict(up=NULL), dict(dg=FAKE), dict(gate=FAKE, dg=FAKE), dict(dx=ODD)):
        assert ffn_bwd(acts, **kw) == vb.ERR_ARG, kw
    assert ffn_bwd(acts, n=16) == vb.ERR_WORKSPACE


def test_norm_refusals():
    lib, N = vb.lib(), vb.make_norm_shape
    good = N(2, 16, 64, "bf16", mod_tokens=5)
    st = pair(16 * 64, 64)

    def fwd(s, m=None, x=FAKE, xs=st, y=NULL, h=NULL, hs=st, out=FAKE, os_=st):
        m = vb.norm_params() if m is None else m
        return lib.vmoba_block_norm(ctypes.byref(s), ctypes.byref(m), x, xs, y, st, h, hs, out, os_, NULL, NULL)

    rows = lambda at, *strides: vb.NormParams(at, None, None, pair(*strides))
    for kw in (dict(x=NULL), dict(out=NULL), dict(x=ODD), dict(xs=None), dict(xs=pair(16 * 64, 60)), dict(os_=pair(16 * 64, 0)), dict(h=FAKE, hs=pair(0, 64)),
               dict(y=ODD), dict(m=rows(0x1004, 256, 64)), dict(m=rows(0x1000, 256, 62)), dict(m=rows(0x1000, 256, 32)), dict(m=vb.NormParams(weight=0x1004))):
        assert fwd(good, **kw) == vb.ERR_ARG, kw
    for bad, code in ((N(2, 16, 60, "bf16"), vb.ERR_SHAPE), (N(2, 16, 8200, "bf16"), vb.ERR_SHAPE), (N(0, 16, 64, "bf16"), vb.ERR_SHAPE),
                      (N(1 << 16, 1 << 16, 64, "bf16"), vb.ERR_SHAPE), (N(2, 16, 64, 7), vb.ERR_ARG), (N(2, 16, 64, "bf16", norm="none"), vb.ERR_ARG),
                      (N(2, 16, 64, "bf16", post_norm=5), vb.ERR_ARG), (N(2, 16, 64, "bf16", mod_tokens=-1), vb.ERR_ARG),
                      (N(2, 16, 64, "bf16", eps=-1.0), vb.ERR_ARG), (N(2, 16, 64, "bf16", eps=float("nan")), vb.ERR_ARG),
                      (N(2, 16, 64, "f32", stream_dtype="bf16"), vb.ERR_NOT_IMPLEMENTED)):
        assert fwd(bad) == code
        assert vb.block_norm_workspace_bytes(bad) == 0

    def bwd(s, m=None, h=FAKE, d_h=NULL, y=NULL, dx=FAKE, dxs=st, dy=NULL, n=1 << 40, ws=FAKE, **grads):
        m = vb.norm_params() if m is None else m
        return lib.vmoba_block_norm_bwd(ctypes.byref(s), ctypes.byref(m), FAKE, st, h, st, d_h, st, y, st, dx, dxs, dy, st,
                                        ctypes.byref(vb.NormGrads(**grads)), NULL, ws, n, NULL)

    gated = vb.NormParams(0x1000, None, None, pair(256, 64))
    for kw in (dict(h=NULL), dict(dx=NULL), dict(dy=FAKE), dict(dxs=pair(0, 64)), dict(scale=0x1000), dict(gate=0x1000), dict(m=gated, gate=0x1000),
               dict(m=gated, y=FAKE, gate=0x1004), dict(weight=0x1000), dict(ws=NULL)):
        assert bwd(good, **kw) == vb.ERR_ARG, kw
    assert bwd(good, n=16) == vb.ERR_WORKSPACE
