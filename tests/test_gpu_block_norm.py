"""The norm between two branches on the GPU against the 64-bit statement, whose bounds of 32-bit arithmetic stand there; a result is rounded once to
its type: half a step of it."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm
from tests import _block64 as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
NAMES = ("gate", "scale", "shift", "weight", "bias", "post_weight")


def check(got, want, what):
    ref, err = want
    got, half = got.detach().cpu(), torch.finfo(got.dtype).eps / 2
    off = (got.double() - ref).abs()
    tol = half * ref.abs() + (1 + half) * err + torch.finfo(got.dtype).tiny
    assert bool((off <= tol).all()), f"{what}: {off.max():.3e}, worst over its tolerance {(off / tol).nan_to_num(posinf=9e9).max():.2f}"


# B, S, C, dtype, stream, norm, post, mod_tokens, parameters, branch
ALL = NAMES
CASES = [
    (1, 1, 8, "bf16", "bf16", "layer", "none", 0, (), False),
    (4, 1, 1536, "bf16", "bf16", "layer", "none", 0, ("gate", "scale", "shift"), True),
    (1, 7, 72, "bf16", "f32", "rms", "rms", 3, ALL[:4] + ALL[5:], True),
    (2, 33, 264, "bf16", "bf16", "layer", "layer", 8, ALL, True),
    (3, 20, 1000, "f32", "f32", "layer", "rms", 7, ALL, True),
    (1, 50, 1536, "bf16", "bf16", "rms", "none", 1, ("gate", "scale", "shift", "weight"), True),
    (2, 200, 2056, "bf16", "f32", "layer", "none", 64, ("scale", "shift", "bias"), True),
    (1, 40, 5120, "bf16", "bf16", "layer", "layer", 0, ALL, True),
    (1, 9, 8192, "f32", "f32", "layer", "layer", 4, ALL, True),
    (2, 17, 4104, "bf16", "f32", "rms", "rms", 0, ("weight", "post_weight"), True),
    (1, 700, 128, "bf16", "bf16", "layer", "none", 100, ("scale",), False),
    (1, 1300, 512, "f32", "f32", "rms", "none", 0, ("gate", "shift"), True),
    (2, 5, 3032, "bf16", "bf16", "layer", "none", 2, ("bias",), False),
]


def wide(x, pad):
    if x is None:
        return None
    big = torch.full((*x.shape[:-1], x.shape[-1] + pad), 7.0, dtype=x.dtype, device=x.device)
    big[..., : x.shape[-1]] = x
    return big[..., : x.shape[-1]]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward_and_backward(i):
    B, S, C, dtype, stream, norm, post, tokens, has, branch = CASES[i]
    g = torch.Generator().manual_seed(i)
    G = -(-S // tokens) if tokens else 1
    r = lambda *s, at=0.0, by=1.0: at + by * torch.randn(s, generator=g)
    x = (r(B, S, C, at=0.7) * torch.exp(0.7 * r(C))).to(DT[stream])
    y = r(B, S, C, at=-0.2, by=2.0).to(DT[dtype]) if branch else None
    d, d_h = r(B, S, C).to(DT[dtype]), r(B, S, C).to(DT[stream])
    p = {n: None for n in NAMES}
    p |= {n: r(B, G, C, by=0.5) if n in NAMES[:3] else r(C, at=1.0, by=0.2) for n in has}
    D = lambda t: None if t is None else t.double()
    p64 = {n: D(t) for n, t in p.items()}
    (h, he), (out, oe) = P.block_norm(D(x), D(y), norm, post, p64, tokens)
    op = BlockNorm(vb.make_norm_shape(B, S, C, dtype, stream, norm, post, tokens))
    # rows of gate, scale and shift as slices of one tensor
    six = torch.zeros((B, 3, G, C), device="cuda")
    pc = {n: None if t is None else t.cuda() for n, t in p.items()}
    for k, n in enumerate(NAMES[:3]):
        if pc[n] is not None:
            six[:, k] = pc[n]
            pc[n] = six[:, k]
    c = lambda t: None if t is None else t.cuda()
    got_h = torch.full((B, S, C + 8), 7.0, dtype=DT[stream], device="cuda")
    got = torch.full((B, S, C + 8), 7.0, dtype=DT[dtype], device="cuda")
    op.forward(wide(c(x), 8), got[..., :C], wide(c(y), 16), got_h[..., :C], **pc)
    check(got_h[..., :C], (h, he), "h")
    check(got[..., :C], (out, oe), "out")
    assert bool((got[..., C:] == 7).all()) and bool((got_h[..., C:] == 7).all())
    # in place, and each result alone
    onto, alone = c(x).clone(), torch.empty((B, S, C), dtype=DT[dtype], device="cuda")
    op.forward(c(x), alone, c(y), **pc)
    op.forward(onto, None, c(y), onto, **pc)
    assert torch.equal(alone, got[..., :C]) and torch.equal(onto, got_h[..., :C])

    h64 = D(onto.cpu())
    want = P.block_norm_grad(D(d), h64, D(d_h), D(y), norm, post, p64, tokens)
    dx, dy = torch.empty_like(onto), None if y is None else torch.empty_like(c(y))
    grads = op.backward(c(d), onto, dx, c(d_h), c(y), dy, **pc)
    check(dx, want["dx"], "dx")
    if branch:
        check(dy, want["dy"], "dy")
    for n, t in grads.items():
        assert (t is None) == (n not in want)
        if t is not None:
            check(t, want[n], n)
    # again bit for bit: over its inputs, from strided rows
    over, over_d = wide(c(d_h), 8), wide(c(d), 8)
    again = op.backward(over_d, wide(onto, 8), over, over, wide(c(y), 8), over_d if branch else None, **pc)
    assert torch.equal(over, dx) and (not branch or torch.equal(over_d, dy))
    for n, t in grads.items():
        assert t is None or torch.equal(t, again[n])
    # without what else arrives at h
    want = P.block_norm_grad(D(d), h64, None, D(y), norm, post, p64, tokens)
    op.backward(c(d), onto, dx, None, c(y), dy, **pc)
    check(dx, want["dx"], "dx alone")


def test_constant_rows_and_values_that_are_not_finite():
    for norm in ("layer", "rms"):
        op = BlockNorm(vb.make_norm_shape(1, 300, 264, "bf16", norm=norm))
        x = torch.randn((1, 300, 264), device="cuda").to(torch.bfloat16)
        a, b = torch.empty_like(x), torch.empty_like(x)
        op.forward(x, a)
        x[0, 3], x[0, 4], x[0, 7, 1], x[0, 9, 2] = 0.0, 2.0, float("nan"), float("inf")
        op.forward(x, b)
        assert bool((b[0, 3] == 0).all()) and bool((b[0, 4] == (0 if norm == "layer" else 1)).all())
        assert bool(b[0, 7].isnan().all()) and bool(b[0, 9, 2].isnan())
        clean = torch.ones(300, dtype=torch.bool, device="cuda")
        clean[[3, 4, 7, 9]] = False
        assert torch.equal(a[:, clean], b[:, clean])


def test_a_gate_shared_by_all_samples():
    B, S, C = 3, 40, 136
    op = BlockNorm(vb.make_norm_shape(B, S, C, "bf16", mod_tokens=9))
    x, y = (torch.randn((B, S, C), device="cuda").to(torch.bfloat16) for _ in range(2))
    gate = torch.randn((1, 5, C), device="cuda")
    res = []
    for g in (gate, gate.expand(B, 5, C), gate.expand(B, 5, C).contiguous(), gate.transpose(1, 2).contiguous().transpose(1, 2)):
        out, h = torch.empty_like(x), torch.empty_like(x)
        op.forward(x, out, y, h, gate=g)
        dx, dy = torch.empty_like(x), torch.empty_like(x)
        dg = op.backward(out, h, dx, x, y, dy, gate=g)["dgate"]
        assert dg.shape == (B, 5, C)
        res.append((out, h, dx, dy, dg))
    for r in res[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, res[0]))


def test_refusals():
    op = BlockNorm(vb.make_norm_shape(2, 16, 64, "bf16", stream_dtype="f32", mod_tokens=5))
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    f = lambda *s: z(*s, dt=torch.float32)
    for bad in (vb.make_norm_shape(2, 16, 60, "bf16"), vb.make_norm_shape(2, 16, 8200, "bf16"), vb.make_norm_shape(2, 16, 64, "f32", stream_dtype="bf16")):
        with pytest.raises(ValueError):
            BlockNorm(bad)
    x, out = f(2, 16, 64), z(2, 16, 64)
    for bad in (dict(x=z(2, 16, 64)), dict(out=f(2, 16, 64)), dict(out=None), dict(out=z(1, 16, 64).expand(2, 16, 64)), dict(y=f(2, 16, 64)), dict(h_out=f(2, 16, 65)[..., :64]),
                dict(gate=f(2, 3, 64)), dict(scale=z(2, 4, 64)), dict(weight=f(72)), dict(weight=f(128)[::2]), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            op.forward(**{"x": x, "out": out, **bad})
    for bad in (dict(dy_out=out), dict(gate=f(2, 4, 64)), dict(dx_out=out), dict(h=out), dict(post_weight=f(64))):
        with pytest.raises(ValueError):
            op.backward(**{"d_out": out, "h": x, "dx_out": f(2, 16, 64), **bad})
