"""Plain 64-bit statements of linear layers with their epilogues, feed-forward blocks and the norm between two branches: what the tests of those
operators compare with.  Torch on the CPU, fp64, no code of the package.  Next to each result stands a bound of what 32-bit arithmetic may
add to it, ahead of the rounding of the result itself; h is the half step of the type that tensors are held in between (0: none is).

Sums of n products: a rounding each, n 2^-24 of the magnitudes added (16 more for sums of parts).  The logistic function of bf16's kernels: exp to
26 units in its last place where the result is not yet 0 or 1 (|x| < 20), 3.1e-6 of it, s (1 - s) <= 1/4 of that in s; times u, whose
u s (1 - s) is below 0.3: 1e-6, and 4e-7 |u| for the other roundings.  Slopes: |u s (1 - s) z'| < 1.2 with twice that relative error: 1e-5.  fp32's
kernels have exp to 2 units: a tenth of both, and 4e-7."""
import math

import torch

EPS = 2.0 ** -24


def errs(f32):
    """(absolute error of an activation, of its slope)"""
    return (4e-7, 2e-6) if f32 else (1e-6, 1e-5)


def act(name, u):
    if name == "gelu":
        return 0.5 * u * (1 + torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))
    return u / (1 + torch.exp(-u)) if name == "silu" else u.clone()


def slope(name, u):
    if name == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3))
        return 0.5 * (1 + t) + 0.5 * u * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * u * u)
    if name == "silu":
        s = 1 / (1 + torch.exp(-u))
        return s + u * s * (1 - s)
    return torch.ones_like(u)


def product(x, w, xe=None):
    """x [.., K] times w [N, K] transposed, and the bound of its error (xe: that of x)."""
    y = x @ w.T
    e = (x.shape[-1] + 16) * EPS * (x.abs() @ w.abs().T)
    return y, e if xe is None else e + xe @ w.abs().T


def through(name, gated, u, ue, f32):
    """act(u), or act(first half) * second half."""
    ea = errs(f32)[0]
    if name == "none":
        ea = 0.0
    a, ae = (u.chunk(2, -1)[0], ue.chunk(2, -1)[0]) if gated else (u, ue)
    y, ye = act(name, a), 1.13 * ae + ea + (0.0 if name == "none" else 4e-7 * a.abs())
    if gated:
        b, be = u.chunk(2, -1)[1], ue.chunk(2, -1)[1]
        y, ye = y * b, ye * b.abs() + y.abs() * be + EPS * (y * b).abs()
    return y, ye


def rows_of(g, S, tokens):
    """[B, groups, C] as [B, S, C]"""
    at = torch.arange(S, device=g.device) // (tokens if tokens else S)
    return g[:, at]


def group_sums(x, tokens):
    B, S, C = x.shape
    tokens = tokens or S
    out = torch.zeros(B, -(-S // tokens), C, dtype=x.dtype, device=x.device)
    return out.index_add_(1, torch.arange(S, device=x.device) // tokens, x)


def linear(x, w, b, name="none", gated=False, gate=None, tokens=0, residual=None, f32=False, order=None, xe=None):
    """((out, error), (kept, error)); x [B, S, K] in whatever order, order[p]: the token of out of its row p."""
    u, ue = product(x, w, xe)
    if b is not None:
        u = u + b
        ue = ue + EPS * u.abs()
    y, ye = through(name, gated, u, ue, f32)
    if order is not None:
        y, ye = (torch.zeros_like(t).index_copy_(1, order, t) for t in (y, ye))
    if gate is not None:
        g = rows_of(gate, x.shape[1], tokens)
        y, ye = y * g, ye * g.abs() + EPS * (y * g).abs()
    if residual is not None:
        y, ye = y + residual, ye + EPS * (y.abs() + residual.abs())
    return (y, ye), (u, ue)


def sums_bound(rows):
    return (96 + rows / 64) * EPS


def du_of(d, kept, name, gated, gate, tokens, f32, order=None, de=None):
    """Gradient of the product in the order of x: ((du, error), (dgate, error) or None)."""
    es = errs(f32)[1] if name != "none" else 0.0
    de = torch.zeros_like(d) if de is None else de
    dg = None
    zero = None if kept is None else torch.zeros_like(kept)
    if gate is not None:
        y, ye = through(name, gated, kept, zero, f32)
        if order is not None:
            y, ye = (torch.zeros_like(t).index_copy_(1, order, t) for t in (y, ye))
        dg = group_sums(d * y, tokens), group_sums(d.abs() * ye + sums_bound(d.shape[1]) * (d * y).abs() + de * y.abs(), tokens)
        g = rows_of(gate, d.shape[1], tokens)
        d, de = d * g, de * g.abs() + EPS * (d * g).abs()
    if order is not None:
        d, de = d[:, order], de[:, order]
    if name == "none" and not gated:
        return (d, de), dg
    if gated:
        a, b = kept.chunk(2, -1)
        sl, (y, ye) = slope(name, a), through(name, False, a, torch.zeros_like(a), f32)
        da, db = d * b * sl, d * y
        dae = de * (b * sl).abs() + (d * b).abs() * (es + 4 * EPS)
        dbe = de * y.abs() + d.abs() * (ye + 2 * EPS * y.abs())
        return (torch.cat([da, db], -1), torch.cat([dae, dbe], -1)), dg
    sl = slope(name, kept)
    return (d * sl, de * sl.abs() + d.abs() * (es + 4 * EPS)), dg


def weight_grad(du, due, x, xe=None):
    f, fe, g = du.flatten(0, 1), due.flatten(0, 1), x.flatten(0, 1)
    e = fe.T @ g.abs() + (f.shape[0] + 16) * EPS * (f.abs().T @ g.abs())
    return f.T @ g, e if xe is None else e + (f.abs() + fe).T @ xe.flatten(0, 1)


def input_grad(du, due, w):
    return du @ w, due @ w.abs() + (du.shape[-1] + 16) * EPS * (du.abs() @ w.abs())


def column_sums(du, due):
    rows = du.shape[0] * du.shape[1]
    return du.sum((0, 1)), (due + sums_bound(rows) * du.abs()).sum((0, 1))


# ------------------------------------------------------------------------------------------------ norms
SUM = 5e-6           # sums of a row: at most 48 terms per thread and a tree of 8 more, 4e-6 of the magnitudes; roots and products


def normed(kind, v, ve, eps=1e-6):
    """((n, error), factor)"""
    if kind == "none":
        return (v, ve), torch.ones_like(v[..., :1])
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
    me = SUM * v.abs().mean(-1, keepdim=True) + ve.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    c = v - mean
    r = 1 / torch.sqrt(c.square().mean(-1, keepdim=True) + eps)
    ce = ve + me
    n = c * r
    # r: the square root halves the relative error of the mean of squares
    re = SUM + (n.abs() * ce * r).mean(-1, keepdim=True)
    return (n, ce * r + n.abs() * re), r


def block_norm(x, y, kind, post, p, tokens, eps=1e-6):
    """((h, error), (out, error)); p: dict of gate, scale, shift, weight, bias, post_weight or None"""
    S = x.shape[1]
    row = lambda n: rows_of(p[n], S, tokens)
    h, he = x, torch.zeros_like(x)
    if y is not None:
        (z, ze), _ = normed(post, y, torch.zeros_like(y), eps)
        if p.get("post_weight") is not None:
            z, ze = z * p["post_weight"], ze * p["post_weight"].abs() + EPS * (z * p["post_weight"]).abs()
        if p.get("gate") is not None:
            z, ze = z * row("gate"), ze * row("gate").abs()
        h, he = x + z, ze + 2 * EPS * (x.abs() + z.abs())
    (n, ne), _ = normed(kind, h, he, eps)
    for name in ("weight", "bias", "scale", "shift"):
        if p.get(name) is None:
            continue
        f = p[name] if name in ("weight", "bias") else row(name)
        if name in ("weight", "scale"):
            f = f if name == "weight" else 1 + f
            n, ne = n * f, ne * f.abs() + 2 * EPS * (n * f).abs()
        else:
            n, ne = n + f, ne + EPS * (n.abs() + f.abs())
    return (h, he), (n, ne)


def block_norm_grad(d, h, d_h, y, kind, post, p, tokens, eps=1e-6):
    """dict of name: (gradient, error) for dx, dy and those of p"""
    B, S, C = h.shape
    out = {}
    row = lambda n: rows_of(p[n], S, tokens)
    has = lambda n: p.get(n) is not None
    cols = lambda v, e: (v.sum((0, 1)), (e + sums_bound(B * S) * v.abs()).sum((0, 1)))
    groups = lambda v, e: (group_sums(v, tokens), group_sums(e + sums_bound(S) * v.abs(), tokens))
    (n, ne), r = normed(kind, h, torch.zeros_like(h), eps)
    m, me = n, ne
    if has("weight"):
        m, me = m * p["weight"], me * p["weight"].abs()
    if has("bias"):
        m = m + p["bias"]
    magnitude = (n * (p["weight"] if has("weight") else 1)).abs() + (p["bias"].abs() if has("bias") else 0)
    if has("scale"):
        out["dscale"] = groups(d * m, d.abs() * (me + 4 * EPS * magnitude) + sums_bound(S) * d.abs() * magnitude)
    if has("shift"):
        out["dshift"] = groups(d, torch.zeros_like(d))
    if has("scale"):
        d = d * (1 + row("scale"))
    if has("bias"):
        out["dbias"] = cols(d, 4 * EPS * d.abs())
    if has("weight"):
        out["dweight"] = cols(d * n, d.abs() * ne + 4 * EPS * (d * n).abs())
        d = d * p["weight"]

    def back(d, de, n, ne, r, kind):
        if kind == "none":
            return d, de
        along, alonge = (d * n).mean(-1, keepdim=True), (d.abs() * ne + de * n.abs() + 2 * SUM * (d * n).abs()).mean(-1, keepdim=True)
        g, ge = d - n * along, de + ne * along.abs() + n.abs() * alonge + 4 * EPS * (d.abs() + (n * along).abs())
        if kind == "layer":
            g, ge = g - d.mean(-1, keepdim=True), ge + (de + 2 * SUM * d.abs()).mean(-1, keepdim=True)
        # (r is off by what n is off by, relatively)
        return r * g, r * (ge + g.abs() * (2 * SUM + (n.abs() * ne).mean(-1, keepdim=True)))

    dh, dhe = back(d, 4 * EPS * d.abs(), n, ne, r, kind)
    if d_h is not None:
        dh, dhe = dh + d_h, dhe + 2 * EPS * (dh.abs() + d_h.abs())
    out["dx"] = (dh, dhe)
    if y is None:
        return out
    (z, ze), rz = normed(post, y, torch.zeros_like(y), eps)
    g = dh, dhe
    if has("gate"):
        pw = p["post_weight"] if has("post_weight") else 1.0
        out["dgate"] = groups(dh * z * pw, (dhe * z.abs() + dh.abs() * ze + 4 * EPS * (dh * z).abs()) * (abs(pw) if isinstance(pw, float) else pw.abs()))
        g = g[0] * row("gate"), g[1] * row("gate").abs() + EPS * (g[0] * row("gate")).abs()
    if has("post_weight"):
        out["dpost_weight"] = cols(g[0] * z, g[1] * z.abs() + g[0].abs() * ze + 4 * EPS * (g[0] * z).abs())
        g = g[0] * p["post_weight"], g[1] * p["post_weight"].abs() + EPS * (g[0] * p["post_weight"]).abs()
    out["dy"] = back(*g, z, ze, rz, post)
    return out
