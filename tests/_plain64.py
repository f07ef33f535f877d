"""Plain 64-bit statements of rotary positions with norm, and of attention over key ranges with capped scores: what the GPU tests of
those operators compare with.  Torch on the CPU, fp64, no code of the package.  Next to each result stands the sum of the magnitudes
that it was added up from, which is what the tolerances of 32-bit sums are stated in."""
import math

import torch


# ------------------------------------------------------------------------------------------------ rotary
def pair_channels(layout, pairs):
    i = torch.arange(pairs)
    return (i, i + pairs) if layout == "half" else (2 * i, 2 * i + 1)


def rotate(x, positions, freq, axis, layout, mscale=1.0, sign=1.0):
    """x [B, S, h, d] fp64; positions [S, axes] or [B, S, axes].  (result, magnitudes)."""
    pos = positions.double() if positions.dim() == 3 else positions.double()[None]
    a = (pos[..., axis.long()] * freq.double())[:, :, None]
    c, s = mscale * torch.cos(a), sign * mscale * torch.sin(a)
    i0, i1 = pair_channels(layout, freq.numel())
    out, mag = x.clone(), x.abs()
    x0, x1 = x[..., i0], x[..., i1]
    out[..., i0], out[..., i1] = x0 * c - x1 * s, x1 * c + x0 * s
    mag[..., i0] = mag[..., i1] = mscale * (x0.abs() + x1.abs())
    return out, mag


def norm_rotate(x, w, positions, freq, axis, layout, norm, mscale=1.0, eps=1e-6):
    x = x.double()
    B, S, h, d = x.shape
    if norm != "none":
        over = (2, 3) if norm == "row" else (3,)
        r = 1.0 / torch.sqrt(x.square().mean(over, keepdim=True) + eps)
        ww = torch.ones((), dtype=torch.float64) if w is None else w.double().view(h, d) if norm == "row" else w.double()
        x = x * r * ww
    return rotate(x, positions, freq, axis, layout, mscale)


def norm_rotate_grad(dy, x, w, positions, freq, axis, layout, norm, mscale=1.0, eps=1e-6):
    """((dx, magnitudes), (dw, magnitudes)); dw None without a norm."""
    g, gmag = rotate(dy.double(), positions, freq, axis, layout, mscale, -1.0)
    if norm == "none":
        return (g, gmag), None
    x = x.double()
    B, S, h, d = x.shape
    over = (2, 3) if norm == "row" else (3,)
    ww = torch.ones((), dtype=torch.float64) if w is None else w.double().view(h, d) if norm == "row" else w.double()
    r = 1.0 / torch.sqrt(x.square().mean(over, keepdim=True) + eps)
    s = g * ww
    dx = r * (s - x * r.square() * (s * x).mean(over, keepdim=True))
    mag = r * (gmag * ww.abs() + x.abs() * r.square() * (gmag * ww.abs() * x.abs()).mean(over, keepdim=True))
    dims = (0, 1) if norm == "row" else (0, 1, 2)
    return (dx, mag), ((g * x * r).sum(dims).reshape(-1), (gmag * (x * r).abs()).sum(dims).reshape(-1))


def block_order(x, grid, block):
    """[B, S, h, d] raster -> [B, h, S, d], blocks and slots with the last axis fastest (Eq. 1)."""
    B, S, h, d = x.shape
    n = [g // b for g, b in zip(grid, block)]
    x = x.reshape(B, n[0], block[0], n[1], block[1], n[2], block[2], h, d).permute(0, 7, 1, 3, 5, 2, 4, 6, 8)
    return x.reshape(B, h, S, d)


# ------------------------------------------------------------------------------------------------ attention over key ranges
def range_attention(q, k, v, ranges, cap=0.0, scale=None, do=None):
    """q [B, Sq, h, d], k and v [B, Sk, hk, d], ranges [1 or B, Sq, 2].  dict of o, lse [B, h, Sq] and, with do, dq, dk, dv, of the
    magnitudes o_mag, dq_mag, dk_mag, dv_mag, and the largest |q| |k| scale."""
    q, k, v = q.double(), k.double(), v.double()
    B, Sq, h, d = q.shape
    Sk, hk = k.shape[1], k.shape[2]
    G = h // hk
    scale = d ** -0.5 if scale is None else scale
    r = ranges.long().expand(B, Sq, 2)
    key = torch.arange(Sk)
    seen = ((key >= r[..., :1]) & (key < r[..., 1:]))[:, None, None]                   # [B, 1, 1, Sq, Sk]
    qh = q.view(B, Sq, hk, G, d).permute(0, 2, 3, 1, 4)
    kh, vh = k.permute(0, 2, 1, 3)[:, :, None], v.permute(0, 2, 1, 3)[:, :, None]
    kh, vh = (torch.where(torch.isfinite(x), x, torch.zeros((), dtype=x.dtype)) if not torch.isfinite(x).all() else x for x in (kh, vh))
    qh = torch.where(torch.isfinite(qh), qh, torch.zeros((), dtype=qh.dtype))          # (rows that see nothing may hold anything)
    t = qh @ kh.transpose(-1, -2) * scale
    u = torch.tanh(t / cap) if cap else None
    if cap:
        t = cap * u
    t = t.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(t, -1)
    p = torch.where(seen, torch.exp(t - lse.clamp(min=-1e300)[..., None]), torch.zeros((), dtype=t.dtype))
    back = lambda x, n, heads: x.permute(0, 3, 1, 2, 4).reshape(B, n, heads, d)
    norms = qh.norm(dim=-1).amax() * kh.norm(dim=-1).amax() * scale
    out = {"top": float(norms), "o": back(p @ vh, Sq, h), "o_mag": back(p @ vh.abs(), Sq, h), "lse": lse.reshape(B, h, Sq)}
    if do is not None:
        doh = do.double().view(B, Sq, hk, G, d).permute(0, 2, 3, 1, 4)
        doh = torch.where(torch.isfinite(doh), doh, torch.zeros((), dtype=doh.dtype))
        oh = p @ vh
        dp, D = doh @ vh.transpose(-1, -2), (doh * oh).sum(-1, keepdim=True)
        slope = 1.0 - u.square() if cap else torch.ones((), dtype=t.dtype)
        ds = p * (dp - D) * slope
        ds_mag = p * (doh.abs() @ vh.abs().transpose(-1, -2) + (doh.abs() * (p @ vh.abs())).sum(-1, keepdim=True)) * slope
        shared = lambda x: x.sum(2, keepdim=True)
        backk = lambda x: x.permute(0, 3, 1, 2, 4).reshape(B, Sk, hk, d)
        out |= {"dq": back(ds @ kh * scale, Sq, h), "dq_mag": back(ds_mag @ kh.abs() * scale, Sq, h),
                "dk": backk(shared(ds.transpose(-1, -2) @ qh) * scale), "dk_mag": backk(shared(ds_mag.transpose(-1, -2) @ qh.abs()) * scale),
                "dv": backk(shared(p.transpose(-1, -2) @ doh)), "dv_mag": backk(shared(p.transpose(-1, -2) @ doh.abs()))}
    return out
