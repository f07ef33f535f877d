"""What stands around the attention layer in a model, as cases that can be timed: rotary positions with the norm of q and k ahead
of them, and attention in which every query sees one run of keys and scores may be capped; forward and backward.

A case of kind ``rotary`` takes q and k of one layer, raster order [B, S, heads, head_dim] on a grid (T, H, W): root-mean-square norm
(none, per head, or over the whole token row), rotation of the first ``2 * pairs`` channels of a head, result in raster order or in the
order of the layer's blocks; with ``backward`` the gradients of that (dq, dk and the weights').  A case of kind ``attn`` takes q
[B, Sq, heads, d] and k, v [B, Sk, kv_heads, d]: forward, or with ``backward`` forward and gradients.

``own`` = False: the operators written out in torch, in 32 bits (angles in 64); True: this package's kernels.
"""
import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------- cases
def _rotary(name, grid, block, B=1, heads=12, head_dim=128, dtype="bf16", layout="interleaved", pairs=(22, 21, 21), norm="row",
            scaling="none", factor=1.0, first=0, order="block", backward=False):
    return {"name": name, "kind": "rotary", "T": grid[0], "H": grid[1], "W": grid[2], "bT": block[0], "bH": block[1], "bW": block[2],
            "B": B, "heads": heads, "head_dim": head_dim, "dtype": dtype, "layout": layout, "pairs": ",".join(map(str, pairs)),
            "norm": norm, "scaling": scaling, "factor": factor, "first": first, "order": order, "backward": backward}


def _attn(name, Sq, Sk, lens, B=1, heads=12, kv_heads=12, head_dim=128, dtype="bf16", cap=0.0, frame=0, prefix=0, window=0,
          packed=True, backward=False):
    """lens: packed, the lengths of the clips that share a sequence (what is left over is padding); else the filled length of each
    sample's cache, of which the queries are the last.  frame: a query sees up to the end of its own group of that many tokens (1:
    itself; 0: the whole clip); prefix: tokens at a clip's start that all of it sees; window: at most that many keys."""
    return {"name": name, "kind": "attn", "Sq": Sq, "Sk": Sk, "lens": ",".join(map(str, lens)), "B": B, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "cap": cap, "frame": frame, "prefix": prefix,
            "window": window, "packed": packed, "backward": backward}


def listed():
    return [
        # one new token of a sequence that is generated piece by piece: latency
        _rotary("rotary_token", (1, 1, 1), (1, 1, 1), first=32760, order="raster"),
        # a fine-tuning test in fp32: odd grid, small heads of which a part turns, positions far out, frequencies scaled by parts
        _rotary("rotary_f32_partial", (5, 7, 11), (1, 7, 11), B=2, heads=5, head_dim=64, dtype="f32", layout="half", pairs=(12,),
                norm="none", scaling="parts", factor=8.0, first=1000000, order="raster"),
        # q and k of a layer at 480p, into the order of the 3D layer's blocks
        _rotary("rotary_33k_blocks", (21, 30, 52), (3, 6, 13)),
        # the largest: 720p with 40 heads
        _rotary("rotary_76k_h40_blocks", (21, 45, 80), (1, 45, 80), heads=40),
        # the gradients of the same step at 480p
        _rotary("rotary_bwd_33k", (21, 30, 52), (3, 6, 13), order="raster", backward=True),
        # low resolution, norm per head, half layout, base of the frequencies raised
        _rotary("rotary_bwd_13k_head", (21, 20, 32), (21, 5, 8), layout="half", norm="head", scaling="base", factor=4.0,
                order="raster", backward=True),
        # one token per sample against caches of up to a 720p clip, three query heads to a key head
        _attn("attn_token_cache", 1, 75600, (75600, 60123, 33333, 7801), B=4, kv_heads=4, packed=False),
        # the next frame of a clip at 480p (1,560 tokens) against the frames before it and itself
        _attn("attn_frame_cache", 1560, 32760, (31200,), packed=False),
        # a training test in fp32: clips of 1 to 90 tokens and padding in one sequence, capped scores
        _attn("attn_clips_f32_train", 256, 256, (64, 1, 37, 90), B=2, heads=2, kv_heads=1, head_dim=64, dtype="f32", cap=20.0,
              backward=True),
        # low-resolution clips of different lengths packed into one training sequence, padding behind the last
        _attn("attn_clips_13k_train", 13440, 13440, (4480, 640, 2561, 77, 1920, 1, 3200, 500), backward=True),
        # a clip at 480p whose frames see the frames before them and the first frame, capped scores: forward
        _attn("attn_frames_33k_cap", 32760, 32760, (32760,), cap=50.0, frame=1560, prefix=1560),
        # training of the same kind at low resolution, key heads shared by three
        _attn("attn_frames_13k_cap_train", 13440, 13440, (6720, 6720), kv_heads=4, cap=30.0, frame=640, prefix=640, backward=True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng):
    while True:
        backward = rng.random() < 0.5
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        d = rng.choice([64, 128, 128])
        block = (rng.choice([1, 1, 2, 3]), _spread(rng, 1, 45), _spread(rng, 1, 80))
        target = _spread(rng, 1, 75600)
        n = max(1.0, target / (block[0] * block[1] * block[2]))
        count = (max(1, round(n ** 0.5)), 1, max(1, round(n ** 0.5)))
        grid = tuple(b * c for b, c in zip(block, count))
        turned = rng.choice([d // 2, d // 2, d // 4, rng.randint(1, d // 2)])
        pairs = (turned,) if turned < 3 or rng.random() < 0.3 else (turned - 2 * (turned // 3), turned // 3, turned // 3)
        scaling = rng.choice(["none", "linear", "base", "parts"])
        case = _rotary("", grid, block, B=rng.choice([1, 1, 2, 3]), heads=_spread(rng, 1, 40), head_dim=d, dtype=dtype,
                       layout=rng.choice(["half", "interleaved"]), pairs=pairs, norm=rng.choice(["none", "head", "row", "row"]),
                       scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                       first=rng.choice([0, 0, _spread(rng, 1, 10 ** 7)]), order="raster" if backward else rng.choice(["raster", "block"]),
                       backward=backward)
        tokens = grid[0] * grid[1] * grid[2]
        if tokens <= 75600 and case["B"] * tokens * case["heads"] * d * (2 if dtype == "f32" else 1) * (1.5 if backward else 1) <= 75600 * 40 * 128:
            return case


def _draw_attn(rng):
    while True:
        f32 = rng.random() < 0.25
        d = rng.choice([64, 128]) if f32 or rng.random() < 0.15 else 128
        kv = _spread(rng, 1, 16)
        heads = kv * rng.choice([1, 1, 2, 3, 4])
        B = rng.choice([1, 1, 2, 3])
        cap = rng.choice([0.0, 0.0, 20.0, 50.0])
        if rng.random() < 0.4:
            Sk = _spread(rng, 1, 4000 if f32 else 75600)
            Sq = min(Sk, rng.choice([1, 1, _spread(rng, 2, 2000)]))
            lens = [rng.randint(Sq, Sk) for _ in range(B)]
            case = _attn("", Sq, Sk, lens, B=B, heads=heads, kv_heads=kv, head_dim=d, dtype="f32" if f32 else "bf16", cap=cap,
                         frame=rng.choice([0, 1, 1, 1560]), window=rng.choice([0, 0, _spread(rng, 1, Sk)]), packed=False)
        else:
            S = _spread(rng, 1, 2000 if f32 or d == 64 else 24000)
            lens, left = [], S
            for _ in range(rng.choice([1, 2, 5, 9])):
                n = min(left, _spread(rng, 1, S))
                lens += [n] if n else []
                left -= n
            frame = rng.choice([0, 0, 1, _spread(rng, 1, S)])
            case = _attn("", S, S, lens, B=B, heads=heads, kv_heads=kv, head_dim=d, dtype="f32" if f32 else "bf16", cap=cap,
                         frame=frame, prefix=rng.choice([0, _spread(rng, 1, S)]) if frame else 0,
                         window=rng.choice([0, 0, 0, _spread(rng, 1, S)]), backward=rng.random() < 0.6)
        dense = B * heads * case["Sq"] * case["Sk"] * (3.5 if case["backward"] else 1.0)
        kv_bytes = B * kv * case["Sk"] * d * 2 * (2 if f32 else 1)
        if dense <= (3e8 if f32 or d == 64 else 7.5e9) and kv_bytes <= 4 * 4 * 75600 * 128 * 2:
            return case


def draw(rng):
    """Rotary: 1 to 75,600 tokens on any grid, 1 to 40 heads of 64 or 128, any share of a head turned, each norm, layout, scaling and
    direction.  Attention: sequences of 1 to 24,000 tokens of any number of clips with padding, caches of up to 75,600 keys with one query or many,
    shared key heads, capped scores, windows."""
    case = _draw_rotary(rng) if rng.random() < 0.45 else _draw_attn(rng)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------- inputs
def _frequencies(case):
    """(fp64 frequency and axis of each pair, factor on the sines and cosines), as a model's configuration gives them."""
    per_axis = [int(n) for n in case["pairs"].split(",")]
    theta, factor, scaling, trained = 10000.0, case["factor"], case["scaling"], 4096
    freq, axis, m = [], [], 1.0
    for a, n in enumerate(per_axis):
        base = theta * factor ** (n / max(1, n - 1)) if scaling == "base" else theta
        f = base ** (-np.arange(n, dtype=np.float64) / n)
        if scaling == "linear":
            f = f / factor
        elif scaling == "parts":       # slow pairs interpolated, fast ones kept, a ramp over 1 to 32 turns of the trained length
            keep = np.clip((trained * f / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
            f = f * keep + f / factor * (1.0 - keep)
        freq.append(f)
        axis.append(np.full(n, a, dtype=np.int32))
    if scaling == "parts":
        m = 0.1 * math.log(factor) + 1.0
    return np.concatenate(freq), np.concatenate(axis), m


def _positions(case):
    """int32 [S, axes]: frame (from the clip's place in the sequence on), row and column; one axis: the token's number."""
    T, H, W = case["T"], case["H"], case["W"]
    if "," not in case["pairs"]:
        return (case["first"] + torch.arange(T * H * W, device="cuda")).to(torch.int32)[:, None]
    t, h, w = (torch.arange(n, device="cuda", dtype=torch.int32) for n in (T, H, W))
    grid = torch.meshgrid(t + case["first"], h, w, indexing="ij")
    return torch.stack([x.reshape(-1) for x in grid], dim=1).contiguous()


def _ranges(case):
    """int32 [1 or B, Sq, 2]: the keys [lo, hi) that each query sees."""
    lens = torch.tensor([int(n) for n in case["lens"].split(",")], device="cuda")
    Sq, frame = case["Sq"], case["frame"]
    if case["packed"]:
        ends = lens.cumsum(0)
        at = torch.arange(Sq, device="cuda")[None]
        clip = torch.searchsorted(ends, at, right=True)
        some = clip < len(lens)
        clip = clip.clamp(max=len(lens) - 1)
        lo, hi = (ends - lens)[clip], ends[clip]
    else:
        at = (lens - Sq)[:, None] + torch.arange(Sq, device="cuda")[None]
        lo, hi = torch.zeros_like(at), lens[:, None].expand_as(at)
        some = at >= 0
    if frame:
        seen = torch.maximum(((at - lo) // frame + 1) * frame, torch.full_like(at, case["prefix"]))
        hi = torch.minimum(hi, lo + seen)
    if case["window"]:
        lo = torch.maximum(lo, hi - case["window"])
    return torch.stack([torch.where(some, lo, 0), torch.where(some, hi, 0)], dim=-1).to(torch.int32).contiguous()


def _shape(case):
    from paper_2506_23858_b200 import binding as vb
    return vb.make_shape(case["B"], case["heads"], case["head_dim"], (case["T"], case["H"], case["W"]),
                         (case["bT"], case["bH"], case["bW"]), case["dtype"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, d, B = DT[case["dtype"]], case["head_dim"], case["B"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32 if math.prod(shape) < 2 ** 24 else dt).to(dt)

    if case["kind"] == "rotary":
        S, heads = case["T"] * case["H"] * case["W"], case["heads"]
        freq, axis, m = _frequencies(case)
        st = {"case": case, "q": normal(B, S, heads, d), "k": normal(B, S, heads, d), "pos": _positions(case),
              "freq": torch.from_numpy(freq).cuda(), "axis": torch.from_numpy(axis).cuda(), "m": m, "wq": None, "wk": None}
        if case["norm"] != "none":
            n = d if case["norm"] == "head" else heads * d
            st["wq"], st["wk"] = (1.0 + 0.2 * torch.randn(n, generator=gen, device="cuda") for _ in range(2))
        if case["backward"]:
            st["dq"], st["dk"] = normal(B, S, heads, d), normal(B, S, heads, d)
    else:
        st = {"case": case, "ranges": _ranges(case), "q": normal(B, case["Sq"], case["heads"], d),
              "k": normal(B, case["Sk"], case["kv_heads"], d), "v": normal(B, case["Sk"], case["kv_heads"], d)}
        if case["cap"]:
            st["q"].mul_(4.0)          # logits that reach the cap
        if case["backward"]:
            st["do"] = normal(B, case["Sq"], case["heads"], d)
    if own:        # what a program keeps from call to call: outputs, tables, the plan of the key ranges, workspaces
        if case["kind"] == "rotary":
            from paper_2506_23858_b200.layer import Rotary
            st["op"] = Rotary(_shape(case), st["pos"], st["freq"], st["axis"], layout=case["layout"], norm=case["norm"], mscale=m,
                              with_backward=case["backward"])
            out = (B, heads, S, d) if case["order"] == "block" else (B, S, heads, d)
            st["out"] = [torch.empty(out, dtype=dt, device="cuda") for _ in range(2)]
        else:
            from paper_2506_23858_b200 import binding as vb
            from paper_2506_23858_b200.layer import RangeAttention
            shape = vb.make_range_shape(B, case["heads"], case["kv_heads"], d, case["Sq"], case["Sk"], case["dtype"],
                                        mask_batch=st["ranges"].shape[0], softcap=case["cap"])
            st["op"] = RangeAttention(shape, st["ranges"], with_backward=case["backward"])
            st["o"] = torch.empty_like(st["q"])
            if case["backward"]:
                st["grads"] = [torch.empty_like(st[n]) for n in ("q", "k", "v")]
    return st


# ---------------------------------------------------------------------------------------------------------------- plain forms
def _angles(st):
    a = st["pos"].double()[:, st["axis"].long()] * st["freq"]
    return (a.cos() * st["m"]).float()[:, None], (a.sin() * st["m"]).float()[:, None]


def _halves(case, x):
    n = sum(int(i) for i in case["pairs"].split(","))
    if case["layout"] == "half":
        return x[..., :n], x[..., n: 2 * n], x[..., 2 * n:]
    return x[..., 0: 2 * n: 2], x[..., 1: 2 * n: 2], x[..., 2 * n:]


def _turned(case, x, cos, sin):
    x0, x1, rest = _halves(case, x)
    y0, y1 = x0 * cos - x1 * sin, x1 * cos + x0 * sin
    y = torch.cat([y0, y1], -1) if case["layout"] == "half" else torch.stack([y0, y1], -1).flatten(-2)
    return torch.cat([y, rest], -1)


def _rows(case, x):
    return x.flatten(2) if case["norm"] == "row" else x


def _rotary_plain(st):
    case = st["case"]
    cos, sin = _angles(st)
    out = {}
    for n in ("q", "k"):
        x, w = st[n].float(), st["w" + n]
        if w is not None:
            rows = _rows(case, x)
            x = (rows * torch.rsqrt(rows.square().mean(-1, keepdim=True) + 1e-6) * w).view(x.shape)
        y = _turned(case, x, cos, sin)
        if case["order"] == "block":
            T, H, W, bT, bH, bW = (case[i] for i in ("T", "H", "W", "bT", "bH", "bW"))
            y = y.view(case["B"], T // bT, bT, H // bH, bH, W // bW, bW, case["heads"], -1).permute(0, 7, 1, 3, 5, 2, 4, 6, 8)
            y = y.reshape(case["B"], case["heads"], T * H * W, -1)
        out[n] = y.to(st[n].dtype)
    return out


def _rotary_backward_plain(st):
    case = st["case"]
    cos, sin = _angles(st)
    out = {}
    for n in ("q", "k"):
        g, w = _turned(case, st["d" + n].float(), cos, -sin), st["w" + n]
        if w is not None:
            x, g = _rows(case, st[n].float()), _rows(case, g)
            r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
            out["dw" + n] = (g * x * r).flatten(0, -2).sum(0)
            g = g * w
            g = (r * (g - x * r.square() * (g * x).mean(-1, keepdim=True))).view(st[n].shape)
        out["d" + n] = g.to(st[n].dtype)
    return out


def _by_key_head(case, x):
    """[B, S, heads, d] as [B * kv_heads, heads / kv_heads * S, d] in 32 bits."""
    B, S, h, d = x.shape
    kv = case["kv_heads"]
    return x.float().view(B, S, kv, h // kv, d).permute(0, 2, 3, 1, 4).reshape(B * kv, h // kv * S, d)


def _from_key_head(case, x, S):
    """The way back."""
    kv = case["kv_heads"]
    n = x.shape[1] // S
    return x.view(case["B"], kv, n, S, -1).permute(0, 3, 1, 2, 4).reshape(case["B"], S, kv * n, -1)


def _attn_plain(st):
    case = st["case"]
    B, Sq, Sk, kv, cap, scale = case["B"], case["Sq"], case["Sk"], case["kv_heads"], case["cap"], case["head_dim"] ** -0.5
    group = case["heads"] // kv
    q, k, v = (_by_key_head(case, st[n]) for n in ("q", "k", "v"))
    do = _by_key_head(case, st["do"]) if case["backward"] else None
    key = torch.arange(Sk, device="cuda")
    r = st["ranges"].expand(B, Sq, 2)
    seen = (key >= r[..., :1]) & (key < r[..., 1:])
    o, dq, dk, dv = (torch.empty_like(x) for x in (q, q, k, v))
    lse = torch.empty(q.shape[:2], device="cuda")
    step = max(1, 2 ** 31 // (group * Sq * Sk))            # heads at a time, for memory
    for i in range(0, B * kv, step):
        part = slice(i, min(i + step, B * kv))
        sample = torch.arange(part.start, part.stop, device="cuda") // kv
        mask = seen[sample].repeat(1, group, 1)
        t = q[part] @ k[part].transpose(1, 2) * scale
        if cap:
            t = cap * torch.tanh(t / cap)
        top = t.masked_fill(~mask, -math.inf).amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp((t - top).masked_fill(~mask, -math.inf))
        total = p.sum(-1, keepdim=True)
        lse[part] = (top + torch.log(total)).squeeze(-1)
        p = p / total.clamp(min=1e-38)
        o[part] = p @ v[part]
        if case["backward"]:
            dv[part] = p.transpose(1, 2) @ do[part]
            ds = p * (do[part] @ v[part].transpose(1, 2) - (do[part] * o[part]).sum(-1, keepdim=True))
            if cap:
                ds = ds * (1.0 - (t / cap).square())
            dq[part] = ds @ k[part] * scale
            dk[part] = ds.transpose(1, 2) @ q[part] * scale
    dt = st["q"].dtype
    out = {"o": _from_key_head(case, o, Sq).to(dt), "lse": lse.view(B, case["heads"], Sq)}
    if case["backward"]:
        out |= {"dq": _from_key_head(case, dq, Sq).to(dt), "dk": _from_key_head(case, dk, Sk).to(dt),
                "dv": _from_key_head(case, dv, Sk).to(dt)}
    return out


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    if case["kind"] == "rotary":
        if not own:
            return _rotary_backward_plain(st) if case["backward"] else _rotary_plain(st)
        weights = None if st["wq"] is None else (st["wq"], st["wk"])
        if not case["backward"]:
            st["op"].forward((st["q"], st["k"]), st["out"], weights, block_order=case["order"] == "block")
            return dict(zip(("q", "k"), st["out"]))
        dw = st["op"].backward((st["dq"], st["dk"]), (st["q"], st["k"]), st["out"], weights)
        out = dict(zip(("dq", "dk"), st["out"]))
        return out if dw is None else out | {"dwq": dw[0], "dwk": dw[1]}
    if not own:
        return _attn_plain(st)
    st["op"].forward(st["q"], st["k"], st["v"], st["o"])
    out = {"o": st["o"], "lse": st["op"].lse}
    if case["backward"]:
        st["op"].backward(st["do"], *st["grads"])
        out |= dict(zip(("dq", "dk", "dv"), st["grads"]))
    return out


def work(case):
    es, d, B = 2 if case["dtype"] == "bf16" else 4, case["head_dim"], case["B"]
    if case["kind"] == "rotary":
        n = B * case["T"] * case["H"] * case["W"] * case["heads"] * d
        tensors = (2 if not case["backward"] else 3 if case["norm"] != "none" else 2)
        return {"bytes": 2 * tensors * n * es, "flops": 2 * n * (12 if case["norm"] != "none" else 4)}
    r = _ranges_on_host(case)
    pairs = float(np.maximum(r[..., 1] - r[..., 0], 0).sum()) * (B if r.shape[0] == 1 else 1) * case["heads"]
    rows, keys = B * case["Sq"] * case["heads"] * d, float((r[..., 1].max(1) - r[..., 0].min(1)).sum())
    keys *= (B if r.shape[0] == 1 else 1) * case["kv_heads"] * d
    tensors = 2 * rows + 2 * keys if not case["backward"] else 4 * rows + 4 * keys
    return {"bytes": tensors * es + 4 * B * case["Sq"] * case["heads"], "flops": (14 if case["backward"] else 4) * d * pairs}


def _ranges_on_host(case):
    return _ranges(case).cpu().numpy().astype(np.int64)


# ---------------------------------------------------------------------------------------------------------------- 64 bits
def _rotation_exact(case, st):
    """Every pair as a complex number of unit length times the factor."""
    angle = torch.empty((st["pos"].shape[0], st["freq"].shape[0]), dtype=torch.float64, device="cuda")
    for a in range(st["pos"].shape[1]):
        mine = (st["axis"] == a).nonzero()[:, 0]
        angle[:, mine] = torch.outer(st["pos"][:, a].double(), st["freq"][mine])
    return torch.polar(torch.full_like(angle, st["m"]), angle)[None, :, None]


def _rotary_exact(case, st):
    unit, n = _rotation_exact(case, st), st["freq"].shape[0]
    out = {}
    for name in ("q", "k"):
        x = st[name].double().requires_grad_()
        w = None if st["w" + name] is None else st["w" + name].double().requires_grad_()
        y = x
        if w is not None:
            over = (2, 3) if case["norm"] == "row" else (3,)
            weight = w.view(case["heads"], -1) if case["norm"] == "row" else w
            y = y / (y.pow(2).mean(over, keepdim=True) + 1e-6).sqrt() * weight
        head = y[..., : 2 * n]
        pairs = head.unflatten(-1, (2, n)).transpose(-1, -2) if case["layout"] == "half" else head.unflatten(-1, (n, 2))
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
        turned = (turned.transpose(-1, -2) if case["layout"] == "half" else turned).flatten(-2)
        y = torch.cat([turned, y[..., 2 * n:]], -1)
        if case["backward"]:
            got = torch.autograd.grad(y, [x] if w is None else [x, w], st["d" + name].double())
            out["d" + name] = got[0]
            if w is not None:
                out["dw" + name] = got[1]
            continue
        y = y.detach().transpose(1, 2)
        if case["order"] == "block":
            t, h, w_ = (torch.arange(case[i], device="cuda") for i in "THW")
            place = torch.cartesian_prod(t, h, w_).view(-1, 3)
            block = torch.tensor([case["bT"], case["bH"], case["bW"]], device="cuda")
            j, s = place // block, place % block
            nH, nW = case["H"] // case["bH"], case["W"] // case["bW"]
            slot = ((j[:, 0] * nH + j[:, 1]) * nW + j[:, 2]) * block.prod() + (s[:, 0] * case["bH"] + s[:, 1]) * case["bW"] + s[:, 2]
            out[name] = torch.empty_like(y)
            out[name][:, :, slot] = y
        else:
            out[name] = y.transpose(1, 2).contiguous()
    return out


def _attn_exact(case, st):
    B, Sq, Sk, cap = case["B"], case["Sq"], case["Sk"], case["cap"]
    group = case["heads"] // case["kv_heads"]
    out = {"o": torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"),
           "lse": torch.empty((B, case["heads"], Sq), dtype=torch.float64, device="cuda")}
    if case["backward"]:
        out |= {"d" + n: torch.zeros(st[n].shape, dtype=torch.float64, device="cuda") for n in "qkv"}
    key = torch.arange(Sk, device="cuda")
    for b in range(B):
        r = st["ranges"][b % st["ranges"].shape[0]]
        hidden = (key < r[:, :1]) | (key >= r[:, 1:])
        some = (~hidden).any(1)
        for h in range(case["heads"]):
            q, k, v = (st[n][b, :, i].double().requires_grad_(case["backward"]) for n, i in (("q", h), ("k", h // group), ("v", h // group)))
            s = q @ k.T / math.sqrt(case["head_dim"])
            if cap:
                s = torch.tanh(s / cap) * cap
            s = s.masked_fill(hidden, -math.inf)
            out["lse"][b, h] = torch.logsumexp(s.detach(), 1)
            w = torch.softmax(torch.where(some[:, None], s, 0.0), 1) * some[:, None]
            o = w @ v
            out["o"][b, :, h] = o.detach()
            if case["backward"]:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), st["do"][b, :, h].double())
                out["dq"][b, :, h] += dq
                out["dk"][b, :, h // group] += dk
                out["dv"][b, :, h // group] += dv
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _rotary_exact(case, st) if case["kind"] == "rotary" else _attn_exact(case, st)
