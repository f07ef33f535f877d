"""What surrounds attention in a transformer block, as cases that can be timed: linear layers with bias, activation, gate and residual,
feed-forward blocks made of two of them, and the norm between two branches with the gated residual ahead of it and the modulation
behind it; forward and backward.

A case of kind ``linear`` takes x [B, S, n_in] (with ``heads``: in the order of an attention layer's blocks, [B, heads, S, n_in / heads]) to
residual + gate * act(x W^T + b), ``gated``: act(first half) * second half.  A case of kind ``ffn`` runs two of them, through
``hidden`` channels.  A case of kind ``norm`` takes the stream x and a branch's output y to h = x + gate * post(y) and
norm(h) * weight + bias, times 1 + scale, plus shift.  With ``backward`` a case is the gradients of that, from what the forward pass left.

``own`` = False: the operators written out in torch, in 32 bits; True: this package's kernels.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------------------- cases
def _linear(name, S, n_in, n_out, B=1, dtype="bf16", act="none", gated=False, bias=True, gate_tokens=-1, residual=False, heads=0,
            grid=(0, 0, 0), block=(0, 0, 0), backward=False):
    """gate_tokens: so many consecutive tokens share a row of the gate (0: all of a sample; -1: there is no gate)."""
    return {"name": name, "kind": "linear", "B": B, "S": S, "n_in": n_in, "n_out": n_out, "dtype": dtype, "act": act, "gated": gated,
            "bias": bias, "gate_tokens": gate_tokens, "residual": residual, "heads": heads, "grid": "x".join(map(str, grid)),
            "block": "x".join(map(str, block)), "backward": backward}


def _ffn(name, S, channels, hidden, B=1, dtype="bf16", act="gelu", gated=False, bias=True, gate_tokens=-1, residual=False, backward=False):
    return {"name": name, "kind": "ffn", "B": B, "S": S, "channels": channels, "hidden": hidden, "dtype": dtype, "act": act, "gated": gated,
            "bias": bias, "gate_tokens": gate_tokens, "residual": residual, "backward": backward}


def _norm(name, S, channels, B=1, dtype="bf16", stream="bf16", norm="layer", post="none", mod_tokens=0, modulate=True, affine=False,
          branch=True, gate=True, backward=False):
    return {"name": name, "kind": "norm", "B": B, "S": S, "channels": channels, "dtype": dtype, "stream": stream, "norm": norm, "post": post,
            "mod_tokens": mod_tokens, "modulate": modulate, "affine": affine, "branch": branch, "gate": gate, "backward": backward}


def listed():
    return [
        # the time step's embedding on its way to the six modulations of a block: one row, latency
        _linear("linear_token", 1, 1536, 9216, act="silu"),
        # a fine-tuning test in fp32, two short samples
        _linear("linear_f32_train", 385, 320, 1288, B=2, dtype="f32", act="gelu", backward=True),
        # q, k and v of a layer at 480p
        _linear("linear_qkv_33k", 32760, 1536, 4608),
        # the projection behind the attention layer at 480p: from the order of the 3D layer's blocks, gated, onto the residual stream
        _linear("linear_out_33k_blocks", 32760, 1536, 1536, gate_tokens=0, residual=True, heads=12, grid=(21, 30, 52), block=(3, 6, 13)),
        # its gradients at low resolution
        _linear("linear_out_13k_blocks_bwd", 13440, 1536, 1536, gate_tokens=0, residual=True, heads=12, grid=(21, 20, 32), block=(21, 5, 8),
                backward=True),
        # one frame (1,560 tokens) of a clip that is generated frame by frame
        _ffn("ffn_frame", 1560, 1536, 6144, gate_tokens=0, residual=True),
        # the largest: 480p with 40 heads
        _ffn("ffn_33k_h40", 32760, 5120, 20480, gate_tokens=0, residual=True),
        # training of a gated block at low resolution, an odd width
        _ffn("ffn_gated_13k_bwd", 13440, 1536, 4104, act="silu", gated=True, bias=False, gate_tokens=640, residual=True, backward=True),
        # one token per sample
        _norm("norm_token", 1, 1536, B=4),
        # 720p with 40 heads, the stream in fp32
        _norm("norm_76k_h40_f32", 75600, 5120, stream="f32"),
        # gradients at 480p
        _norm("norm_33k_bwd", 32760, 1536, backward=True),
        # norms before and after the branch, a noise level per frame, odd number of samples
        _norm("norm_sandwich_13k_bwd", 13440, 1536, B=3, norm="rms", post="rms", mod_tokens=640, affine=True, backward=True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _channels(rng, lo, hi):
    return 8 * _spread(rng, max(1, lo // 8), hi // 8)


def _flops(case):
    rows = case["B"] * case["S"]
    per = 3 if case["gated"] else 2
    if case["kind"] == "linear":
        per_row = 2 * case["n_in"] * case["n_out"] * (per - 1)
    else:
        per_row = 2 * case["channels"] * case["hidden"] * per
    return float(rows) * per_row * (2 if case["backward"] else 1)


def draw(rng):
    """Linear layers of 1 to 75,600 tokens, 8 to 20,480 channels in and out, and feed-forward blocks of those; fp32 at sizes of tests;
    norms of 1 to 75,600 tokens of 8 to 8,192 channels.  Every activation, gate, order and direction."""
    while True:
        kind = rng.choice(["linear", "linear", "ffn", "norm", "norm"])
        f32 = rng.random() < 0.2
        B, backward, bias = rng.choice([1, 1, 1, 2, 3]), rng.random() < 0.5, rng.random() < 0.7
        dtype = "f32" if f32 else "bf16"
        S = _spread(rng, 1, 75600)
        frame = rng.choice([0, 0, _spread(rng, 1, S), 1560])
        if kind == "norm":
            case = _norm("", S, _channels(rng, 8, 8192), B=B, dtype=dtype, stream="f32" if f32 else rng.choice(["bf16", "bf16", "f32"]),
                         norm=rng.choice(["layer", "rms"]), post=rng.choice(["none", "none", "rms", "layer"]),
                         mod_tokens=frame if frame == 0 or frame > S // 200 else 0, modulate=rng.random() < 0.8,
                         affine=rng.random() < 0.4, branch=rng.random() < 0.8, gate=rng.random() < 0.8, backward=backward)
            if not case["branch"]:
                case["post"], case["gate"] = "none", False
            if B * S * case["channels"] * (3 if backward else 2) * (2 if f32 else 1) > 75600 * 5120 * 2:
                continue
        elif kind == "ffn":
            case = _ffn("", S, _channels(rng, 8, 5120), _channels(rng, 8, 20480), B=B, dtype=dtype, act=rng.choice(["gelu", "silu"]),
                        gated=rng.random() < 0.5, bias=bias, gate_tokens=rng.choice([-1, frame]), residual=rng.random() < 0.6, backward=backward)
        elif rng.random() < 0.35:
            block = (rng.choice([1, 1, 2, 3]), _spread(rng, 1, 45), _spread(rng, 1, 80))
            n = max(1.0, S / (block[0] * block[1] * block[2]))
            grid = (block[0] * max(1, round(n ** 0.5)), block[1], block[2] * max(1, round(n ** 0.5)))
            S, heads, d = grid[0] * grid[1] * grid[2], _spread(rng, 1, 40), rng.choice([64, 128, 128])
            case = _linear("", S, heads * d, _channels(rng, 64, 5120), B=B, dtype=dtype, bias=bias, gate_tokens=rng.choice([-1, 0, frame]),
                           residual=rng.random() < 0.7, heads=heads, grid=grid, block=block, backward=backward)
            if S > 75600:
                continue
        else:
            case = _linear("", S, _channels(rng, 8, 20480), _channels(rng, 8, 20480), B=B, dtype=dtype, act=rng.choice(["none", "none", "gelu", "silu"]),
                           gated=rng.random() < 0.25, bias=bias, gate_tokens=rng.choice([-1, -1, frame]), residual=rng.random() < 0.4,
                           backward=backward)
        if kind != "norm":
            rows, wide = B * S, case["hidden"] if kind == "ffn" else max(case["n_in"], case["n_out"])
            if case["gate_tokens"] > 0 and -(-S // case["gate_tokens"]) > 200:
                case["gate_tokens"] = 0
            if _flops(case) > (2e11 if f32 else 1.2e13) or rows * wide * (3 if case["gated"] else 1) > 32760 * 20480:
                continue
        del case["name"]
        return case


# ---------------------------------------------------------------------------------------------------------------- inputs
def _three(text):
    return tuple(int(i) for i in text.split("x"))


def _perm(case):
    """int32 [S]: the raster token at each position of block order."""
    T, H, W = _three(case["grid"])
    bT, bH, bW = _three(case["block"])
    at = torch.arange(T * H * W, device="cuda", dtype=torch.int32)
    return at.view(T // bT, bT, H // bH, bH, W // bW, bW).permute(0, 2, 4, 1, 3, 5).reshape(-1).contiguous()


def _groups(case, tokens):
    return 1 if tokens <= 0 else -(-case["S"] // tokens)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, B, S = DT[case["dtype"]], case["B"], case["S"]

    def normal(*shape, dtype=dt, scale=1.0):
        big = math.prod(shape) >= 2 ** 24
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt if big else torch.float32).mul_(scale).to(dtype)

    st = {"case": case}
    if case["kind"] == "norm":
        C, G = case["channels"], _groups(case, case["mod_tokens"])
        spread = torch.exp(0.5 * torch.randn(C, generator=gen, device="cuda")) * 1.5        # some channels of a stream are large
        stream = lambda: normal(B, S, C, dtype=DT[case["stream"]]).mul_(spread).add_(0.3)
        rows = lambda: normal(B, 6, G, C, dtype=torch.float32, scale=0.5)
        six = rows()                   # shift, scale and gate are slices of one tensor, as a model's modulation leaves them
        st |= {"gate": six[:, 2] if case["gate"] else None, "scale": six[:, 1] if case["modulate"] else None,
               "shift": six[:, 0] if case["modulate"] else None, "y": normal(B, S, C) if case["branch"] else None}
        vector = lambda at: at + normal(C, dtype=torch.float32, scale=0.2)
        st |= {"weight": vector(1.0) if case["affine"] else None, "bias": vector(0.0) if case["affine"] and case["norm"] == "layer" else None,
               "post_weight": vector(1.0) if case["affine"] and case["post"] != "none" else None}
        if case["backward"]:
            st |= {"h": stream(), "d_out": normal(B, S, C), "d_h": normal(B, S, C, dtype=DT[case["stream"]])}
        else:
            st["x"] = stream()
    else:
        rows = 2 if case["gated"] else 1
        gated = case["gate_tokens"] >= 0
        weight = lambda n, k: normal(n, k, scale=k ** -0.5)
        if case["kind"] == "linear":
            n_in, n_out = case["n_in"], case["n_out"]
            heads = case["heads"]
            st["x"] = normal(B, heads, S, n_in // heads) if heads else normal(B, S, n_in)
            st["w"] = weight(rows * n_out, n_in)
            st["b"] = normal(rows * n_out, scale=0.2) if case["bias"] else None
            st["perm"] = _perm(case) if heads else None
        else:
            n_out = case["channels"]
            st["x"] = normal(B, S, n_out)
            st["w1"], st["w2"] = weight(rows * case["hidden"], n_out), weight(n_out, case["hidden"])
            st["b1"] = normal(rows * case["hidden"], scale=0.2) if case["bias"] else None
            st["b2"] = normal(n_out, scale=0.2) if case["bias"] else None
        st["gate"] = normal(B, _groups(case, case["gate_tokens"]), n_out, dtype=torch.float32, scale=0.5) if gated else None
        if case["backward"]:
            st["d_out"] = normal(B, S, n_out)
            # what the forward pass left: the products ahead of activation and gate
            if case["kind"] == "ffn":
                st["kept"] = normal(B, S, rows * case["hidden"])
                st["kept2"] = normal(B, S, n_out, scale=0.5) if gated else None
            else:
                st["kept"] = normal(B, S, rows * n_out) if gated or case["act"] != "none" or case["gated"] else None
        else:
            st["residual"] = normal(B, S, n_out) if case["residual"] else None
    if own:        # what a program keeps from call to call: the operators and their outputs
        _prepare_own(case, st)
    return st


def _prepare_own(case, st):
    from paper_2506_23858_b200 import binding as vb
    from paper_2506_23858_b200.layer import BlockNorm, FeedForward, Linear
    B, S = case["B"], case["S"]
    if case["kind"] == "norm":
        shape = vb.make_norm_shape(B, S, case["channels"], case["dtype"], stream_dtype=case["stream"], norm=case["norm"],
                                   post_norm=case["post"], mod_tokens=case["mod_tokens"])
        st["op"] = BlockNorm(shape)
        if case["backward"]:
            st["dx"] = torch.empty_like(st["h"])
            st["dy"] = None if st["y"] is None else torch.empty_like(st["y"])
        else:
            st["h"] = torch.empty_like(st["x"]) if case["branch"] else None
            st["out"] = torch.empty(st["x"].shape, dtype=DT[case["dtype"]], device="cuda")
        return
    gate_tokens = max(0, case["gate_tokens"])
    if case["kind"] == "linear":
        st["op"] = Linear(vb.make_linear_shape(B, S, case["n_in"], case["n_out"], case["dtype"], activation=case["act"], gated=case["gated"],
                                               heads=case["heads"], gate_tokens=gate_tokens))
        n_out = case["n_out"]
    else:
        st["op"] = FeedForward(B, S, case["channels"], case["hidden"], case["dtype"], activation=case["act"], gated=case["gated"],
                               gate_tokens=gate_tokens)
        n_out = case["channels"]
    if case["backward"]:
        st["dx"] = torch.empty_like(st["x"])
    else:
        st["out"] = torch.empty((B, S, n_out), dtype=DT[case["dtype"]], device="cuda")


# ---------------------------------------------------------------------------------------------------------------- plain forms
def _per_token(case, rows, tokens):
    """[B, groups, C] as [B, S, C]."""
    if rows.shape[1] == 1:
        return rows
    return rows.repeat_interleave(tokens, 1)[:, : case["S"]]


def _group_sums(case, x, tokens):
    """[B, S, C] summed over the tokens that share a row."""
    G = _groups(case, tokens)
    if G == 1:
        return x.sum(1, keepdim=True)
    pad = G * tokens - case["S"]
    if pad:
        x = torch.cat([x, x.new_zeros(x.shape[0], pad, x.shape[2])], 1)
    return x.view(x.shape[0], G, tokens, -1).sum(2)


def _act(name, u):
    if name == "gelu":
        return 0.5 * u * (1.0 + torch.tanh(0.7978845608028654 * (u + 0.044715 * u * u * u)))
    return u / (1.0 + torch.exp(-u)) if name == "silu" else u


def _act_slope(name, u):
    if name == "gelu":
        t = torch.tanh(0.7978845608028654 * (u + 0.044715 * u * u * u))
        return 0.5 * (1.0 + t) + 0.5 * u * (1.0 - t * t) * 0.7978845608028654 * (1.0 + 3.0 * 0.044715 * u * u)
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-u))
        return s * (1.0 + u * (1.0 - s))
    return torch.ones_like(u)


def _activated(case, u):
    if case["gated"]:
        a, b = u.chunk(2, -1)
        return _act(case["act"], a) * b
    return _act(case["act"], u)


def _activated_slope(case, u, d):
    if case["gated"]:
        a, b = u.chunk(2, -1)
        return torch.cat([d * b * _act_slope(case["act"], a), d * _act(case["act"], a)], -1)
    return d * _act_slope(case["act"], u)


def _times(x, w, b):
    y = x @ w.float().t()
    return y if b is None else y + b.float()


def _onto(st, y):
    case = st["case"]
    if st["gate"] is not None:
        y = y * _per_token(case, st["gate"], case["gate_tokens"])
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(DT[case["dtype"]])


def _linear_plain(st):
    case = st["case"]
    x = st["x"].float()
    if not case["heads"]:
        return {"out": _onto(st, _activated(case, _times(x, st["w"], st["b"])))}
    y = _times(x.transpose(1, 2).flatten(2), st["w"], st["b"])
    raster = torch.empty_like(y)
    raster[:, st["perm"].long()] = y
    return {"out": _onto(st, raster)}


def _linear_grads(du, x, w, bias, dt):
    """Gradients of x, the weight and the bias from du [B, S, n]."""
    flat = du.flatten(0, 1)
    return (du @ w.float()).to(dt), (flat.t() @ x.flatten(0, 1)).to(dt), flat.sum(0).to(dt) if bias else None


def _linear_backward_plain(st):
    case, dt = st["case"], DT[st["case"]["dtype"]]
    x, d, out = st["x"].float(), st["d_out"].float(), {}
    if case["heads"]:
        x = x.transpose(1, 2).flatten(2)
    kept = None if st["kept"] is None else st["kept"].float()        # (in the order of x)
    order = st["perm"].long() if case["heads"] else None
    if st["gate"] is not None:
        y = _activated(case, kept)
        if order is not None:
            raster = torch.empty_like(y)
            raster[:, order] = y
            y = raster
        out["dgate"] = _group_sums(case, d * y, case["gate_tokens"])
        d = d * _per_token(case, st["gate"], case["gate_tokens"])
    if order is not None:
        d = d[:, order]
    if kept is not None:
        d = _activated_slope(case, kept, d)
    dx, out["dw"], db = _linear_grads(d, x, st["w"], case["bias"], dt)
    if case["heads"]:
        dx = dx.view(case["B"], case["S"], case["heads"], -1).transpose(1, 2).contiguous()
    out["dx"] = dx
    if db is not None:
        out["db"] = db
    return out


def _ffn_plain(st):
    h = _activated(st["case"], _times(st["x"].float(), st["w1"], st["b1"]))
    return {"out": _onto(st, _times(h, st["w2"], st["b2"]))}


def _ffn_backward_plain(st):
    case, dt, out = st["case"], DT[st["case"]["dtype"]], {}
    d, u = st["d_out"].float(), st["kept"].float()
    if st["gate"] is not None:
        out["dgate"] = _group_sums(case, d * st["kept2"].float(), case["gate_tokens"])
        d = d * _per_token(case, st["gate"], case["gate_tokens"])
    out["dw2"] = (d.flatten(0, 1).t() @ _activated(case, u).flatten(0, 1)).to(dt)
    du = _activated_slope(case, u, d @ st["w2"].float())
    out["dx"], out["dw1"], db1 = _linear_grads(du, st["x"].float(), st["w1"], case["bias"], dt)
    if db1 is not None:
        out["db1"], out["db2"] = db1, d.sum((0, 1)).to(dt)
    return out


def _normed(kind, x):
    """x normed over its channels, and one over its size."""
    if kind == "none":
        return x, None
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
    return x * r, r


def _normed_slope(kind, d, n, r):
    """Gradient of x from d, that of its normed values n."""
    if kind == "none":
        return d
    dx = d - n * (d * n).mean(-1, keepdim=True)
    if kind == "layer":
        dx = dx - d.mean(-1, keepdim=True)
    return dx * r


def _norm_plain(st):
    case, out = st["case"], {}
    h = st["x"].float()
    if st["y"] is not None:
        z = _normed(case["post"], st["y"].float())[0]
        if st["post_weight"] is not None:
            z = z * st["post_weight"]
        h = h + (z if st["gate"] is None else z * _per_token(case, st["gate"], case["mod_tokens"]))
        out["h"] = h.to(DT[case["stream"]])
    n = _normed(case["norm"], h)[0]
    if st["weight"] is not None:
        n = n * st["weight"]
    if st["bias"] is not None:
        n = n + st["bias"]
    if st["scale"] is not None:
        n = n * (1.0 + _per_token(case, st["scale"], case["mod_tokens"])) + _per_token(case, st["shift"], case["mod_tokens"])
    out["out"] = n.to(DT[case["dtype"]])
    return out


def _norm_backward_plain(st):
    case, out, tokens = st["case"], {}, st["case"]["mod_tokens"]
    d = st["d_out"].float()
    n, r = _normed(case["norm"], st["h"].float())
    if st["scale"] is not None:
        m = n if st["weight"] is None else n * st["weight"]
        m = m if st["bias"] is None else m + st["bias"]
        out["dscale"], out["dshift"] = _group_sums(case, d * m, tokens), _group_sums(case, d, tokens)
        d = d * (1.0 + _per_token(case, st["scale"], tokens))
    if st["bias"] is not None:
        out["dbias"] = d.sum((0, 1))
    if st["weight"] is not None:
        out["dweight"] = (d * n).sum((0, 1))
        d = d * st["weight"]
    dh = st["d_h"].float() + _normed_slope(case["norm"], d, n, r)
    out["dx"] = dh.to(DT[case["stream"]])
    if st["y"] is None:
        return out
    z, rz = _normed(case["post"], st["y"].float())
    if st["gate"] is not None:
        out["dgate"] = _group_sums(case, dh * (z if st["post_weight"] is None else z * st["post_weight"]), tokens)
        dh = dh * _per_token(case, st["gate"], tokens)
    if st["post_weight"] is not None:
        out["dpost_weight"] = (dh * z).sum((0, 1))
        dh = dh * st["post_weight"]
    out["dy"] = _normed_slope(case["post"], dh, z, rz).to(DT[case["dtype"]])
    return out


# ---------------------------------------------------------------------------------------------------------------- one pass
_PLAIN = {("linear", False): _linear_plain, ("linear", True): _linear_backward_plain, ("ffn", False): _ffn_plain,
          ("ffn", True): _ffn_backward_plain, ("norm", False): _norm_plain, ("norm", True): _norm_backward_plain}


def run(st):
    case = st["case"]
    if not own:
        return _PLAIN[case["kind"], case["backward"]](st)
    op = st["op"]
    if case["kind"] == "norm":
        args = {n: st[n] for n in ("gate", "scale", "shift", "weight", "bias", "post_weight")}
        if not case["backward"]:
            op.forward(st["x"], st["out"], y=st["y"], h_out=st["h"], **args)
            return {n: st[n] for n in ("h", "out") if st[n] is not None}
        got = op.backward(st["d_out"], st["h"], st["dx"], d_h=st["d_h"], y=st["y"], dy_out=st["dy"], **args)
        out = {"dx": st["dx"]} | {n: g for n, g in got.items() if g is not None}
        return out if st["dy"] is None else out | {"dy": st["dy"]}
    if case["kind"] == "linear":
        if not case["backward"]:
            op.forward(st["x"], st["w"], st["out"], bias=st["b"], gate=st["gate"], residual=st["residual"], perm=st["perm"])
            return {"out": st["out"]}
        dw, db, dgate = op.backward(st["d_out"], st["x"], st["w"], st["dx"], kept=st["kept"], gate=st["gate"], perm=st["perm"],
                                    with_bias=case["bias"])
        out = {"dx": st["dx"], "dw": dw, "db": db, "dgate": dgate}
    else:
        if not case["backward"]:
            op.forward(st["x"], st["w1"], st["w2"], st["out"], b_up=st["b1"], b_down=st["b2"], gate=st["gate"], residual=st["residual"])
            return {"out": st["out"]}
        dw1, dw2, db1, db2, dgate = op.backward(st["d_out"], st["x"], st["w1"], st["w2"], (st["kept"], st["kept2"]), st["dx"],
                                                gate=st["gate"], with_bias=case["bias"])
        out = {"dx": st["dx"], "dw1": dw1, "dw2": dw2, "db1": db1, "db2": db2, "dgate": dgate}
    return {n: t for n, t in out.items() if t is not None}


def work(case):
    es, B, S = 2 if case["dtype"] == "bf16" else 4, case["B"], case["S"]
    if case["kind"] == "norm":
        ss, n = 2 if case["stream"] == "bf16" else 4, B * S * case["channels"]
        if case["backward"]:          # d_out, h and d_h in, dx out; the branch in, its gradient out
            per = es + 3 * ss + (2 * es if case["branch"] else 0)
        else:
            per = ss + es + (es + ss if case["branch"] else 0)
        return {"bytes": n * per, "flops": n * (20 if case["backward"] else 12)}
    rows, two = B * S, 2 if case["gated"] else 1
    if case["kind"] == "linear":
        weights, n_in, n_out, wide = two * case["n_in"] * case["n_out"], case["n_in"], case["n_out"], two * case["n_out"]
    else:
        weights, n_in, n_out, wide = (two + 1) * case["channels"] * case["hidden"], case["channels"], case["channels"], two * case["hidden"]
    gated, kept = case["gate_tokens"] >= 0, 0
    if case["backward"]:
        if case["kind"] == "ffn":
            kept = wide + (n_out if gated else 0)
        elif gated or case["gated"] or case["act"] != "none":
            kept = wide
        rows_bytes = 2 * n_in + n_out + kept
    else:
        rows_bytes = n_in + n_out * (2 if case["residual"] else 1)
    return {"bytes": (rows * rows_bytes + weights * (2 if case["backward"] else 1)) * es, "flops": _flops(case)}


# ---------------------------------------------------------------------------------------------------------------- 64 bits
def _act64(name, u):
    if name == "gelu":
        return u * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (u + 0.044715 * u.pow(3)))
    return u * torch.sigmoid(u) if name == "silu" else u


def _through64(case, u):
    if not case["gated"]:
        return _act64(case["act"], u)
    n = u.shape[-1] // 2
    return _act64(case["act"], u[..., :n]) * u[..., n:]


def _token_rows64(case, rows, tokens):
    at = torch.arange(case["S"], device="cuda") // (tokens if tokens > 0 else case["S"])
    return rows.index_select(1, at)


def _linear_exact(case, st):
    x, w = st["x"].double(), st["w"].double()
    B, S, heads = case["B"], case["S"], case["heads"]
    if heads:                          # by raster token
        where = torch.empty(S, dtype=torch.long, device="cuda")
        where[st["perm"].long()] = torch.arange(S, device="cuda")
        x = x.index_select(2, where).permute(0, 2, 1, 3).reshape(B, S, -1)
    if not case["backward"]:
        y = torch.einsum("bsk,nk->bsn", x, w)
        y = _through64(case, y if st["b"] is None else y + st["b"].double())
        if st["gate"] is not None:
            y = y * _token_rows64(case, st["gate"].double(), case["gate_tokens"])
        return {"out": y if st["residual"] is None else st["residual"].double() + y}
    if st["kept"] is None:
        u, leaf = None, None
        d = st["d_out"].double()
    else:
        leaf = st["kept"].double()
        if heads:
            leaf = leaf.index_select(1, where)
        leaf.requires_grad_()
        u = _through64(case, leaf)
        wanted = [leaf]
        if st["gate"] is not None:
            gate = st["gate"].double().requires_grad_()
            u = u * _token_rows64(case, gate, case["gate_tokens"])
            wanted.append(gate)
        d, *dgate = torch.autograd.grad(u, wanted, st["d_out"].double())
    out = {"dx": torch.einsum("bsn,nk->bsk", d, w), "dw": torch.einsum("bsn,bsk->nk", d, x)}
    if heads:
        out["dx"] = out["dx"].view(B, S, heads, -1).permute(0, 2, 1, 3).index_select(2, st["perm"].long())
    if case["bias"]:
        out["db"] = d.sum((0, 1))
    if leaf is not None and dgate:
        out["dgate"] = dgate[0]
    return out


def _ffn_exact(case, st):
    x, w1, w2 = st["x"].double(), st["w1"].double(), st["w2"].double()
    gate = None if st["gate"] is None else st["gate"].double()
    if not case["backward"]:
        u = torch.einsum("bsk,nk->bsn", x, w1)
        y = torch.einsum("bsn,kn->bsk", _through64(case, u if st["b1"] is None else u.add_(st["b1"].double())), w2)
        y = y if st["b2"] is None else y + st["b2"].double()
        y = y if gate is None else y * _token_rows64(case, gate, case["gate_tokens"])
        return {"out": y if st["residual"] is None else st["residual"].double() + y}
    d, out = st["d_out"].double(), {}
    if gate is not None:
        gate.requires_grad_()
        out["dgate"], = torch.autograd.grad(_token_rows64(case, gate, case["gate_tokens"]), gate, d * st["kept2"].double())
        d = d * _token_rows64(case, gate.detach(), case["gate_tokens"])
    u = st["kept"].double().requires_grad_()
    h = _through64(case, u)
    du, = torch.autograd.grad(h, u, torch.einsum("bsk,kn->bsn", d, w2))
    out |= {"dw2": torch.einsum("bsk,bsn->kn", d, h.detach()), "dw1": torch.einsum("bsn,bsk->nk", du, x), "dx": torch.einsum("bsn,nk->bsk", du, w1)}
    if case["bias"]:
        out |= {"db1": du.sum((0, 1)), "db2": d.sum((0, 1))}
    return out


def _norm64(kind, x):
    if kind == "none":
        return x
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True) if kind == "layer" else (x.pow(2).mean(-1, keepdim=True), 0.0)
    return (x - mean) / (var + 1e-6).sqrt()


def _norm_exact(case, st):
    tokens, leaves = case["mod_tokens"], {}
    for name in ("gate", "scale", "shift", "weight", "bias", "post_weight", "y"):
        leaves[name] = None if st[name] is None else st[name].double().requires_grad_(case["backward"])

    def rows(name):
        return _token_rows64(case, leaves[name], tokens)

    def added(y):
        z = _norm64(case["post"], y)
        z = z if leaves["post_weight"] is None else z * leaves["post_weight"]
        return z if leaves["gate"] is None else z * rows("gate")

    def outer(h):
        n = _norm64(case["norm"], h)
        n = n if leaves["weight"] is None else n * leaves["weight"]
        n = n if leaves["bias"] is None else n + leaves["bias"]
        return n if leaves["scale"] is None else n + n * rows("scale") + rows("shift")

    if not case["backward"]:
        h = st["x"].double()
        if leaves["y"] is None:
            return {"out": outer(h)}
        h = h + added(leaves["y"])
        return {"h": h, "out": outer(h)}
    h = st["h"].double().requires_grad_()
    names = [n for n in ("scale", "shift", "weight", "bias") if leaves[n] is not None]
    dh, *got = torch.autograd.grad(outer(h), [h] + [leaves[n] for n in names], st["d_out"].double())
    out = {"d" + n: g for n, g in zip(names, got)}
    dh = dh + st["d_h"].double()
    out["dx"] = dh
    if leaves["y"] is not None:
        names = [n for n in ("y", "gate", "post_weight") if leaves[n] is not None]
        got = torch.autograd.grad(added(leaves["y"]), [leaves[n] for n in names], dh)
        out |= {"d" + n: g for n, g in zip(names, got)}
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"linear": _linear_exact, "ffn": _ffn_exact, "norm": _norm_exact}[case["kind"]](case, st)
