"""Buffer management and stage sequencing for one VMoBA attention layer on one GPU.

Everything numerical happens inside the C-ABI library; this module only allocates torch
tensors (device memory), passes their pointers to the entry points in order, and exposes the
intermediate buffers so that tests can compare each stage with the oracle.
"""
from __future__ import annotations

import contextlib
import math

import torch

from . import binding as vb


def torch_dtype(shape):
    return torch.bfloat16 if shape.dtype == vb.BF16 else torch.float32


_HERE = contextlib.nullcontext()


def _on(device):
    """The context in which `device` is the current one (nothing to do where it is)."""
    return _HERE if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


def _strides_bsh(x):
    """Element strides (batch, token, head) of a [B, S, heads, d] tensor, as the kernels need them: those of dimensions of size
    one, which address nothing, are taken for dense ones (torch leaves them at any value)."""
    n, st = x.shape, list(x.stride()[:3])
    for i, dense in ((2, n[3]), (1, n[2] * n[3]), (0, n[1] * n[2] * n[3])):
        if n[i] == 1:
            st[i] = dense
    return tuple(st)


def default_capacity(shape, tau: float, slack: float = 0.02) -> int:
    """Upper bound on the number of selected pairs: the threshold rule keeps at most ceil(tau*P)
    pairs per head (the kept fraction never exceeds tau, Section 4.1), plus exact ties."""
    P = shape.S * shape.n_blocks
    per_head = int(min(P, tau * P * (1.0 + slack) + 1024))
    return min(per_head * shape.B * shape.heads, 2 ** 31 - 1)


def rotary_frequencies(pairs_per_axis, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained: int = 4096):
    """What Rotary takes, as host tensors: fp64 frequency and int32 axis of every pair, and the factor on sines and cosines.

    Axis a has pairs_per_axis[a] pairs; its pair i turns by theta^(-i / pairs) per position.  scaling, for contexts `factor`
    times as long as the model was trained on: "linear" (positions interpolated), "base" (theta raised so that the slowest pair is
    interpolated and the fastest kept), "parts" (pairs that make one turn or less over `trained` positions are interpolated,
    those of 32 and more kept, a ramp in between; sines and cosines times 0.1 ln(factor) + 1)."""
    if scaling not in ("none", "linear", "base", "parts"):
        raise ValueError(f"rotary_frequencies: unknown scaling {scaling!r}")
    if not factor >= 1.0 or not theta > 0.0 or any(n < 0 for n in pairs_per_axis):
        raise ValueError("rotary_frequencies: factor >= 1, theta > 0 and no negative number of pairs required")
    freq, axis = [], []
    for a, n in enumerate(pairs_per_axis):
        i = torch.arange(n, dtype=torch.float64)
        base = theta * factor ** (n / max(1, n - 1)) if scaling == "base" else theta
        f = base ** (-i / max(n, 1))
        if scaling == "linear":
            f = f / factor
        elif scaling == "parts":
            keep = ((trained * f / (2.0 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
            f = f * keep + f / factor * (1.0 - keep)
        freq.append(f)
        axis.append(torch.full((n,), a, dtype=torch.int32))
    return torch.cat(freq), torch.cat(axis), 0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0


class Rotary:
    """Norm and rotary positions of q and k of layers of one shape, in whatever blocks: holds the tables, which nothing writes, so that
    any number of layers, streams and captured graphs can use one at the same time.

    positions: int32 [S, axes], or [B, S, axes] where samples differ (clips packed into one sequence restart theirs); freq fp64 and
    axis int32 [pairs] on the device (rotary_frequencies); layout "interleaved" or "half"; norm "none", "head" or "row".  with_backward is taken as
    by the other classes; nothing is held for it, since a backward's scratch is the call's own."""

    def __init__(self, shape, positions, freq, axis, layout="interleaved", norm="none", mscale=1.0, eps=1e-6, with_backward=False):
        s = shape
        if positions.dim() not in (2, 3) or positions.shape[-2] != s.S or (positions.dim() == 3 and positions.shape[0] not in (1, s.B)):
            raise ValueError("Rotary: positions are [S, axes] or [B, S, axes]")
        if positions.dtype != torch.int32 or freq.dtype != torch.float64 or axis.dtype != torch.int32 or freq.shape != axis.shape or freq.dim() != 1:
            raise ValueError("Rotary: int32 positions, fp64 frequencies and as many int32 axes required")
        if not (positions.is_cuda and positions.device == freq.device == axis.device):
            raise ValueError("Rotary: positions, frequencies and axes have to be on one GPU")
        self.shape, self.device, self.dtype = s, positions.device, torch_dtype(s)
        self._size = torch.Size((s.B, s.S, s.heads, s.head_dim))
        self._dense = (s.S * s.heads * s.head_dim, s.heads * s.head_dim, s.head_dim)
        self.positions, self.freq, self.axis = positions.contiguous(), freq.contiguous(), axis.contiguous()
        self.spec = vb.RotarySpec(freq.numel(), positions.shape[-1], {"half": vb.ROTARY_HALF, "interleaved": vb.ROTARY_INTERLEAVED}[layout],
                                  {"none": vb.ROTARY_NORM_NONE, "head": vb.ROTARY_NORM_HEAD, "row": vb.ROTARY_NORM_ROW}[norm],
                                  s.B if positions.dim() == 3 and positions.shape[0] == s.B else 1, mscale, eps)
        self.n_weights = {"none": 0, "head": s.head_dim, "row": s.heads * s.head_dim}[norm]
        if vb.rotary_workspace_bytes(s, self.spec, 1) == 0:
            raise ValueError("Rotary: shape, pairs (up to head_dim / 2), axes (1 to 4), mscale (> 0) or eps (>= 0) out of range")
        # bytes of a backward's scratch by the number of tensors
        self._scratch = {n: vb.rotary_workspace_bytes(s, self.spec, n) for n in range(1, 5)} if self.n_weights else {}

    def _raster(self, x, what):
        if x.shape == self._size and x.dtype is self.dtype and x.device == self.device:
            if x.is_contiguous():          # (a size of one may have any stride)
                return self._dense
            if x.stride(3) == 1:
                return _strides_bsh(x)
        raise ValueError(f"Rotary: {what} has to be [B, S, heads, head_dim] of the layer's type on {self.device}, head_dim contiguous")

    def _block_major(self, x, what):
        s = self.shape
        if x.shape != (s.B, s.heads, s.S, s.head_dim) or x.dtype is not self.dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"Rotary: {what} has to be [B, heads, S, head_dim] of the layer's type on {self.device}, contiguous")

    def _weights(self, weights, n):
        if weights is None or self.n_weights == 0:
            return None
        weights = [*weights, *[None] * (n - len(weights))]
        for w in weights:
            if w is not None and (w.numel() != self.n_weights or w.dtype != torch.float32 or not w.is_contiguous() or w.device != self.device):
                raise ValueError(f"Rotary: a weight has to be {self.n_weights} contiguous fp32 values on {self.device}")
        return weights

    def _blocks(self, shape):
        """The shape whose blocks block order means: this object's, or another of the same sizes (positions know no blocks)."""
        if shape is None:
            return self.shape
        if any(getattr(shape, n) != getattr(self.shape, n) for n in ("B", "S", "heads", "head_dim", "dtype")):
            raise ValueError("Rotary: a layer's shape has to have the samples, tokens, heads, head_dim and type of the Rotary's")
        return shape

    def forward(self, xs, outs, weights=None, block_order=False, moved=(), moved_outs=(), perm=None, shape=None):
        """Norms and rotates the raster-order tensors xs into outs: raster order, or block-major [B, heads, S, d] with block_order.
        moved: tensors that only go along (v into block order).  shape: one of the same sizes in other blocks."""
        xs, outs = list(xs) + list(moved), list(outs) + list(moved_outs)
        if len(xs) != len(outs) or not 1 <= len(xs) <= 4:
            raise ValueError("Rotary: one to four tensors, and an output for each")
        shape = self._blocks(shape)
        src = [self._raster(x, "an input") for x in xs]
        dst = None if block_order else [self._raster(x, "an output") for x in outs]
        if block_order:
            for x in outs:
                self._block_major(x, "an output in block order")
        if perm is not None and (perm.numel() < self.shape.S or perm.dtype != torch.int32 or not perm.is_contiguous() or perm.device != self.device):
            raise ValueError(f"Rotary: perm has to be {self.shape.S} contiguous int32 values on {self.device}")
        with _on(self.device):
            vb.vmoba_rotary(shape, self.spec, len(xs) - len(moved), xs, src, outs, dst, self._weights(weights, len(xs)),
                            self.positions, self.freq, self.axis, perm)

    def backward(self, d_outs, xs, dxs, weights=None, block_order=False, shape=None):
        """Gradients of forward(): dxs (raster order; may be d_outs) from d_outs (block-major with block_order) and the forward's
        xs (unused without a norm); shape as given to that.  Returns the weights' gradients, fp32, or None without a norm."""
        n = len(d_outs)
        shape = self._blocks(shape)
        if n != len(dxs) or not 1 <= n <= 4 or (self.n_weights and (xs is None or len(xs) != n)):
            raise ValueError("Rotary: one to four gradients, as many results and, with a norm, as many inputs")
        d_strides = None if block_order else [self._raster(x, "a gradient") for x in d_outs]
        if block_order:
            for x in d_outs:
                self._block_major(x, "a gradient in block order")
        dx_strides = [self._raster(x, "a result") for x in dxs]
        x_strides = [self._raster(x, "an input") for x in xs] if self.n_weights else None
        dw = [torch.empty(self.n_weights, dtype=torch.float32, device=self.device) for _ in range(n)] if self.n_weights else None
        ws = torch.empty(self._scratch[n], dtype=torch.uint8, device=self.device) if self.n_weights else None
        with _on(self.device):
            vb.vmoba_rotary_bwd(shape, self.spec, d_outs, d_strides, xs if self.n_weights else None, x_strides,
                                self._weights(weights, n), dxs, dx_strides, dw, self.positions, self.freq, self.axis, ws)
        return dw


_F32, _BF16 = torch.float32, torch.bfloat16


class _Rows:
    """What Linear, FeedForward and BlockNorm share: checks of tensors [B, S, channels] and of rows of gates."""

    def _rows(self, x, channels, dtype, what, written=False):
        """x as the kernels can address it (an input that they cannot is copied) and its strides (batch, token)."""
        known = self._sizes.get(channels)
        if known is None:
            known = self._sizes[channels] = (torch.Size((self.shape.B, self.shape.S, channels)), (self.shape.S * channels, channels))
        size, dense = known
        if x.shape != size or x.dtype is not dtype or x.device != self.device:
            raise ValueError(f"{type(self).__name__}: {what} has to be {dtype} {list(size)} on {self.device}")
        if x.is_contiguous() and x.data_ptr() % 16 == 0:
            return x, dense
        st, per = x.stride(), 16 // x.element_size()
        if x.stride(2) == 1 and x.data_ptr() % 16 == 0 and all(n == 1 or (i % per == 0 and channels <= i < 2 ** 38) for n, i in zip(size, st[:2])):
            return x, st[:2]
        if written:
            raise ValueError(f"{type(self).__name__}: {what} needs 16-byte rows on 16-byte boundaries that do not share memory")
        x = torch.empty(size, dtype=dtype, device=x.device).copy_(x)
        return x, dense

    def _groups(self, g, channels, what):
        """Rows of a gate, scale or shift [B (or 1), groups, channels] and their strides (batch, group)."""
        if g is None:
            return None, (0, 0)
        n, B = g.shape, self._B
        if len(n) != 3 or (n[0] != B and n[0] != 1) or n[1] != self._n_groups or n[2] != channels or g.dtype is not _F32 or g.device != self.device:
            raise ValueError(f"{type(self).__name__}: {what} has to be fp32 [{B} or 1, {self._n_groups}, {channels}] on {self.device}")
        st = g.stride()
        sb, sg = 0 if n[0] == 1 else st[0], 0 if n[1] == 1 else st[1]
        if st[2] != 1 or g.data_ptr() % 16 or sb % 4 or sg % 4 or (sb and not channels <= sb < 2 ** 38) or (sg and not channels <= sg < 2 ** 38):
            g = torch.empty(n, dtype=_F32, device=g.device).copy_(g)
            sb, sg = 0 if n[0] == 1 else n[1] * channels, 0 if n[1] == 1 else channels
        return g, (sb, sg)

    def _dense(self, x, shape, dtype, what):
        """A contiguous tensor of this shape; one that begins elsewhere than on 16 bytes is copied."""
        if x is None:
            return None
        if x.shape != shape or x.dtype is not dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{type(self).__name__}: {what} has to be {dtype} {list(shape)} on {self.device}, contiguous")
        return x if x.data_ptr() % 16 == 0 else torch.empty_like(x).copy_(x)

    def _written(self, x, shape, dtype, what):
        if x is not None and self._dense(x, shape, dtype, what) is not x:
            raise ValueError(f"{type(self).__name__}: {what} has to begin on a 16-byte boundary")
        return x

    def _new(self, shape, dtype, wanted=True):
        return torch.empty(shape, dtype=dtype, device=self.device) if wanted else None

    def _start(self, shape, device):
        self.shape, self.device = shape, _cuda_device(device, type(self).__name__)
        self._n_groups, self._B, self._sizes = shape.groups, shape.B, {}
        self.dtype = torch_dtype(shape)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self._nothing = torch.empty(256, dtype=torch.uint8, device=self.device)      # what calls take that need no scratch

    def _scratch(self, n):
        """A call's own, so that calls on any streams and in any graphs can be under way at the same time (256 bytes: it uses none)."""
        return self._nothing if n == 256 else torch.empty(n, dtype=torch.uint8, device=self.device)

    def check_status(self):
        code = int(self.dev_status.item())
        if code != vb.OK:
            raise vb.VmobaError(code, "device status")


def _cuda_device(device, what):
    d = torch.device(device)
    if d.type != "cuda":
        raise ValueError(f"{what}: a GPU required")
    return torch.device("cuda", torch.cuda.current_device() if d.index is None else d.index)


class Linear(_Rows):
    """A linear layer with what follows it in a transformer block: out = residual + gate * act(x W^T + bias); gated: W is [2 n_out, n_in], and
    act(first half of the product) * second half takes the place of act(..).

    shape: binding.make_linear_shape().  x is [B, S, n_in], or with heads the block-major [B, heads, S, n_in / heads] that an attention layer
    leaves, perm then being the raster token of its every position (VmobaLayer.perm).  The object holds no tensors of a call (but a word for
    the device's status), so that any number of streams and captured graphs can use it at the same time."""

    def __init__(self, shape, device="cuda"):
        self._start(shape, device)
        self._ws = vb.linear_workspace_bytes(shape)
        if self._ws == 0:
            raise ValueError("Linear: channels are multiples of 8, heads of 64 or 128 channels; shape out of range")
        self._ws_bwd = vb.linear_workspace_bytes(shape, True)

    def _input(self, x, what, written=False):
        s = self.shape
        if not s.heads:
            return self._rows(x, s.n_in, self.dtype, what, written)
        return (self._written if written else self._dense)(x, (s.B, s.heads, s.S, s.n_in // s.heads), self.dtype, what), None

    def _perm(self, perm):
        if perm is not None and (not self.shape.heads or perm.dtype != torch.int32 or perm.numel() != self.shape.S or not perm.is_contiguous()
                                 or perm.device != self.device):
            raise ValueError(f"Linear: perm goes with heads, and is {self.shape.S} contiguous int32 values on {self.device}")
        return perm

    def forward(self, x, weight, out, bias=None, gate=None, residual=None, perm=None, kept=None):
        """Writes out [B, S, n_out], which may be the residual.  kept [B, S, n_out or 2 n_out]: receives x W^T + bias, in the order of x, for
        backward()."""
        s, dt = self.shape, self.dtype
        x, xs = self._input(x, "x")
        weight = self._dense(weight, (s.wide, s.n_in), dt, "weight")
        bias = self._dense(bias, (s.wide,), dt, "bias")
        gate, gs = self._groups(gate, s.n_out, "gate")
        residual, rs = (None, None) if residual is None else self._rows(residual, s.n_out, dt, "residual")
        out, os_ = self._rows(out, s.n_out, dt, "out", True)
        kept = self._written(kept, (s.B, s.S, s.wide), dt, "kept")
        with _on(self.device):
            vb.vmoba_linear(s, x, xs, weight, bias, gate, gs, residual, rs, out, os_, kept, self._perm(perm), self.dev_status,
                            self._scratch(self._ws))

    def backward(self, d_out, x, weight, dx_out, kept=None, gate=None, perm=None, with_weight=True, with_bias=False):
        """Gradients of forward(), whose residual's is d_out: writes dx_out (the order of x; None: not wanted), returns those of weight, bias
        and gate (fp32 [B, groups, n_out]), None for what is not wanted or not there.  kept as forward() left it; without an activation, gated product
        or gate it may be None.  In bf16 the gradient of the product is rounded once ahead of dx_out and the weight's (small calls hold it to
        2^-16).  Places that perm sends outside the sample have gradients of zero; x has to be finite there."""
        s, dt = self.shape, self.dtype
        d_out, dos = self._rows(d_out, s.n_out, dt, "d_out")
        x, xs = self._input(x, "x")
        weight = self._dense(weight, (s.wide, s.n_in), dt, "weight")
        kept = self._dense(kept, (s.B, s.S, s.wide), dt, "kept")
        gate, gs = self._groups(gate, s.n_out, "gate")
        if kept is None and (s.activation != vb.ACT_NONE or s.gated or gate is not None):
            raise ValueError("Linear: this layer's backward() needs what forward() left in kept")
        dx_out, dxs = (None, None) if dx_out is None else self._input(dx_out, "dx_out", True)
        dw, db = self._new((s.wide, s.n_in), dt, with_weight), self._new((s.wide,), dt, with_bias)
        dg = self._new((s.B, s.groups, s.n_out), _F32, gate is not None)
        with _on(self.device):
            vb.vmoba_linear_bwd(s, d_out, dos, x, xs, weight, kept, gate, gs, dx_out, dxs, dw, db, dg, self._perm(perm), self.dev_status,
                                self._scratch(self._ws_bwd))
        return dw, db, dg


class FeedForward(_Rows):
    """A feed-forward block: out = residual + gate * (h W_down^T + b_down), h = act(x W_up^T + b_up); gated: W_up is [2 hidden, channels], and
    h = act(first half of the product) * second half.  Holds no tensors of a call (but a word for the device's status)."""

    def __init__(self, B, S, channels, hidden, dtype="bf16", activation="gelu", gated=False, gate_tokens=0, device="cuda"):
        self._start(vb.make_linear_shape(B, S, channels, hidden, dtype, activation, gated, 0, gate_tokens), device)
        self._ws = vb.ffn_workspace_bytes(self.shape)
        if self._ws == 0:
            raise ValueError("FeedForward: channels are multiples of 8; shape out of range")
        self._ws_bwd = vb.ffn_workspace_bytes(self.shape, True)

    def keep(self):
        """Tensors for forward() to leave in what backward() needs: the products ahead of the activation and of the gate."""
        s = self.shape
        return self._new((s.B, s.S, s.wide), self.dtype), self._new((s.B, s.S, s.n_in), self.dtype)

    def _weights(self, w_up, w_down):
        s = self.shape
        return (self._dense(w_up, (s.wide, s.n_in), self.dtype, "w_up"), self._dense(w_down, (s.n_in, s.n_out), self.dtype, "w_down"))

    def forward(self, x, w_up, w_down, out, b_up=None, b_down=None, gate=None, residual=None, kept=None):
        """Writes out [B, S, channels], which may be the residual.  kept: keep(), filled for backward()."""
        s, dt = self.shape, self.dtype
        x, xs = self._rows(x, s.n_in, dt, "x")
        w_up, w_down = self._weights(w_up, w_down)
        b_up, b_down = self._dense(b_up, (s.wide,), dt, "b_up"), self._dense(b_down, (s.n_in,), dt, "b_down")
        gate, gs = self._groups(gate, s.n_in, "gate")
        residual, rs = (None, None) if residual is None else self._rows(residual, s.n_in, dt, "residual")
        out, os_ = self._rows(out, s.n_in, dt, "out", True)
        up, down = (None, None) if kept is None else kept
        up, down = self._written(up, (s.B, s.S, s.wide), dt, "kept"), self._written(down, (s.B, s.S, s.n_in), dt, "kept")
        with _on(self.device):
            vb.vmoba_ffn(s, x, xs, w_up, b_up, w_down, b_down, gate, gs, residual, rs, out, os_, up, down, self.dev_status,
                         self._scratch(self._ws))

    def backward(self, d_out, x, w_up, w_down, kept, dx_out, gate=None, with_weights=True, with_bias=False):
        """Gradients of forward(), whose residual's is d_out: writes dx_out (None: not wanted), returns those of w_up, w_down, b_up, b_down and
        gate (fp32 [B, groups, channels]), None for what is not wanted or not there.  kept: as forward() left it; without a gate the
        second of the two may be None."""
        s, dt = self.shape, self.dtype
        d_out, dos = self._rows(d_out, s.n_in, dt, "d_out")
        x, xs = self._rows(x, s.n_in, dt, "x")
        w_up, w_down = self._weights(w_up, w_down)
        up, down = self._dense(kept[0], (s.B, s.S, s.wide), dt, "kept"), self._dense(kept[1], (s.B, s.S, s.n_in), dt, "kept")
        gate, gs = self._groups(gate, s.n_in, "gate")
        if up is None or (gate is not None and down is None):
            raise ValueError("FeedForward: backward() needs what forward() left in kept")
        dx_out, dxs = (None, None) if dx_out is None else self._rows(dx_out, s.n_in, dt, "dx_out", True)
        dwu, dwd = self._new((s.wide, s.n_in), dt, with_weights), self._new((s.n_in, s.n_out), dt, with_weights)
        dbu, dbd = self._new((s.wide,), dt, with_bias), self._new((s.n_in,), dt, with_bias)
        dg = self._new((s.B, s.groups, s.n_in), _F32, gate is not None)
        with _on(self.device):
            vb.vmoba_ffn_bwd(s, d_out, dos, x, xs, w_up, w_down, up, down, gate, gs, dx_out, dxs, dwu, dbu, dwd, dbd, dg, self.dev_status,
                             self._scratch(self._ws_bwd))
        return dwu, dwd, dbu, dbd, dg


class BlockNorm(_Rows):
    """What stands between two branches of a transformer block: h = x + gate * post(y), out = (norm(h) * weight + bias) * (1 + scale) + shift.

    shape: binding.make_norm_shape().  x, y, h and out are [B, S, channels], x and h of the stream's type; gate, scale and shift fp32
    [B or 1, groups, channels], one row for mod_tokens tokens; weight, bias and post_weight fp32 [channels]; everything but x may be
    left out.  Holds no tensors of a call (but a word for the device's status)."""

    def __init__(self, shape, device="cuda"):
        self._start(shape, device)
        self._ws = vb.block_norm_workspace_bytes(shape)
        if self._ws == 0:
            raise ValueError("BlockNorm: channels are multiples of 8 up to 8192, fp32 branches go with fp32 streams; shape out of range")
        self.stream_dtype = _BF16 if shape.stream_dtype == vb.BF16 else _F32

    def _params(self, gate, scale, shift, weight, bias, post_weight):
        C = self.shape.C
        gs = ss = hs = (0, 0)
        if gate is not None:
            gate, gs = self._groups(gate, C, "gate")
        if scale is not None:
            scale, ss = self._groups(scale, C, "scale")
        if shift is not None:
            shift, hs = self._groups(shift, C, "shift")
        if weight is not None:
            weight = self._dense(weight, (C,), _F32, "weight")
        if bias is not None:
            bias = self._dense(bias, (C,), _F32, "bias")
        if post_weight is not None:
            post_weight = self._dense(post_weight, (C,), _F32, "post_weight")
        # (with what the pointers are of: copies live until the launch)
        return vb.norm_params(gate, gs, scale, ss, shift, hs, weight, bias, post_weight), (gate, scale, shift, weight, bias, post_weight)

    def _opt(self, x, dtype, what, written=False):
        return (None, None) if x is None else self._rows(x, self.shape.C, dtype, what, written)

    def forward(self, x, out=None, y=None, h_out=None, gate=None, scale=None, shift=None, weight=None, bias=None, post_weight=None):
        """Writes out and h_out (either may be None; h_out may be x)."""
        params, held = self._params(gate, scale, shift, weight, bias, post_weight)
        x, xs = self._rows(x, self.shape.C, self.stream_dtype, "x")
        y, ys = self._opt(y, self.dtype, "y")
        h_out, hs = self._opt(h_out, self.stream_dtype, "h_out", True)
        out, os_ = self._opt(out, self.dtype, "out", True)
        if out is None and h_out is None:
            raise ValueError("BlockNorm: out or h_out required")
        with _on(self.device):
            vb.vmoba_block_norm(self.shape, params, x, xs, y, ys, h_out, hs, out, os_, self.dev_status)

    def backward(self, d_out, h, dx_out, d_h=None, y=None, dy_out=None, gate=None, scale=None, shift=None, weight=None, bias=None,
                 post_weight=None):
        """Gradients of forward() from its h (x, where there was no y): writes dx_out (that of x; may be d_h, what else arrives at h) and
        dy_out; returns a dict of dgate, dscale, dshift (fp32 [B, groups, channels]), dweight, dbias and dpost_weight (fp32 [channels]), None
        where the parameter is not there."""
        s, C = self.shape, self.shape.C
        params, held = self._params(gate, scale, shift, weight, bias, post_weight)
        if y is None and (dy_out is not None or gate is not None or post_weight is not None):
            raise ValueError("BlockNorm: dy_out, gate and post_weight go with y")
        d_out, dos = self._rows(d_out, C, self.dtype, "d_out")
        h, hs = self._rows(h, C, self.stream_dtype, "h")
        d_h, dhs = self._opt(d_h, self.stream_dtype, "d_h")
        y, ys = self._opt(y, self.dtype, "y")
        dx_out, dxs = self._rows(dx_out, C, self.stream_dtype, "dx_out", True)
        dy_out, dys = self._opt(dy_out, self.dtype, "dy_out", True)
        there = {"gate": gate, "scale": scale, "shift": shift, "weight": weight, "bias": bias, "post_weight": post_weight}
        grads = {n: self._new((s.B, s.groups, C) if n in ("gate", "scale", "shift") else (C,), _F32) for n, t in there.items() if t is not None}
        with _on(self.device):
            vb.vmoba_block_norm_bwd(s, params, d_out, dos, h, hs, d_h, dhs, y, ys, dx_out, dxs, dy_out, dys, grads, self.dev_status,
                                    self._scratch(self._ws))
        return {"d" + n: grads.get(n) for n in there}


class VmobaLayer:
    """Owns the device buffers of one layer shape and runs the stages on the current stream."""

    def __init__(self, shape, capacity: int, device="cuda", with_backward: bool = False):
        self.shape = shape
        self.capacity = int(capacity)
        self.device = torch.device(device)
        s = shape
        dt = torch_dtype(s)
        dev = self.device
        BH, S, d, Nb = s.B * s.heads, s.S, s.head_dim, s.n_blocks
        self.BH, self.S, self.d, self.Nb = BH, S, d, Nb
        bm = lambda: torch.empty((s.B, s.heads, S, d), dtype=dt, device=dev)
        self.q_bm, self.k_bm, self.v_bm, self.o_bm = bm(), bm(), bm(), bm()
        self.centroids = torch.empty((s.B, s.heads, Nb, d), dtype=torch.float32, device=dev)
        self.scores = torch.empty((s.B, s.heads, S, Nb), dtype=torch.float32, device=dev)
        self.mask_bits = torch.empty((BH * S, s.mask_words), dtype=torch.int32, device=dev)
        self.kb_ptr = torch.empty(BH * Nb + 1, dtype=torch.int32, device=dev)
        self.q_idx = torch.empty(self.capacity, dtype=torch.int32, device=dev)
        self.q_ptr = torch.empty(BH * S + 1, dtype=torch.int32, device=dev)
        self.q_pairs = torch.empty(self.capacity, dtype=torch.int32, device=dev)
        self.k_per_head = torch.empty(BH, dtype=torch.int64, device=dev)
        self.cutoff = torch.empty(BH, dtype=torch.float32, device=dev)
        self.score_range = torch.empty((BH, 2), dtype=torch.float32, device=dev)   # per head: smallest, largest score
        self.range_valid = False
        self.lse = torch.empty(BH * S, dtype=torch.float32, device=dev)
        self.perm = torch.empty(S, dtype=torch.int32, device=dev)     # raster token of block-major position p (Eq. 1)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        stages = [vb.STAGE_SCORES, vb.STAGE_SELECT, vb.STAGE_ATTN_FWD]
        if with_backward:
            stages.append(vb.STAGE_ATTN_BWD)
            self.do_bm, self.dq_bm, self.dk_bm, self.dv_bm = bm(), bm(), bm(), bm()
        # rounding residual of o, kept for the backward's rowsum(dO * O) (bf16 training only)
        self.o_resid = bm() if (with_backward and s.dtype == vb.BF16) else None
        ws_bytes = max(vb.workspace_bytes(s, st, self.capacity) for st in stages)
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        self.with_backward = with_backward
        self.o_raster = None          # the raster-order o of the last attn_fwd_raster, if that is how o was written

    # ---- stage wrappers -----------------------------------------------------------------
    @staticmethod
    def raster_strides(x):
        """Element strides (batch, token, head) of a [B, S, heads, d] tensor."""
        s = x.stride()
        assert s[3] == 1
        return s[:3]

    def partition(self, raster, bm, inverse=False, perm=None, inv_perm=None):
        src, dst = (bm, raster) if inverse else (raster, bm)
        vb.vmoba_partition(self.shape, int(inverse), src, dst, self.raster_strides(raster), perm, inv_perm)

    def partition_many(self, rasters, bms, inverse=False, perm=None):
        """Up to four tensors of the layer's shape into block-major order (inverse: back), and the permutation table, in
        one launch."""
        srcs, dsts = (bms, rasters) if inverse else (rasters, bms)
        vb.vmoba_partition_many(self.shape, int(inverse), srcs, dsts, [self.raster_strides(x) for x in rasters], perm=perm)

    def partitions(self, raster) -> bool:
        """Whether partition() takes this tensor as it lies: the layer's type, 16-byte rows on 16-byte boundaries."""
        e = 16 // raster.element_size()
        return (raster.dtype == self.q_bm.dtype and raster.stride(3) == 1 and raster.data_ptr() % 16 == 0
                and all(x % e == 0 for x in raster.stride()[:3]))

    def block_scores(self, with_range=True):
        """Centroids and scores; with_range: the scores kernel also takes each head's smallest and largest score,
        which lets select() skip its own pass for them (valid until self.scores is overwritten by other means)."""
        if with_range:
            vb.vmoba_block_scores_range(self.shape, self.q_bm, self.k_bm, self.centroids, self.scores, self.score_range,
                                        self.dev_status, self.ws)
        else:
            vb.vmoba_block_scores(self.shape, self.q_bm, self.k_bm, self.centroids, self.scores, self.dev_status, self.ws)
        self.range_valid = bool(with_range)

    def select(self, tau, scores=None, use_range=None):
        """Eq. 3 + Eq. 4.  use_range: take the score range the last block_scores() left (default: if it left one and
        the scores are the layer's own)."""
        if use_range is None:
            use_range = self.range_valid and scores is None
        if use_range:
            vb.vmoba_select_ranged(self.shape, self.scores, self.score_range, vb.SELECT_THRESHOLD_GLOBAL, tau, 0,
                                   self.mask_bits, self.kb_ptr, self.q_idx, self.q_ptr, self.q_pairs, self.capacity,
                                   self.k_per_head, self.cutoff, self.dev_status, self.ws)
            return
        vb.vmoba_select(self.shape, self.scores if scores is None else scores, tau, self.mask_bits, self.kb_ptr,
                        self.q_idx, self.q_ptr, self.q_pairs, self.capacity, self.k_per_head, self.cutoff,
                        self.dev_status, self.ws)

    def select_rule(self, rule, tau=0.25, topk=1, scores=None):
        ws = self.ws
        if (rule & 0xff) == vb.SELECT_THRESHOLD_GLOBAL_ROWNORM:
            # this rule keeps a transformed copy of the score matrix in its scratch: allocated on first use
            need = vb.workspace_bytes(self.shape, vb.STAGE_SELECT_ROWNORM, self.capacity)
            if getattr(self, "ws_rownorm", None) is None or self.ws_rownorm.numel() < need:
                self.ws_rownorm = torch.empty(need, dtype=torch.uint8, device=self.ws.device)
            ws = self.ws_rownorm
        vb.vmoba_select_rule_apply(self.shape, self.scores if scores is None else scores, rule, tau, topk, self.mask_bits,
                                   self.kb_ptr, self.q_idx, self.q_ptr, self.q_pairs, self.capacity, self.k_per_head,
                                   self.cutoff, self.dev_status, ws)

    def attn_fwd(self):
        self.o_raster = None
        vb.vmoba_attn_fwd(self.shape, self.q_bm, self.k_bm, self.v_bm, self.kb_ptr, self.q_idx, self.q_ptr,
                          self.q_pairs, self.capacity, self.o_bm, self.o_resid, self.lse, self.dev_status, self.ws)

    def attn_bwd(self):
        vb.vmoba_attn_bwd(self.shape, self.q_bm, self.k_bm, self.v_bm, self.o_bm, self.o_resid, self.lse, self.do_bm,
                          self.kb_ptr, self.q_idx, self.q_ptr, self.capacity, self.dq_bm, self.dk_bm, self.dv_bm,
                          self.dev_status, self.ws)

    def can_fold_inverse(self, dq_out, dk_out, dv_out) -> bool:
        """Whether the backward kernels can write these raster-order gradients themselves."""
        strides = self.raster_strides(dq_out)
        return (self.shape.dtype == vb.BF16 and self.d == 128 and self.raster_strides(dk_out) == strides
                and self.raster_strides(dv_out) == strides)

    def can_fold_o(self) -> bool:
        """Whether the forward kernels can write o in raster order themselves."""
        return self.shape.dtype == vb.BF16 and self.d == 128

    def attn_fwd_raster(self, o_out):
        """Forward writing o straight into the raster-order tensor o_out (needs self.perm from the partition of q).
        The tensor is remembered: a following attn_bwd_raster reads o from it."""
        vb.vmoba_attn_fwd_raster(self.shape, self.q_bm, self.k_bm, self.v_bm, self.kb_ptr, self.q_idx, self.q_ptr,
                                 self.q_pairs, self.capacity, o_out, self.raster_strides(o_out), self.perm,
                                 self.o_resid, self.lse, self.dev_status, self.ws)
        self.o_raster = o_out

    def attn_bwd_raster(self, do_raster_or_none, dq_out, dk_out, dv_out, keep_do=False):
        """Backward writing dq, dk, dv in raster order (needs self.perm from the forward's partition of q); dO is
        read in raster order too if given, else from self.do_bm; keep_do: the pass that reads it first leaves it in
        self.do_bm and the attention kernel reads it there; o is read from the raster-order tensor the last
        attn_fwd_raster wrote, else from self.o_bm."""
        do = self.do_bm if do_raster_or_none is None else do_raster_or_none
        dos = None if do_raster_or_none is None else self.raster_strides(do)
        o = self.o_bm if self.o_raster is None else self.o_raster
        os_ = None if self.o_raster is None else self.raster_strides(o)
        vb.vmoba_attn_bwd_raster(self.shape, self.q_bm, self.k_bm, self.v_bm, o, os_, self.o_resid, self.lse, do,
                                 dos, self.kb_ptr, self.q_idx, self.q_ptr, self.capacity, dq_out,
                                 dk_out, dv_out, self.raster_strides(dq_out), self.perm, self.dev_status, self.ws,
                                 do_bm=self.do_bm if keep_do else None)

    # ---- whole layer --------------------------------------------------------------------
    def forward(self, q, k, v, tau, o_out, fold_o=None, rotary=None, weights=None, projection=None, projected=None):
        """q, k, v, o_out: [B, S, heads, d] raster-order tensors on the device.

        projection: a Linear of the layer's samples, tokens and heads that o goes through on its way out of block order, instead of an inverse
        partition pass; o_out is then its output [B, S, n_out].  projected: what its forward() takes besides (weight, and as wanted bias, gate,
        residual, kept).

        rotary: a Rotary of the layer's sizes, whatever its blocks, that q and k go through on their way into block order (its weights:
        of q and of k).

        fold_o: let the forward kernels write o in raster order themselves (bf16, head_dim 128) instead of an inverse
        partition pass; off by default (measured on B200: the scattered 256-byte row writes cost the attention kernel
        more than the pass they save, at 12 heads as at 40).  o_out must then stay alive and unchanged until backward()."""
        if projection is not None:
            self._projects(projection, projected)
            if fold_o:
                raise ValueError("VmobaLayer: a projection takes o in block order (fold_o)")
        # k last: the centroids, computed next, find the end of it in L2
        if rotary is not None:
            rotary.forward((k, q), (self.k_bm, self.q_bm), None if weights is None else (weights[1], weights[0]), block_order=True,
                           moved=(v,), moved_outs=(self.v_bm,), perm=self.perm, shape=self.shape)
        else:
            self.partition_many((v, q, k), (self.v_bm, self.q_bm, self.k_bm), perm=self.perm)
        self.block_scores()
        self.select(tau)
        if projection is not None:
            self.attn_fwd()
            projection.forward(self.o_bm, out=o_out, perm=self.perm, **projected)
            return
        if fold_o:
            self.attn_fwd_raster(o_out)
            return
        self.attn_fwd()
        self.partition(o_out, self.o_bm, inverse=True)

    def _projects(self, projection, projected):
        s, p = self.shape, projection.shape
        if not projected or "weight" not in projected:
            raise ValueError("VmobaLayer: projected has to have the projection's weight")
        if (p.B, p.S, p.heads, p.n_in, p.dtype) != (s.B, s.S, s.heads, s.heads * s.head_dim, s.dtype):
            raise ValueError("VmobaLayer: a projection has to be a Linear of the layer's samples, tokens, heads, channels and type")

    def backward(self, do, dq_out, dk_out, dv_out, fold_inverse=None, fold_do=False, rotary=None, qk=None, weights=None, projection=None,
                 projected=None):
        """Gradients of the last forward(); do and the outputs are raster-order [B, S, heads, d].

        projection: as given to forward(); do is then the gradient of its output [B, S, n_out], and projected what its backward() takes
        besides (weight, and as wanted kept, gate, with_weight, with_bias).  What that returns comes back, with a rotary after the
        weights' gradients of that.

        rotary, weights: as given to forward(), with its (q, k) in qk where the Rotary has a norm; dq_out and dk_out are then the
        gradients of those, and the weights' are returned.

        fold_inverse: let the backward kernels write dq, dk, dv in raster order themselves (bf16, head_dim 128,
        outputs with equal strides) instead of three inverse partition passes; default: whenever possible.
        fold_do: also let the attention kernel read dO in raster order; by default the pass before it, which reads dO
        for its own purpose, leaves a block-major copy."""
        if fold_inverse is None:
            fold_inverse = self.can_fold_inverse(dq_out, dk_out, dv_out)
        if projection is not None:               # its input's gradient is block-major: do as the kernels read it
            self._projects(projection, projected)
            if fold_do or self.o_raster is not None:
                raise ValueError("VmobaLayer: a projection takes o and hands do over in block order (fold_o, fold_do)")
            grads = projection.backward(do, self.o_bm, dx_out=self.do_bm, perm=self.perm, **projected)
            if fold_inverse:
                self.attn_bwd_raster(None, dq_out, dk_out, dv_out)
                return grads if rotary is None else (rotary.backward((dq_out, dk_out), qk, (dq_out, dk_out), weights), grads)
            self.attn_bwd()
            dw = self._gradients_out(dq_out, dk_out, dv_out, rotary, qk, weights)
            return grads if rotary is None else (dw, grads)
        if fold_inverse:
            if fold_do:
                self.attn_bwd_raster(do, dq_out, dk_out, dv_out)
            else:
                self.attn_bwd_raster(do, dq_out, dk_out, dv_out, keep_do=True)
            return None if rotary is None else rotary.backward((dq_out, dk_out), qk, (dq_out, dk_out), weights)
        self.partition(do, self.do_bm)
        if self.o_raster is not None:      # the block-major backward reads o_bm, which the raster forward did not write
            self.partition(self.o_raster, self.o_bm)
        self.attn_bwd()
        return self._gradients_out(dq_out, dk_out, dv_out, rotary, qk, weights)

    def _gradients_out(self, dq_out, dk_out, dv_out, rotary, qk, weights):
        """The block-major gradients into raster order, through the rotary where there is one."""
        if rotary is not None:
            self.partition(dv_out, self.dv_bm, inverse=True)
            return rotary.backward((self.dq_bm, self.dk_bm), qk, (dq_out, dk_out), weights, block_order=True, shape=self.shape)
        self.partition_many((dq_out, dk_out, dv_out), (self.dq_bm, self.dk_bm, self.dv_bm), inverse=True)

    def check_status(self):
        code = int(self.dev_status.item())
        if code != vb.OK:
            raise vb.VmobaError(code, "device status")

    def n_selected(self) -> int:
        return int(self.k_per_head.sum().item())


def dense_step_schedule(n_steps: int, dense_fraction: float = 0.25):
    """Which denoising steps of a sampling run use full attention: the paper's training-free setting runs the
    first 25 % of the steps dense and the rest through VMoBA (Section 4.1, implementation details).  Returns a list
    of n_steps booleans, True = dense; the number of dense steps is ceil(dense_fraction * n_steps)."""
    if n_steps < 0 or not (0.0 <= dense_fraction <= 1.0):
        raise ValueError("n_steps >= 0 and 0 <= dense_fraction <= 1 required")
    n_dense = min(n_steps, int(math.ceil(dense_fraction * n_steps - 1e-9)))
    return [i < n_dense for i in range(n_steps)]


class SteppedAttention:
    """Host-side switch between the dense path and the sparse layer over the steps of a sampler: step i of
    n_steps calls vmoba_full_attn while dense_step_schedule says so, the VMoBA layer afterwards (forward only:
    this is the inference setting).  Tensors are raster-order [B, S, heads, d] on the device."""

    def __init__(self, layer: VmobaLayer, tau: float, n_steps: int, dense_fraction: float = 0.25):
        self.layer, self.tau = layer, tau
        self.schedule = dense_step_schedule(n_steps, dense_fraction)
        s = layer.shape
        self._lse = torch.empty(s.B * s.heads * s.S, dtype=torch.float32, device=layer.device)
        # the grid as one block: the partition into it keeps the raster order of the tokens
        self._one_block = vb.Shape.from_buffer_copy(s)
        self._one_block.bT, self._one_block.bH, self._one_block.bW = s.T, s.H, s.W

    def forward(self, step: int, q, k, v, o_out, rotary=None, weights=None, projection=None, projected=None) -> str:
        """Runs step `step`; returns which path ran ("dense" or "sparse").  rotary, weights, projection, projected: as for
        VmobaLayer.forward()."""
        if self.schedule[step]:
            # the dense kernels take [B, heads, S, d].  The tokens stay in raster order: the running maximum that a row's
            # weights are rounded against, and with it the last bits of o, depends on the order of the keys.
            L, one = self.layer, self._one_block
            if projection is not None:
                L._projects(projection, projected)
            # (a fresh tensor, not contiguous(): that returns a contiguous tensor as it is, whatever its address, the strides
            # of its dimensions of size one and its type)
            fresh = lambda x: torch.empty(x.shape, dtype=L.q_bm.dtype, device=L.device)
            q, k, v = (x if L.partitions(x) else fresh(x).copy_(x) for x in (q, k, v))
            qd, kd, vd, od = (torch.empty_like(L.q_bm) for _ in range(4))
            if rotary is not None:
                rotary.forward((q, k), (qd, kd), weights, block_order=True, moved=(v,), moved_outs=(vd,), shape=one)
            else:
                vb.vmoba_partition_many(one, 0, (q, k, v), (qd, kd, vd), [L.raster_strides(x) for x in (q, k, v)])
            vb.vmoba_full_attn(L.shape, qd, kd, vd, od, self._lse, dev_status=L.dev_status)
            if projection is not None:       # (od has the tokens in raster order)
                projection.forward(od, out=o_out, **projected)
                return "dense"
            # (an o_out whose elements share memory goes through copy_, which refuses it)
            shared = any(st == 0 and n > 1 for st, n in zip(o_out.stride(), o_out.shape))
            o = o_out if L.partitions(o_out) and not shared else fresh(o_out)
            vb.vmoba_partition(one, 1, od, o, L.raster_strides(o))
            if o is not o_out:
                o_out.copy_(o)
            return "dense"
        self.layer.forward(q, k, v, self.tau, o_out, rotary=rotary, weights=weights, projection=projection, projected=projected)
        return "sparse"


def key_ranges(lens, n_tokens=None, n_queries=None, frame: int = 0, prefix: int = 0, window: int = 0, device="cuda"):
    """The key ranges of RangeAttention, int32 [.., n_queries, 2].

    lens, with n_tokens: the lengths of the clips packed one behind another into a sequence of n_tokens (what is left over is padding
    and sees nothing); [1, n_tokens, 2].  lens, with n_queries: the filled length of each sample's cache, of which the queries are the
    last n_queries tokens; [len(lens), n_queries, 2].
    frame: a token sees up to the end of its own group of that many tokens, counted from its clip's start (1: causal; 0: its whole
    clip); prefix: the first tokens of a clip that all of it sees nevertheless; window: of those keys only the last so many."""
    lens = torch.as_tensor(lens, dtype=torch.int64, device=device)
    if (n_tokens is None) == (n_queries is None) or lens.dim() != 1 or lens.numel() == 0 or min(frame, prefix, window) < 0 or bool((lens < 0).any()):
        raise ValueError("key_ranges: lengths, and either n_tokens or n_queries, none of them negative, required")
    if n_tokens is not None:
        ends = lens.cumsum(0)
        if int(ends[-1]) > n_tokens:
            raise ValueError("key_ranges: the clips do not fit into the sequence")
        at = torch.arange(n_tokens, device=device)[None]
        clip = torch.searchsorted(ends, at, right=True)
        some = clip < lens.numel()
        clip = clip.clamp(max=lens.numel() - 1)
        lo, hi = (ends - lens)[clip], ends[clip]
    else:
        at = (lens - n_queries)[:, None] + torch.arange(n_queries, device=device)
        lo, hi, some = torch.zeros_like(at), lens[:, None].expand_as(at), at >= 0
    if frame:
        hi = torch.minimum(hi, lo + torch.maximum(((at - lo) // frame + 1) * frame, torch.full_like(at, prefix)))
    if window:
        lo = torch.maximum(lo, hi - window)
    return torch.stack([torch.where(some, lo, 0), torch.where(some, hi, 0)], -1).to(torch.int32).contiguous()


class RangeAttention:
    """Attention over key ranges, forward and gradients: the plan of the ranges, scratch, lse and the rounding residual.

    shape: binding.make_range_shape(); key_range: int32 [1 or B, Sq, 2] on the device (key_ranges).  Tensors are [B, S, heads, d], in
    whatever order of their dimensions but the last.  An object serves one stream at a time."""

    def __init__(self, shape, key_range, with_backward: bool = False):
        s = self.shape = shape
        self.device = key_range.device
        if not key_range.is_cuda or vb.range_plan_bytes(s) == 0:
            raise ValueError("RangeAttention: a valid shape and key ranges on a GPU required")
        e = lambda n, dt=torch.uint8: torch.empty(n, dtype=dt, device=self.device)
        self.plan = e(vb.range_plan_bytes(s))
        self.lse = e((s.B, s.heads, s.Sq), torch.float32)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=self.device)
        self.o_resid = e((s.B, s.Sq, s.heads, s.head_dim), torch.bfloat16) if with_backward and s.dtype == vb.BF16 else None
        self.ws = e(max(vb.range_workspace_bytes(s), vb.range_workspace_bytes(s, True) if with_backward else 0))
        self.with_backward = with_backward
        self.set_ranges(key_range)

    def set_ranges(self, key_range):
        """Takes other key ranges (a cache that has grown, another packing).  backward() then needs another forward()."""
        s = self.shape
        if tuple(key_range.shape) != (s.mask_batch, s.Sq, 2) or key_range.dtype != torch.int32 or key_range.device != self.device:
            raise ValueError("RangeAttention: key ranges are int32 [mask_batch, Sq, 2] on the plan's device")
        key_range = key_range.contiguous()
        if key_range.data_ptr() % 8:
            key_range = key_range.clone()                # (a pair is read as one word)
        self._kept = None          # (the last forward's lse and o belong to the ranges it ran under)
        with _on(self.device):
            vb.vmoba_range_plan(s, key_range, self.plan)

    def _tensor(self, x, S, heads, what, written=False):
        """x as the kernels can address it (an input that they cannot is copied) and its strides."""
        s = self.shape
        if x.shape != (s.B, S, heads, s.head_dim) or x.dtype is not torch_dtype(s) or x.device != self.device:
            raise ValueError(f"RangeAttention: {what} has to be [{s.B}, {S}, {heads}, {s.head_dim}] of the shape's type on {self.device}")
        if x.is_contiguous() and x.data_ptr() % 16 == 0:
            return x, (S * heads * s.head_dim, heads * s.head_dim, s.head_dim)
        st, per = _strides_bsh(x), 16 // x.element_size()
        if x.stride(3) == 1 and x.data_ptr() % 16 == 0 and all(i % per == 0 and i >= s.head_dim for i in st):
            return x, st
        if written:
            raise ValueError(f"RangeAttention: {what} needs 16-byte rows on 16-byte boundaries that do not share memory")
        x = torch.empty(x.shape, dtype=x.dtype, device=x.device).copy_(x)
        return x, _strides_bsh(x)

    def forward(self, q, k, v, o_out):
        """o_out = attention of q over k and v; self.lse [B, heads, Sq].  With a backward to come q, k, v and o_out stay as they are."""
        s = self.shape
        q, qs = self._tensor(q, s.Sq, s.heads, "q")
        k, ks = self._tensor(k, s.Sk, s.kv_heads, "k")
        v, vs = self._tensor(v, s.Sk, s.kv_heads, "v")
        _, os_ = self._tensor(o_out, s.Sq, s.heads, "o_out", True)
        with _on(self.device):
            vb.vmoba_range_attn_fwd(s, self.plan, q, qs, k, ks, v, vs, o_out, os_, self.o_resid, self.lse, self.dev_status, self.ws)
        if self.with_backward:
            self._kept = (q, qs, k, ks, v, vs, o_out, os_)

    def backward(self, do, dq_out, dk_out, dv_out):
        """Gradients of the last forward()."""
        s = self.shape
        if self._kept is None:
            raise ValueError("RangeAttention: backward() follows a forward() under the same ranges, of an object made with_backward")
        do, dos = self._tensor(do, s.Sq, s.heads, "do")
        _, dqs = self._tensor(dq_out, s.Sq, s.heads, "dq_out", True)
        _, dks = self._tensor(dk_out, s.Sk, s.kv_heads, "dk_out", True)
        _, dvs = self._tensor(dv_out, s.Sk, s.kv_heads, "dv_out", True)
        with _on(self.device):
            vb.vmoba_range_attn_bwd(s, self.plan, *self._kept, self.o_resid, self.lse, do, dos, dq_out, dqs, dk_out, dks, dv_out, dvs,
                                    self.dev_status, self.ws)

    def check_status(self):
        code = int(self.dev_status.item())
        if code != vb.OK:
            raise vb.VmobaError(code, "device status")


def lists_from_mask(mask_bh, capacity=None, device="cuda"):
    """Builds kb_ptr / q_idx / q_ptr / q_pairs on the host from a boolean mask [BH, S, Nb]
    (used by tests to feed the attention kernels a selection that did not come from
    vmoba_select).  Pure index bookkeeping."""
    import numpy as np
    BH, S, Nb = mask_bh.shape
    kb_ptr = [0]
    q_idx = []
    pos_of = {}
    for bh in range(BH):
        for j in range(Nb):
            qs = np.nonzero(mask_bh[bh, :, j])[0]
            base = len(q_idx)
            for n, qq in enumerate(qs):
                pos_of[(bh, int(qq), j)] = base + n
            q_idx.extend(qs.tolist())
            kb_ptr.append(len(q_idx))
    q_ptr = [0]
    q_pairs = []
    for bh in range(BH):
        for qq in range(S):
            for j in np.nonzero(mask_bh[bh, qq])[0]:
                q_pairs.append(pos_of[(bh, qq, int(j))])
            q_ptr.append(len(q_pairs))
    n = len(q_idx)
    cap = max(n, 1) if capacity is None else capacity
    pad = lambda a: a + [0] * (cap - len(a))
    mk = lambda a: torch.tensor(a, dtype=torch.int32, device=device)
    return mk(kb_ptr), mk(pad(q_idx)), mk(q_ptr), mk(pad(q_pairs)), n
