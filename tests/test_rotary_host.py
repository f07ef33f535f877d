"""Rotary positions without a GPU: the frequency tables, the 64-bit statement the GPU tests compare with (norms kept, relative positions,
gradients against differences) and the entry points' refusals (no kernel is launched)."""
import ctypes
import math

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import rotary_frequencies
from tests import _plain64 as P


def test_frequencies_of_every_scaling():
    f, axis, m = rotary_frequencies((22, 21, 21))
    assert f.dtype == torch.float64 and axis.dtype == torch.int32 and m == 1.0
    assert axis.tolist() == [0] * 22 + [1] * 21 + [2] * 21
    assert f[0] == f[22] == f[43] == 1.0 and math.isclose(f[23].item(), 10000.0 ** (-1 / 21))
    lin, _, _ = rotary_frequencies((64,), scaling="linear", factor=4.0)
    assert torch.equal(lin, rotary_frequencies((64,))[0] / 4.0)
    base, _, _ = rotary_frequencies((64,), scaling="base", factor=4.0)
    assert base[0] == 1.0 and math.isclose(base[-1].item(), lin[-1].item(), rel_tol=1e-12)      # the slowest pair is interpolated
    parts, _, m = rotary_frequencies((64,), scaling="parts", factor=4.0, trained=4096)
    assert parts[0] == 1.0 and parts[-1] == lin[-1] and math.isclose(m, 0.1 * math.log(4.0) + 1.0)
    assert torch.all(parts >= lin) and torch.all(parts <= rotary_frequencies((64,))[0])
    for bad in (dict(scaling="twice"), dict(factor=0.5), dict(theta=0.0)):
        with pytest.raises(ValueError):
            rotary_frequencies((8,), **bad)
    with pytest.raises(ValueError):
        rotary_frequencies((-1,))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_statement_keeps_lengths_and_relative_positions(layout):
    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn((1, 1, 1, 64), generator=g, dtype=torch.float64) for _ in range(2))
    f, axis, _ = rotary_frequencies((24,))
    at = lambda x, p: P.rotate(x, torch.tensor([[p]], dtype=torch.int32), f, axis, layout)[0]
    assert torch.allclose(at(q, 12345).norm(), q.norm(), rtol=1e-14, atol=0)
    assert torch.equal(at(q, 77)[..., 48:], q[..., 48:])
    a, b = (at(q, 1000) * at(k, 990)).sum(), (at(q, 17) * at(k, 7)).sum()
    assert abs(a - b) < 1e-10


@pytest.mark.parametrize("layout,norm", [("half", "none"), ("interleaved", "head"), ("half", "row")])
def test_statement_of_the_gradients_against_differences(layout, norm):
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    x, dy, u = r(2, 3, 2, 64), r(2, 3, 2, 64), r(2, 3, 2, 64)
    n = {"none": 0, "head": 64, "row": 128}[norm]
    w, uw = (1 + 0.2 * r(n), r(n)) if n else (None, None)
    f, axis, _ = rotary_frequencies((10, 7))
    pos = torch.randint(0, 50, (3, 2), generator=g, dtype=torch.int32)
    (dx, _), dw = P.norm_rotate_grad(dy, x, w, pos, f, axis, layout, norm, 1.3)
    h = 1e-5
    val = lambda x, w: (P.norm_rotate(x, w, pos, f, axis, layout, norm, 1.3)[0] * dy).sum()
    diff = (val(x + h * u, w) - val(x - h * u, w)) / (2 * h)
    assert abs(diff - (dx * u).sum()) < 1e-7 * (dx * u).abs().sum()
    if n:
        diff = (val(x, w + h * uw) - val(x, w - h * uw)) / (2 * h)
        assert abs(diff - (dw[0] * uw).sum()) < 1e-7 * (dw[0] * uw).abs().sum()


FAKE = 0x1000        # aligned, never dereferenced: the checks come first


def _call(shape=None, spec=None, n=1, turned=1, src=FAKE, dst=FAKE, src_strides=(1024, 128, 64), dst_strides=(1024, 128, 64), weight=None,
          pos=FAKE, freq=FAKE, axis=FAKE):
    shape = shape or vb.make_shape(1, 2, 64, (2, 2, 2), (1, 2, 2), "f32")
    spec = spec or _spec()
    arr = lambda v: (ctypes.c_void_p * max(n, 1))(*[v] * max(n, 1))
    st = lambda t: None if t is None else (ctypes.c_int64 * (3 * max(n, 1)))(*list(t) * max(n, 1))
    return vb.lib().vmoba_rotary(ctypes.byref(shape), ctypes.byref(spec), n, turned, arr(src), st(src_strides), arr(dst), st(dst_strides),
                                 arr(weight), pos, freq, axis, None, None)


def _spec(**kw):
    return vb.RotarySpec(**{**dict(pairs=32, axes=1, layout=vb.ROTARY_HALF, norm=vb.ROTARY_NORM_NONE, pos_batch=1, mscale=1.0, eps=1e-6), **kw})


def test_refusals_of_the_forward():
    E = vb
    for kw, code in ((dict(pairs=33), E.ERR_SHAPE), (dict(pairs=-1), E.ERR_SHAPE), (dict(axes=0), E.ERR_SHAPE), (dict(axes=5), E.ERR_SHAPE),
                     (dict(pos_batch=2), E.ERR_SHAPE), (dict(layout=2), E.ERR_ARG), (dict(norm=3), E.ERR_ARG), (dict(mscale=0.0), E.ERR_ARG),
                     (dict(mscale=float("nan")), E.ERR_ARG), (dict(eps=-1.0), E.ERR_ARG)):
        assert _call(spec=_spec(**kw)) == code, kw
    for kw in (dict(n=0), dict(n=5), dict(turned=2), dict(turned=-1), dict(src=0x1004), dict(dst=0x1008), dict(src=None), dict(dst=None),
               dict(src_strides=(1024, 128, 63)), dict(src_strides=(1024, -128, 64)), dict(dst_strides=(1024, 0, 64)),
               dict(dst_strides=(1024, 128, 32)), dict(pos=None), dict(freq=None), dict(axis=None),
               dict(spec=_spec(norm=1), weight=0x1004)):
        assert _call(**kw) == E.ERR_ARG, kw
    assert _call(shape=vb.make_shape(1, 2, 96, (2, 2, 2), (1, 2, 2), "f32")) == E.ERR_SHAPE


def test_refusals_and_scratch_of_the_backward():
    shape = vb.make_shape(1, 2, 64, (2, 2, 2), (1, 2, 2), "f32")
    one, st = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_int64 * 3)(1024, 128, 64)

    def call(spec, d_out=one, x=one, xs=st, dx=one, dxs=st, ws=FAKE, size=1 << 20, pos=FAKE):
        return vb.lib().vmoba_rotary_bwd(ctypes.byref(shape), ctypes.byref(spec), 1, d_out, st, x, xs, None, dx, dxs, None, pos, FAKE, FAKE, ws,
                                         size, None)

    row = _spec(norm=vb.ROTARY_NORM_ROW)
    need = vb.rotary_workspace_bytes(shape, row, 1)
    assert need >= 8 * 128 * 4
    assert call(row, size=need - 1) == vb.ERR_WORKSPACE
    for kw in (dict(x=None), dict(xs=None), dict(ws=None), dict(ws=0x1004), dict(d_out=None), dict(dx=None), dict(dxs=None), dict(pos=None)):
        assert call(row, **kw) == vb.ERR_ARG, kw
    assert call(_spec(norm=7)) == vb.ERR_ARG
    assert vb.rotary_workspace_bytes(shape, _spec(pairs=40), 1) == 0
    assert vb.rotary_workspace_bytes(shape, row, 0) == vb.rotary_workspace_bytes(shape, row, 5) == 0
    assert vb.rotary_workspace_bytes(shape, row, 2) >= 2 * 8 * 128 * 4
