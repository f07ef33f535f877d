"""Rows of 2^31 bytes and more are refused (vectors of a row are counted in 32 bits): no kernel is launched."""
import ctypes

import pytest

from paper_2506_23858_b200 import binding as vb

FAKE = 0x1000        # aligned, never dereferenced: the checks come first


@pytest.mark.parametrize("heads,d,dtype,ok", [(2 ** 22, 128, "f32", False), (2 ** 22 - 1, 128, "f32", True), (2 ** 23, 128, "bf16", False),
                                              (2 ** 24, 64, "bf16", False), (2 ** 22, 64, "f32", True)])
@pytest.mark.parametrize("norm", [vb.ROTARY_NORM_NONE, vb.ROTARY_NORM_ROW])
def test_longest_row(heads, d, dtype, ok, norm):
    shape = vb.make_shape(1, heads, d, (1, 1, 2), (1, 1, 2), dtype)
    spec = vb.RotarySpec(pairs=32, axes=1, layout=vb.ROTARY_HALF, norm=norm, pos_batch=1, mscale=1.0, eps=1e-6)
    need = vb.rotary_workspace_bytes(shape, spec, 1)
    assert (need > 0) == ok
    one, st = (ctypes.c_void_p * 1)(FAKE), (ctypes.c_int64 * 3)(2 * heads * d, heads * d, d)
    if ok:
        return
    call = (ctypes.byref(shape), ctypes.byref(spec), 1)
    assert vb.lib().vmoba_rotary(*call, 1, one, st, one, st, None, FAKE, FAKE, FAKE, None, None) == vb.ERR_SHAPE
    assert vb.lib().vmoba_rotary_bwd(*call, one, st, one, st, None, one, st, None, FAKE, FAKE, FAKE, FAKE, 1 << 50, None) == vb.ERR_SHAPE
