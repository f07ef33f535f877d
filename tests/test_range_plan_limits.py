"""A plan of more masks than a grid is made for: refused ahead of every launch, by the size and by all entry points alike."""
import ctypes

from paper_2506_23858_b200 import binding as vb

FAKE = 0x1000        # aligned, never dereferenced: the checks come first


def test_more_masks_than_a_plan_takes():
    shape = lambda B, masks: vb.make_range_shape(B, 1, 1, 64, 1, 1, "f32", mask_batch=masks)
    most = 1 << 20
    assert vb.range_plan_bytes(shape(most, most)) > 0 and vb.range_plan_bytes(shape(most + 1, 1)) > 0
    s = shape(most + 1, most + 1)
    assert vb.range_plan_bytes(s) == 0 and vb.range_workspace_bytes(s) == 0 and vb.range_workspace_bytes(s, True) == 0
    before = vb.kernel_launches()
    assert vb.lib().vmoba_range_plan(ctypes.byref(s), FAKE, FAKE, 1 << 50, None) == vb.ERR_SHAPE
    st = (ctypes.c_int64 * 3)(64, 64, 64)
    assert vb.lib().vmoba_range_attn_fwd(ctypes.byref(s), FAKE, FAKE, st, FAKE, st, FAKE, st, FAKE, st, None, FAKE, FAKE, FAKE, 1 << 50, None) == vb.ERR_SHAPE
    assert vb.kernel_launches() == before
