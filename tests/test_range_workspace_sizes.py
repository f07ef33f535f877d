"""Plans and scratch of range attention and rotary positions are functions of the shape alone: the same numbers without a GPU, on this one and on
another."""
import pytest

from paper_2506_23858_b200 import binding as vb

# (B, heads, key heads, head_dim, Sq, Sk, type, masks), bytes of the plan, of the forward's scratch, of the backward's
RANGES = [
    ((1, 12, 12, 128, 32760, 32760, 'bf16', 1), 275200, 256, 202862592),
    ((4, 12, 4, 128, 1, 75600, 'bf16', 4), 81152, 1585152, 99072),
    ((1, 12, 12, 128, 1560, 32760, 'bf16', 1), 23552, 144892928, 38416128),
    ((2, 2, 1, 64, 256, 256, 'f32', 1), 3328, 256, 4096),
    ((2, 3, 3, 128, 5, 4100, 'f32', 2), 7936, 990720, 256),
    ((1, 64, 1, 64, 900, 900, 'bf16', 1), 26624, 256, 230400),
    ((1, 132, 44, 128, 1600, 1600, 'bf16', 1), 14592, 256, 108986112),
]
# (B, heads, head_dim, grid, block, type), norm, bytes of the backward's scratch for one, two and four tensors
ROTARY = [
    ((1, 12, 128, (21, 30, 52), (3, 6, 13), 'bf16'), 0, [256, 256, 256]),
    ((1, 12, 128, (21, 30, 52), (3, 6, 13), 'bf16'), 1, [262144, 524288, 1048576]),
    ((1, 12, 128, (21, 30, 52), (3, 6, 13), 'bf16'), 2, [3145728, 6291456, 12582912]),
    ((1, 12, 128, (1, 1, 1), (1, 1, 1), 'bf16'), 0, [256, 256, 256]),
    ((1, 12, 128, (1, 1, 1), (1, 1, 1), 'bf16'), 1, [512, 1024, 2048]),
    ((1, 12, 128, (1, 1, 1), (1, 1, 1), 'bf16'), 2, [6144, 12288, 24576]),
    ((2, 5, 64, (5, 7, 11), (1, 7, 11), 'f32'), 0, [256, 256, 256]),
    ((2, 5, 64, (5, 7, 11), (1, 7, 11), 'f32'), 1, [131072, 262144, 524288]),
    ((2, 5, 64, (5, 7, 11), (1, 7, 11), 'f32'), 2, [655360, 1310720, 2621440]),
    ((1, 401, 128, (1, 30, 52), (1, 30, 52), 'bf16'), 0, [256, 256, 256]),
    ((1, 401, 128, (1, 30, 52), (1, 30, 52), 'bf16'), 1, [262144, 524288, 1048576]),
    ((1, 401, 128, (1, 30, 52), (1, 30, 52), 'bf16'), 2, [105119744, 210239488, 420478976]),
]


def _check():
    for (B, h, hk, d, Sq, Sk, dtype, masks), plan, fwd, bwd in RANGES:
        s = vb.make_range_shape(B, h, hk, d, Sq, Sk, dtype, mask_batch=masks)
        assert (vb.range_plan_bytes(s), vb.range_workspace_bytes(s), vb.range_workspace_bytes(s, True)) == (plan, fwd, bwd), (B, h, Sq, Sk)
    for args, norm, sizes in ROTARY:
        spec = vb.RotarySpec(pairs=32, axes=1, layout=vb.ROTARY_HALF, norm=norm, pos_batch=1, mscale=1.0, eps=1e-6)
        assert [vb.rotary_workspace_bytes(vb.make_shape(*args), spec, n) for n in (1, 2, 4)] == sizes, (args, norm)


def test_sizes_without_a_gpu():
    _check()


@pytest.mark.gpu
def test_sizes_on_a_gpu():
    import torch
    torch.zeros(1, device="cuda")
    _check()
