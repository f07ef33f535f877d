"""Other key ranges between a forward and its backward."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import key_ranges
from tests import _plain64 as P
from tests.test_gpu_range_attn import check_all, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_backward_after_set_ranges_asks_for_a_forward(dtype, d):
    """What the forward left (lse, o) belongs to the ranges it ran under."""
    first, second = (key_ranges(n, n_tokens=200, frame=1, device="cpu") for n in ([90, 60], [120, 80]))
    shape, op, host, dev, place = make(1, 200, 200, 2, 1, d, dtype, first, seed=3)
    o, grads = torch.empty_like(dev[0]), [torch.full_like(x, 4.0) for x in dev[:3]]
    op.forward(*dev[:3], o)
    op.set_ranges(second.cuda())
    before = vb.kernel_launches()
    with pytest.raises(ValueError):
        op.backward(dev[3], *grads)
    assert vb.kernel_launches() == before and all(bool((x == 4).all()) for x in grads)
    op.forward(*dev[:3], o)
    op.backward(dev[3], *grads)
    op.check_status()
    check_all(P.range_attention(*host[:3], second, do=host[3]), dtype, d, 0.0, o, op.lse, grads)


def test_ranges_anywhere_in_a_buffer():
    """Views that begin on an odd word, and ones that are not contiguous, are taken as any other."""
    first, second = (key_ranges(n, n_tokens=200, frame=1, device="cpu") for n in ([90, 60], [120, 80]))
    shape, op, host, dev, place = make(1, 200, 200, 2, 1, 64, "f32", first, seed=3)
    odd = torch.zeros(2 * 200 + 1, dtype=torch.int32, device="cuda")[1:].view(1, 200, 2)
    wide = torch.zeros((1, 200, 5), dtype=torch.int32, device="cuda")[..., 1:3]
    for view in (odd, wide):
        view.copy_(second)
        op.set_ranges(view)
        o = torch.empty_like(dev[0])
        op.forward(*dev[:3], o)
        op.check_status()
        check_all(P.range_attention(*host[:3], second), "f32", 64, 0.0, o, op.lse)
        op.set_ranges(first.cuda())
