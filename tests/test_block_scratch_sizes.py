"""Scratch of the smallest linear layers and feed-forward blocks, without a GPU: 256 bytes are stated where a call uses none of them, and only there, since
calls under way at the same time on one object are then given the same."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import FeedForward, Linear

L = vb.make_linear_shape


def of(cls):
    """An object of the class as far as its scratch goes, on the CPU."""
    op = cls.__new__(cls)
    op.device, op._nothing = torch.device("cpu"), torch.empty(256, dtype=torch.uint8)
    return op


@pytest.mark.parametrize("rows,hidden,dtype", [(1, 8, "bf16"), (1, 128, "bf16"), (16, 8, "bf16"), (2, 64, "bf16"), (1, 64, "f32"), (8, 8, "f32"), (1, 136, "bf16")])
def test_h_of_a_feed_forward_block_is_the_calls_own(rows, hidden, dtype):
    n = vb.ffn_workspace_bytes(L(1, rows, 1536, hidden, dtype, "gelu"))
    assert n > 256 and n >= rows * hidden * (2 if dtype == "bf16" else 4)
    op = of(FeedForward)
    a, b = op._scratch(n), op._scratch(n)
    assert a.numel() >= n and a.data_ptr() != b.data_ptr()


def test_partial_sums_of_a_linear_layer_are_the_calls_own():
    # one token: a slice for every 128 of the summed indices
    for K in (256, 512, 1024):
        n = vb.linear_workspace_bytes(L(1, 1, K, 8, "f32"))
        assert n > 256, K
        op = of(Linear)
        assert op._scratch(n).data_ptr() != op._scratch(n).data_ptr()
    for s in (L(1, 1, 8, 8, "bf16"), L(1, 1, 8, 8, "f32"), L(4, 4, 64, 8, "bf16", "gelu", True)):
        assert vb.linear_workspace_bytes(s, True) > 256


def test_calls_without_scratch_take_no_memory():
    op = of(Linear)
    for s in (L(1, 1, 1536, 9216, "bf16"), L(1, 4096, 1536, 4608, "bf16"), L(1, 1, 64, 8, "f32")):
        n = vb.linear_workspace_bytes(s)
        assert n == 256 and op._scratch(n) is op._nothing
