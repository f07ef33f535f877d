"""Caps at the ends of their range.  Tolerances: test_gpu_range_attn.py (the share of a capped score's error that goes by the cap goes by the
score where the cap is not reached)."""
import math

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import RangeAttention, key_ranges
from tests import _plain64 as P
from tests.test_gpu_range_attn import DT, KINDS, check_all, make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap", [1e-3, 1e-5, 1e-12, 1e-25])
def test_small_caps(cap, kind):
    """Scores of the size of the cap: weights that are all but equal, slopes of every size."""
    dtype, d = kind
    ranges = key_ranges([100, 111], n_tokens=230, frame=1, device="cpu")
    shape, op, host, dev, place = make(2, 230, 230, 2, 1, d, dtype, ranges, cap, seed=14, gain=cap)
    ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
    o, grads = run(op, dev, place, host)
    assert all(bool(torch.isfinite(x).all()) for x in grads)
    check_all(ref, dtype, d, 0.0, o, op.lse, grads)


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap", [400.0, 3e3, 1e4])
def test_scores_of_hundreds_under_larger_caps(cap, kind):
    """All scores near 300, a few apart: an error of them that is the same for all does not show in the forward, whose weights add up to one
    whatever it is, and shows in full where the backward works the weights out again."""
    dtype, d = kind
    ranges = key_ranges([100, 70], n_tokens=190, frame=1, device="cpu")
    _, _, host, dev, place = make(1, 190, 190, 2, 1, d, dtype, ranges, seed=15)
    g = torch.Generator().manual_seed(16)
    u = torch.randn(d, generator=g)
    u *= math.sqrt(300.0 * math.sqrt(d)) / u.norm()
    host = [(u + 0 * host[0].float()).to(DT[dtype]), (u + 0.3 * host[1].float()).to(DT[dtype]), host[2], host[3]]
    dev = [x.cuda() for x in host]
    op = RangeAttention(vb.make_range_shape(1, 2, 1, d, 190, 190, dtype, softcap=cap), ranges.cuda(), with_backward=True)
    ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
    assert 280 < ref["top"] < 340
    o, grads = run(op, dev, lambda x: x.cuda(), host)
    check_all(ref, dtype, d, min(cap, ref["top"]), o, op.lse, grads)
