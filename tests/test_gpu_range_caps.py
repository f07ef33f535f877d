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
