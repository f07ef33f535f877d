"""Caps at the ends of their range.  Tolerances: test_gpu_range_attn.py (the share of a capped score's error that goes by the cap goes by the
score where the cap is not reached)."""
import math

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import RangeAttention, key_ranges
from tests import _plain64 as P
from tests.test_gpu_range_attn import DT, KINDS, check, check_all, make, run

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


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap,scale", [(1e6, 0.0), (1e5, 100.0), (2e3, 1.0)])
def test_rows_that_reach_a_large_cap_leave_the_others_exact(cap, scale, kind):
    """One query in twenty has scores of the size of the cap; those of the others are of the size of one, and so is what may be wrong with them.
    (The large ones get no gradient, so that dk and dv are sums over the others.)"""
    dtype, d = kind
    S = 260
    s = scale or d ** -0.5
    g = torch.Generator().manual_seed(17)
    mk = lambda n: torch.randn((1, S, n, d), generator=g)
    q, k, v, do = mk(2) / (s * math.sqrt(d)) / 64, mk(1) * 64, mk(1), mk(2)
    large = torch.arange(S) % 20 == 3
    big = q.clone()
    big[:, large] *= cap
    q[:, large] = 0
    do[:, large] = 0
    q, big, k, v, do = (x.to(DT[dtype]) for x in (q, big, k, v, do))
    ranges = key_ranges([S], n_tokens=S, device="cpu")
    ref = P.range_attention(q, k, v, ranges, cap, scale=scale or None, do=do)
    far = P.range_attention(big, k, v, ranges, cap, scale=scale or None)
    assert ref["top"] < 40 and float(far["lse"][..., large].max()) > 0.8 * cap
    op = RangeAttention(vb.make_range_shape(1, 2, 1, d, S, S, dtype, softmax_scale=scale, softcap=cap), ranges.cuda(), with_backward=True)
    dev = [x.cuda() for x in (big, k, v, do)]
    o, grads = run(op, dev, lambda x: x.cuda(), (big, k, v, do))
    lse = op.lse.cpu()
    assert bool(((lse - far["lse"])[..., large].abs() <= 1e-5 * cap).all())
    # the rows of the large ones as the statement without them has them: what is compared is the others
    o, dq, lse = o.cpu(), grads[0].cpu(), lse
    o[:, large] = ref["o"][:, large].to(o.dtype)
    dq[:, large] = ref["dq"][:, large].to(o.dtype)
    lse[..., large] = ref["lse"][..., large].float()
    check_all(ref, dtype, d, ref["top"], o, lse, [dq, grads[1], grads[2]])


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap", [44.0, 50.0, 55.0, 58.0, 66.0])
@pytest.mark.parametrize("sign,size", [(1, 1e8), (-1, 1e-6)])
def test_all_scores_at_the_cap_and_large_or_small_values(sign, size, cap, kind):
    """Every score of a row at the cap's one end, so that no weight is small against the others: sums of thousands of them times values of
    10^8 are in fp32's range whatever stands for the row's maximum."""
    dtype, d = kind
    Sq, Sk = 70, 4100
    ranges = key_ranges([Sk], n_queries=Sq, device="cpu")
    g = torch.Generator().manual_seed(23)
    mk = lambda S, n: torch.randn((1, S, n, d), generator=g)
    u = torch.randn(d, generator=g)
    u *= math.sqrt(8.0 * cap * math.sqrt(d)) / u.norm()
    host = [(sign * u + 0.05 * mk(Sq, 2)).to(DT[dtype]), (u + 0.05 * mk(Sk, 1)).to(DT[dtype]),
            (size * (1 + 0.1 * mk(Sk, 1))).to(DT[dtype]), (mk(Sq, 2) / size).to(DT[dtype])]
    ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
    op = RangeAttention(vb.make_range_shape(1, 2, 1, d, Sq, Sk, dtype, softcap=cap), ranges.cuda(), with_backward=True)
    o, grads = run(op, [x.cuda() for x in host], lambda x: x.cuda(), host)
    assert all(bool(torch.isfinite(x).all()) for x in [o, op.lse] + grads)
    check_all(ref, dtype, d, cap, o, op.lse)
    # (slopes are 0 to 2^-21 here, and so is what dq and dk are relative to dv's magnitudes: what they are is the slopes' rounding)
    check(grads[2], ref["dv"], ref["dv_mag"], 4 * (4 * math.sqrt(d) * 2.0 ** -24 * ref["top"] + 3e-7 * cap + 2e-5) + (2.0 ** -8 if dtype == "bf16" else 0), "dv")


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap", [0.3, 5.0, 27.0, 300.0])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_far_beyond_the_cap_have_no_gradient(sign, cap, kind):
    """From 9 caps on tanh is 1 to half a step of fp32 (2 exp(-18) < 2^-25) and its slope 0; dq and dk are sums of what it multiplies."""
    dtype, d = kind
    ranges = key_ranges([130, 90], n_tokens=230, frame=1, device="cpu")
    g = torch.Generator().manual_seed(24)
    mk = lambda n: torch.randn((1, 230, n, d), generator=g)
    u = torch.randn(d, generator=g)
    u *= math.sqrt(20.0 * cap * math.sqrt(d)) / u.norm()
    s = 0.05 * u.norm() / math.sqrt(d)
    host = [(sign * u + s * mk(2)).to(DT[dtype]), (u + s * mk(1)).to(DT[dtype]), mk(1).to(DT[dtype]), mk(2).to(DT[dtype])]
    ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
    op = RangeAttention(vb.make_range_shape(1, 2, 1, d, 230, 230, dtype, softcap=cap), ranges.cuda(), with_backward=True)
    o, grads = run(op, [x.cuda() for x in host], lambda x: x.cuda(), host)
    assert float(ref["dq"].abs().max()) < 1e-9 and float(ref["dk"].abs().max()) < 1e-9
    assert bool((grads[0] == 0).all()) and bool((grads[1] == 0).all())
    check_all(ref, dtype, d, cap, o, op.lse)
    check(grads[2], ref["dv"], ref["dv_mag"], 4 * (4 * math.sqrt(d) * 2.0 ** -24 * ref["top"] + 3e-7 * cap + 2e-5) + (2.0 ** -8 if dtype == "bf16" else 0), "dv")
