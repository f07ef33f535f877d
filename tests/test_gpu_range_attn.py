"""Attention over key ranges on the GPU against the 64-bit statement.

Tolerances.  A score is a sum of d products in 32 bits: its error stays within 4 sqrt(d) 2^-24 |q| |k| scale (roundings of partial sums no larger
than |q| |k|, four deviations of their random walk); a capped score adds 3e-7 of the cap (exponential, reciprocal and two roundings near
1).  Call that e: a weight is then off by e relative, and a sum of weights times values by e of the sum of magnitudes, twice for o, which
is divided by another such sum.  Sums over the keys are of 64 to 128 terms inside a tile and of as many partial sums as there are tiles (at
most 64 here): 2e-5 of the magnitudes on top.  fp32: that is all.  bf16 on the tensor cores: weights, and dS = P (dP - D), are rounded once to
bf16 ahead of the second product, half a step 2^-8 each: o 2 * 2^-8 (numerator and denominator) of its magnitudes, dv 2^-8, dq and dk 2^-8 for
dS and 2^-7 for the D that is made of that o: 3 * 2^-8.  Every result is rounded to its type once more: finfo.eps / 2 of it."""
import math

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import RangeAttention, Rotary, key_ranges, rotary_frequencies
from tests import _plain64 as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def check(got, ref, mag, rel, what):
    half = torch.finfo(got.dtype).eps / 2
    err = (got.detach().double().cpu() - ref).abs()
    tol = half * ref.abs() + rel * (1 + half) * mag + 1e-30
    assert bool((err <= tol).all()), f"{what}: {err.max():.3e} off, {(err / tol).max():.2f} of its tolerance"


def check_all(ref, dtype, d, cap, o, lse, grads=None):
    e = 4 * math.sqrt(d) * 2.0 ** -24 * ref["top"] + 3e-7 * cap + 2e-5
    bf = 2.0 ** -8 if dtype == "bf16" else 0.0
    check(o, ref["o"], ref["o_mag"], 2 * e + 2 * bf, "o")
    lse, want = lse.double().cpu(), ref["lse"]
    assert torch.equal(torch.isinf(lse), torch.isinf(want)) and not torch.isnan(lse).any()
    some = torch.isfinite(want)
    assert bool(((lse - want)[some].abs() <= 2 * e + 2.0 ** -22 * want[some].abs()).all()), f"lse {(lse - want)[some].abs().max()}"
    for g, n in zip(grads or (), ("dq", "dk", "dv")):
        check(g, ref[n], ref[n + "_mag"], 4 * e + (bf if n == "dv" else 3 * bf), n)


def random_ranges(Bm, Sq, Sk, g):
    """Any ranges: empty ones, ones that stick out at both ends, single keys."""
    a, b = (torch.randint(-20, Sk + 20, (Bm, Sq), generator=g) for _ in range(2))
    r = torch.stack([torch.minimum(a, b), torch.maximum(a, b)], -1)
    kind = torch.randint(0, 6, (Bm, Sq), generator=g)
    r[..., 1] = torch.where(kind == 0, r[..., 0], r[..., 1])
    r[..., 1] = torch.where(kind == 1, r[..., 0] + 1, r[..., 1])
    r = torch.where((kind == 2)[..., None], r.flip(-1), r)
    return r.to(torch.int32)


def make(B, Sq, Sk, h, hk, d, dtype, ranges, cap=0.0, layout="raster", seed=0, gain=1.0, backward=True):
    g = torch.Generator().manual_seed(seed)
    mk = lambda S, n: torch.randn((B, S, n, d), generator=g).to(DT[dtype])
    q, k, v, do = mk(Sq, h) * gain, mk(Sk, hk), mk(Sk, hk), mk(Sq, h)
    shape = vb.make_range_shape(B, h, hk, d, Sq, Sk, dtype, mask_batch=ranges.shape[0], softcap=cap)

    def place(x):
        if layout == "raster":
            return x.cuda()
        if layout == "heads":          # [B, heads, S, d] in memory
            return x.transpose(1, 2).contiguous().cuda().transpose(1, 2)
        big = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + 2, 2 * d), 9.0, dtype=x.dtype).cuda()
        view = big[:, 1:, 1:-1, d:]
        view.copy_(x)
        return view

    return shape, RangeAttention(shape, ranges.cuda(), with_backward=backward), (q, k, v, do), [place(x) for x in (q, k, v, do)], place


def run(op, dev, place, like):
    q, k, v, do = dev
    o = place(torch.full_like(like[0], 5.0))
    op.forward(q, k, v, o)
    grads = [place(torch.full_like(x, 5.0)) for x in like[:3]]
    op.backward(do, *grads)
    op.check_status()
    return o, grads


KINDS = [("f32", 64), ("f32", 128), ("bf16", 64), ("bf16", 128)]
G0 = torch.Generator().manual_seed(77)
CASES = [
    # B, Sq, Sk, heads, key heads, ranges, cap, layout
    dict(B=1, Sq=1, Sk=1, h=1, hk=1, r=lambda: key_ranges([1], n_tokens=1, device="cpu")),
    dict(B=2, Sq=2, Sk=2, h=3, hk=1, r=lambda: key_ranges([1, 1], n_tokens=2, device="cpu"), cap=10.0),
    dict(B=1, Sq=63, Sk=63, h=2, hk=2, r=lambda: key_ranges([63], n_tokens=63, frame=1, device="cpu")),
    dict(B=1, Sq=128, Sk=128, h=2, hk=2, r=lambda: key_ranges([128], n_tokens=128, device="cpu"), layout="heads"),
    dict(B=2, Sq=129, Sk=129, h=4, hk=2, r=lambda: key_ranges([50, 0, 1, 70], n_tokens=129, device="cpu"), layout="slices", cap=3.0),
    dict(B=1, Sq=257, Sk=257, h=5, hk=1, r=lambda: key_ranges([257], n_tokens=257, frame=1, device="cpu")),
    dict(B=1, Sq=300, Sk=300, h=3, hk=1, r=lambda: key_ranges([100, 200], n_tokens=300, frame=30, prefix=70, device="cpu"), cap=8.0, layout="heads"),
    dict(B=1, Sq=513, Sk=513, h=1, hk=1, r=lambda: key_ranges([200, 113, 128], n_tokens=513, device="cpu")),
    dict(B=1, Sq=640, Sk=640, h=2, hk=2, r=lambda: key_ranges([640], n_tokens=640, frame=1, window=37, device="cpu")),
    dict(B=2, Sq=385, Sk=385, h=2, hk=1, r=lambda: random_ranges(2, 385, 385, G0)),
    dict(B=3, Sq=70, Sk=450, h=6, hk=2, r=lambda: random_ranges(1, 70, 450, G0), cap=5.0, layout="slices"),
    dict(B=2, Sq=64, Sk=64, h=2, hk=2, r=lambda: torch.zeros((2, 64, 2), dtype=torch.int32)),
    dict(B=3, Sq=1, Sk=1000, h=4, hk=2, r=lambda: key_ranges([1000, 3, 517], n_queries=1, device="cpu")),
    dict(B=1, Sq=1, Sk=3001, h=8, hk=1, r=lambda: key_ranges([2999], n_queries=1, window=2222, device="cpu"), cap=20.0),
    dict(B=2, Sq=5, Sk=4100, h=3, hk=3, r=lambda: key_ranges([4100, 2], n_queries=5, frame=1, device="cpu")),
    dict(B=1, Sq=140, Sk=2500, h=2, hk=2, r=lambda: key_ranges([2400], n_queries=140, frame=1, device="cpu"), layout="heads"),
    dict(B=1, Sq=2000, Sk=40, h=2, hk=1, r=lambda: random_ranges(1, 2000, 40, G0)),
    dict(B=1, Sq=900, Sk=900, h=64, hk=1, r=lambda: key_ranges([900], n_tokens=900, frame=300, device="cpu")),
]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("i", range(len(CASES)))
def test_against_the_statement(i, kind):
    c = CASES[i]
    dtype, d = kind
    ranges, cap = c["r"](), c.get("cap", 0.0)
    shape, op, host, dev, place = make(c["B"], c["Sq"], c["Sk"], c["h"], c["hk"], d, dtype, ranges, cap, c.get("layout", "raster"), seed=i)
    ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
    o, grads = run(op, dev, place, host)
    check_all(ref, dtype, d, cap, o, op.lse, grads)
    # without the residual's buffer and the backward, and a second time: the same bits
    plain = RangeAttention(shape, ranges.cuda())
    o2 = place(torch.full_like(host[0], 5.0))
    plain.forward(*dev[:3], o2)
    assert torch.equal(o2, o) and torch.equal(plain.lse, op.lse)
    o3, grads3 = run(op, dev, place, host)
    assert torch.equal(o3, o) and all(torch.equal(a, b) for a, b in zip(grads, grads3))


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
def test_large_logits_and_rescaling(kind):
    """Scores of a hundred and more, growing along the keys, so that the running maximum moves on; with and without a cap."""
    dtype, d = kind
    for cap in (0.0, 15.0):
        ranges = key_ranges([700], n_tokens=700, frame=1, device="cpu")
        shape, op, host, dev, place = make(1, 700, 700, 2, 2, d, dtype, ranges, cap, seed=4, gain=10.0)
        host[1].mul_(torch.linspace(0.2, 3.0, 700)[None, :, None, None].to(host[1].dtype))
        dev[1].copy_(host[1])
        ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
        o, grads = run(op, dev, place, host)
        check_all(ref, dtype, d, cap, o, op.lse, grads)


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_nobody_sees_may_hold_anything(kind, bad):
    """Keys ahead of the first and behind the last range, and rows of q and do that see nothing."""
    dtype, d = kind
    for cap, hk in ((0.0, 2), (6.0, 1)):
        S, n = 333, 290
        ranges = key_ranges([150, n - 150], n_tokens=S, frame=1, device="cpu")
        ranges[0, :5] = 0
        ranges[..., 0].clamp_(min=7)
        ranges[..., 1] = torch.where(ranges[..., 1] > ranges[..., 0], ranges[..., 1], 0)
        empty = ranges[0, :, 1] <= ranges[0, :, 0]
        assert 40 <= int(empty.sum()) < 60
        shape, op, host, dev, place = make(2, S, S, 2, hk, d, dtype, ranges, cap, seed=8)
        for x in (host[0], host[3], dev[0], dev[3]):
            x[:, empty] = bad
        for x in (host[1], host[2], dev[1], dev[2]):
            x[:, :7] = bad
            x[:, n:] = bad
        ref = P.range_attention(*host[:3], ranges, cap, do=host[3])
        o, grads = run(op, dev, place, host)
        check_all(ref, dtype, d, cap, o, op.lse, grads)
        assert bool((o[:, empty] == 0).all()) and bool((grads[0][:, empty] == 0).all())
        for x in grads[1:]:
            assert bool((x[:, :7] == 0).all()) and bool((x[:, n:] == 0).all())
        # one token against a cache whose rest was never written
        cache = RangeAttention(vb.make_range_shape(2, 2, hk, d, 1, S, dtype, softcap=cap), torch.tensor([[[7, n]]], dtype=torch.int32, device="cuda"))
        q1, o1 = dev[0][:, 100:101], torch.empty_like(dev[0][:, 100:101])
        cache.forward(q1, dev[1], dev[2], o1)
        ref1 = P.range_attention(host[0][:, 100:101], host[1], host[2], torch.tensor([[[7, n]]]), cap)
        check_all(ref1, dtype, d, cap, o1, cache.lse)


@pytest.mark.parametrize("kind", [("f32", 64), ("bf16", 128)], ids=lambda k: f"{k[0]}_{k[1]}")
def test_a_query_that_is_not_finite_shows(kind):
    dtype, d = kind
    ranges = key_ranges([200], n_tokens=200, frame=1, device="cpu")
    shape, op, host, dev, place = make(1, 200, 200, 2, 2, d, dtype, ranges)
    clean = torch.empty_like(dev[0])
    op.forward(*dev[:3], clean)
    dev[0][0, 77, 1, 3] = float("nan")
    o = torch.empty_like(dev[0])
    op.forward(*dev[:3], o)
    assert torch.isnan(o[0, 77, 1]).all() and torch.isnan(op.lse[0, 1, 77])
    o[0, 77, 1] = clean[0, 77, 1]
    assert torch.equal(o, clean)


def test_full_ranges_equal_the_dense_path():
    """Every query sees every key: the same function as vmoba_full_attn."""
    for dtype, d in KINDS:
        ranges = torch.tensor([[[0, 320]] * 320], dtype=torch.int32)
        shape, op, host, dev, place = make(2, 320, 320, 3, 3, d, dtype, ranges, layout="heads")
        o, grads = run(op, dev, place, host)
        s = vb.make_shape(2, 3, d, (5, 8, 8), (5, 8, 8), dtype)
        q, k, v, do = (x.transpose(1, 2) for x in dev)
        assert q.is_contiguous()
        out = [torch.empty_like(q) for _ in range(4)]
        lse, status = torch.empty(2 * 3 * 320, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(vb.workspace_bytes(s, vb.STAGE_FULL_BWD), dtype=torch.uint8, device="cuda")
        vb.vmoba_full_attn(s, q, k, v, out[0], lse, do, *out[1:], status, ws)
        tol = 2.0 ** -6 if dtype == "bf16" else 2e-5
        for a, b in zip([o] + grads, out):
            a = a.transpose(1, 2).float()
            assert (a - b.float()).norm() <= tol * b.float().norm()
        assert (op.lse.reshape(-1) - lse).abs().max() < 1e-5


@pytest.mark.parametrize("kind", [("f32", 64), ("bf16", 128)], ids=lambda k: f"{k[0]}_{k[1]}")
def test_other_stream_and_captured_graphs(kind):
    """On another stream, and in two captured graphs of two objects, with an eager call in between, replayed with new inputs."""
    dtype, d = kind
    ranges = [key_ranges([150, 100], n_tokens=260, device="cpu"), key_ranges([260], n_tokens=260, frame=1, device="cpu")]
    made = [make(1, 260, 260, 2, 1, d, dtype, r, 12.0, seed=i) for i, r in enumerate(ranges)]
    want, bufs = [], []
    for shape, op, host, dev, place in made:
        o, grads = run(op, dev, place, host)
        want.append([x.clone() for x in [o, op.lse] + grads])
        bufs.append([torch.empty_like(o)] + [torch.empty_like(x) for x in grads])

    def both(i):
        shape, op, host, dev, place = made[i]
        op.forward(*dev[:3], bufs[i][0])
        op.backward(dev[3], *bufs[i][1:])

    def same(i):
        torch.cuda.synchronize()
        o, lse, *grads = want[i]
        assert torch.equal(bufs[i][0], o) and torch.equal(made[i][1].lse, lse) and all(torch.equal(a, b) for a, b in zip(bufs[i][1:], grads))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(0)
    same(0)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both(i)
        graphs.append(g)
    for i in (1, 0, 0, 1):
        for x in bufs[i]:
            x.fill_(3.0)
        graphs[i].replay()
        same(i)
        both(1 - i)
    # new inputs in the same buffers, and new ranges in the same plan
    shape, op, host, dev, place = made[0]
    for x in dev:
        x.copy_(torch.randn_like(x.float()).to(x.dtype))
    op.set_ranges(key_ranges([60, 190], n_tokens=260, frame=1, device="cuda"))
    both(0)
    torch.cuda.synchronize()
    keep = [x.clone() for x in bufs[0]]
    for x in bufs[0]:
        x.fill_(3.0)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(keep, bufs[0]))
    made[0][1].check_status()


def test_inputs_that_have_to_be_copied_and_refused_calls():
    ranges = key_ranges([100], n_tokens=100, device="cpu")
    shape, op, host, dev, place = make(1, 100, 100, 4, 2, 64, "f32", ranges)
    ref = P.range_attention(host[0], host[1][:, :, :1].expand(-1, -1, 2, -1), host[2], ranges, do=torch.ones_like(host[3]))
    o, grads = torch.empty_like(dev[0]), [torch.empty_like(x) for x in dev[:3]]
    v_odd = torch.empty(dev[2].numel() + 1, device="cuda")[1:].view(dev[2].shape)          # off the 16-byte grid
    v_odd.copy_(dev[2])
    op.forward(dev[0], dev[1][:, :, :1].expand(-1, -1, 2, -1), v_odd, o)
    op.backward(torch.ones((), device="cuda").expand(dev[0].shape), *grads)                # a sum's gradient
    check_all(ref, "f32", 64, 0.0, o, op.lse, grads)
    before = vb.kernel_launches()
    with pytest.raises(ValueError):
        op.forward(dev[0].bfloat16(), dev[1], dev[2], o)
    with pytest.raises(ValueError):
        op.forward(dev[0], dev[1][:, :50], dev[2], o)
    with pytest.raises(ValueError):
        op.forward(dev[0], dev[1], dev[2], o[:, :, :1].expand(-1, -1, 4, -1))
    with pytest.raises(ValueError):
        op.forward(host[0], dev[1], dev[2], o)
    with pytest.raises(ValueError):
        RangeAttention(shape, ranges.cuda()).backward(dev[3], *grads)
    with pytest.raises(ValueError):
        op.set_ranges(ranges.cuda().long())
    with pytest.raises(ValueError):
        RangeAttention(vb.make_range_shape(1, 3, 2, 64, 8, 8, "f32"), ranges.cuda())
    assert vb.kernel_launches() - before <= 2          # (the plan of the one valid object)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_norm_rotary_and_attention_on_packed_clips(dtype, d):
    """The path of a layer on packed clips: positions that restart with each clip, norm and rotation, attention inside the clips, and
    all of it backwards."""
    g = torch.Generator().manual_seed(21)
    B, h, grid, clips, cap = 2, 3, (5, 6, 8), [2, 1, 1], 9.0           # frames of 48 tokens; the fifth is padding
    S, per = 240, 48
    frame = torch.cat([torch.arange(n) for n in clips] + [torch.zeros(1, dtype=torch.int64)])
    t = frame.repeat_interleave(per)
    hw = torch.arange(S) % per
    pos = torch.stack([t, hw // 8, hw % 8], 1).to(torch.int32)
    f, axis, _ = rotary_frequencies((d // 2 - 2 * (d // 6), d // 6, d // 6))
    mk = lambda: torch.randn((B, S, h, d), generator=g).to(DT[dtype])
    q, k, v, do = mk(), mk(), mk(), mk()
    w = [1 + 0.2 * torch.randn(h * d, generator=g) for _ in range(2)]
    ranges = key_ranges([n * per for n in clips], n_tokens=S, frame=per, device="cpu")
    rot = Rotary(vb.make_shape(B, h, d, grid, (1, 6, 8), dtype), pos.cuda(), f.cuda(), axis.cuda(), norm="row", with_backward=True)
    att = RangeAttention(vb.make_range_shape(B, h, h, d, S, S, dtype, softcap=cap), ranges.cuda(), with_backward=True)
    qd, kd, vd, dod, wd = q.cuda(), k.cuda(), v.cuda(), do.cuda(), [x.cuda() for x in w]
    qr, kr, o = torch.empty_like(qd), torch.empty_like(kd), torch.empty_like(qd)
    rot.forward((qd, kd), (qr, kr), wd)
    att.forward(qr, kr, vd, o)
    dq, dk, dv = (torch.empty_like(qd) for _ in range(3))
    att.backward(dod, dq, dk, dv)
    dqr, dkr = dq.cpu(), dk.cpu()
    dw = rot.backward((dq, dk), (qd, kd), (dq, dk), wd)
    att.check_status()
    # each stage against the statement on what the stage before handed over
    for x, got, ww in ((q, qr, w[0]), (k, kr, w[1])):
        check(got, *P.norm_rotate(x, ww, pos, f, axis, "interleaved", "row"), 5e-6, "rotated")
    ref = P.range_attention(qr.cpu(), kr.cpu(), v, ranges, cap, do=do)
    check_all(ref, dtype, d, cap, o, att.lse, (dqr, dkr, dv))
    for x, gin, got, ww, gw in ((q, dqr, dq, w[0], dw[0]), (k, dkr, dk, w[1], dw[1])):
        (dx, mag), wref = P.norm_rotate_grad(gin, x, ww, pos, f, axis, "interleaved", "row")
        check(got, dx, mag, 5e-6, "dx")
        check(gw, *wref, 1.3e-5, "dw")
    assert bool((o[:, 192:] == 0).all()) and bool((dv[:, 192:] == 0).all())


@pytest.mark.parametrize("kind", [("bf16", 64), ("bf16", 128)], ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("i", [1, 4, 6, 10, 13])
def test_results_do_not_depend_on_what_ran_before(i, kind):
    """Between two runs others leave large scores and NaN in what registers, shared and tensor memory hold: units of fewer rows than a
    tile, tiles of fewer keys and groups that do not divide one keep their bits (how a capped score is worked out is a warp's choice)."""
    c = CASES[i]
    dtype, d = kind
    ranges, cap = c["r"](), 4.0
    shape, op, host, dev, place = make(c["B"], c["Sq"], c["Sk"], c["h"], c["hk"], d, dtype, ranges, cap, c.get("layout", "raster"), seed=i)
    full = torch.tensor([[[0, 640]] * 640], dtype=torch.int32)
    others = [make(2, 640, 640, 80, 80, d, dtype, full, cap, seed=50 + k, gain=g) for k, g in enumerate((100.0, float("nan")))]
    o, grads = run(op, dev, place, host)
    for _, other, oh, odev, oplace in others:
        run(other, odev, oplace, oh)
        o2, grads2 = run(op, dev, place, host)
        assert torch.equal(o2, o) and all(torch.equal(a, b) for a, b in zip(grads, grads2))


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("cap,scale", [(100.0, 0.0), (700.0, 0.0), (1e6, 0.0), (0.5, 0.0), (30.0, 2.0), (30.0, 1e-6), (0.0, 1.5)])
def test_caps_and_scales_far_from_the_usual(cap, scale, kind):
    """Caps that nothing reaches and caps that everything exceeds, scales other than head_dim^-1/2."""
    dtype, d = kind
    ranges = key_ranges([100, 111], n_tokens=230, frame=1, device="cpu")
    _, _, host, dev, place = make(2, 230, 230, 2, 1, d, dtype, ranges, seed=12)
    shape = vb.make_range_shape(2, 2, 1, d, 230, 230, dtype, softmax_scale=scale, softcap=cap)
    op = RangeAttention(shape, ranges.cuda(), with_backward=True)
    ref = P.range_attention(*host[:3], ranges, cap, scale=scale or None, do=host[3])
    o, grads = run(op, dev, place, host)
    # (the error of a capped score by the exponential is 3e-7 of the cap where the cap is reached; where it is not, of the score)
    check_all(ref, dtype, d, min(cap, ref["top"]), o, op.lse, grads)


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
def test_offsets_beyond_32_bits(dtype, d):
    """A cache whose last token lies more than 2^31 elements behind its first; gradients of the same layout."""
    Sq, Sk, apart = 3, 2200, 2 ** 20
    ranges = torch.tensor([[[0, 2200], [2100, 2200], [1, 2199]]], dtype=torch.int32)
    g = torch.Generator().manual_seed(3)
    mk = lambda S, n: torch.randn((1, S, n, d), generator=g).to(DT[dtype])
    q, k, v, do = mk(Sq, 2), mk(Sk, 1), mk(Sk, 1), mk(Sq, 2)
    big = torch.empty(Sk * apart, dtype=DT[dtype], device="cuda")
    k_far, v_far, dk, dv = [big.as_strided((1, Sk, 1, d), (Sk * apart, apart, d, 1), i * d) for i in range(4)]
    k_far.copy_(k)
    v_far.copy_(v)
    op = RangeAttention(vb.make_range_shape(1, 2, 1, d, Sq, Sk, dtype), ranges.cuda(), with_backward=True)
    o, dq = torch.empty_like(q, device="cuda"), torch.empty_like(q, device="cuda")
    op.forward(q.cuda(), k_far, v_far, o)
    op.backward(do.cuda(), dq, dk, dv)
    op.check_status()
    ref = P.range_attention(q, k, v, ranges, 0.0, do=do)
    check_all(ref, dtype, d, 0.0, o, op.lse, [dq, dk, dv])
    del big, k_far, v_far, dk, dv


@pytest.mark.parametrize("kind", [("f32", 64), ("bf16", 128)], ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("B,Sq,shared", [(3, 1, True), (3, 1, False), (1, 300, True), (3, 700, False)])
def test_a_captured_call_takes_new_ranges_of_a_growing_cache(B, Sq, shared, kind):
    """The pieces that a long cache is cut into follow from the ranges: one captured forward, replayed as the cache grows from nothing to its
    whole length, with samples that differ, against the statement; what lies behind a sequence does not matter."""
    dtype, d = kind
    Sk = 1500
    g = torch.Generator().manual_seed(21)
    mk = lambda S, n: torch.randn((B, S, n, d), generator=g).to(DT[dtype])
    q, k, v = mk(Sq, 2), mk(Sk, 1), mk(Sk, 1)
    dev = [x.cuda() for x in (q, k, v)]
    of = lambda n: key_ranges([n] if shared else [n, n // 3, max(n - 1, 0)], n_queries=Sq, device="cpu")
    op = RangeAttention(vb.make_range_shape(B, 2, 1, d, Sq, Sk, dtype, mask_batch=of(1).shape[0]), of(Sk).cuda())
    o = torch.empty_like(dev[0])
    op.forward(*dev, o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        op.forward(*dev, o)
    for n in (0, 1, 129, 1024, Sk):
        op.set_ranges(of(n).cuda())
        o.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        check_all(P.range_attention(q, k, v, of(n), 0.0), dtype, d, 0.0, o, op.lse)
    op.check_status()
