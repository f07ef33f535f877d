"""Attention over key ranges without a GPU: the helper that makes ranges, the 64-bit statement the GPU tests compare with (against a second
one and against differences), and the entry points' refusals (no kernel is launched)."""
import ctypes
import math

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import key_ranges
from tests import _plain64 as P


def _seen(r, Sk):
    key = torch.arange(Sk)
    return (key >= r[..., :1]) & (key < r[..., 1:])


def test_ranges_of_packed_clips():
    r = key_ranges([3, 0, 2], n_tokens=7, device="cpu")
    assert r.dtype == torch.int32 and r.tolist() == [[[0, 3]] * 3 + [[3, 5]] * 2 + [[0, 0]] * 2]
    assert key_ranges([3, 2], n_tokens=5, frame=1, device="cpu").tolist() == [[[0, 1], [0, 2], [0, 3], [3, 4], [3, 5]]]
    assert key_ranges([5], n_tokens=5, frame=2, prefix=3, device="cpu").tolist() == [[[0, 3], [0, 3], [0, 4], [0, 4], [0, 5]]]
    assert key_ranges([5], n_tokens=5, frame=1, window=2, device="cpu").tolist() == [[[0, 1], [0, 2], [1, 3], [2, 4], [3, 5]]]
    assert key_ranges([0], n_tokens=2, device="cpu").tolist() == [[[0, 0], [0, 0]]]


def test_ranges_of_caches():
    r = key_ranges([4, 1], n_queries=2, frame=1, device="cpu")
    assert r.tolist() == [[[0, 3], [0, 4]], [[0, 0], [0, 1]]]        # a sample shorter than the queries: its first one is none
    assert key_ranges([6], n_queries=1, window=4, device="cpu").tolist() == [[[2, 6]]]
    for bad in (dict(lens=[3], n_tokens=2), dict(lens=[3]), dict(lens=[], n_tokens=2), dict(lens=[-1], n_tokens=2),
                dict(lens=[3], n_tokens=4, n_queries=1), dict(lens=[3], n_tokens=4, frame=-1)):
        with pytest.raises(ValueError):
            key_ranges(device="cpu", **bad)


@pytest.mark.parametrize("cap", [0.0, 5.0])
def test_statement_against_autograd_and_differences(cap):
    g = torch.Generator().manual_seed(3)
    r_ = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    B, Sq, Sk, h, hk, d = 2, 6, 9, 4, 2, 64
    q, k, v, do = r_(B, Sq, h, d) * 3, r_(B, Sk, hk, d), r_(B, Sk, hk, d), r_(B, Sq, h, d)
    ranges = torch.tensor([[[0, 9], [2, 3], [4, 4], [-5, 7], [8, 30], [5, 2]]], dtype=torch.int32)
    ref = P.range_attention(q, k, v, ranges, cap, do=do)
    assert torch.isinf(ref["lse"][:, :, [2, 5]]).all() and torch.isfinite(ref["lse"][:, :, [0, 1, 3, 4]]).all()
    assert (ref["o"][:, [2, 5]] == 0).all() and (ref["dq"][:, [2, 5]] == 0).all()
    x = [t.clone().requires_grad_() for t in (q, k, v)]
    kk, vv = (t.repeat_interleave(h // hk, 2) for t in x[1:])
    s = torch.einsum("bihd,bjhd->bhij", x[0], kk) / math.sqrt(d)
    s = cap * torch.tanh(s / cap) if cap else s
    seen = _seen(ranges.long(), Sk)[:, None]
    w = torch.softmax(torch.where(seen, s, torch.tensor(-1e30, dtype=s.dtype)), -1) * seen
    o = torch.einsum("bhij,bjhd->bihd", w, vv)
    assert torch.allclose(o, ref["o"], atol=1e-12)
    for a, b in zip(torch.autograd.grad(o, x, do), (ref["dq"], ref["dk"], ref["dv"])):
        assert torch.allclose(a, b, atol=1e-12)
    u, e = r_(B, Sk, hk, d), 1e-5
    val = lambda k: (P.range_attention(q, k, v, ranges, cap)["o"] * do).sum()
    assert abs((val(k + e * u) - val(k - e * u)) / (2 * e) - (ref["dk"] * u).sum()) < 1e-7 * (ref["dk"] * u).abs().sum()


FAKE = 0x1000        # aligned, never dereferenced: the checks come first


def _shape(**kw):
    return vb.make_range_shape(**{**dict(B=2, heads=4, kv_heads=2, head_dim=64, Sq=8, Sk=16, dtype="f32"), **kw})


BAD_SHAPES = [(dict(B=0), vb.ERR_SHAPE), (dict(Sq=0), vb.ERR_SHAPE), (dict(Sk=0), vb.ERR_SHAPE), (dict(Sk=-4), vb.ERR_SHAPE),
              (dict(heads=3), vb.ERR_SHAPE), (dict(heads=130, kv_heads=2), vb.ERR_SHAPE), (dict(kv_heads=0), vb.ERR_SHAPE),
              (dict(head_dim=96), vb.ERR_SHAPE), (dict(mask_batch=3), vb.ERR_SHAPE), (dict(dtype=5), vb.ERR_ARG),
              (dict(softmax_scale=-1.0), vb.ERR_ARG), (dict(softcap=float("nan")), vb.ERR_ARG), (dict(softcap=-2.0), vb.ERR_ARG),
              (dict(Sk=2 ** 30, B=8), vb.ERR_SHAPE)]


@pytest.mark.parametrize("i", range(len(BAD_SHAPES)))
def test_bad_shapes(i):
    kw, code = BAD_SHAPES[i]
    s = _shape(**kw)
    assert vb.range_plan_bytes(s) == 0 and vb.range_workspace_bytes(s) == 0 and vb.range_workspace_bytes(s, True) == 0
    assert vb.lib().vmoba_range_plan(ctypes.byref(s), FAKE, FAKE, 1 << 40, None) == code
    assert _fwd(s) == code and _bwd(s) == code


def _st(x):
    return (ctypes.c_int64 * 3)(*x) if x is not None else None


QS, KS = (8 * 4 * 64, 4 * 64, 64), (16 * 2 * 64, 2 * 64, 64)


def _fwd(s, plan=FAKE, q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, status=FAKE, ws=FAKE, size=1 << 40, resid=None, qs=QS, ks=KS, vs=KS, os_=QS):
    return vb.lib().vmoba_range_attn_fwd(ctypes.byref(s), plan, q, _st(qs), k, _st(ks), v, _st(vs), o, _st(os_), resid, lse, status, ws, size, None)


def _bwd(s, plan=FAKE, q=FAKE, o=FAKE, lse=FAKE, do=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, size=1 << 40, dos=QS, dqs=QS, dks=KS, dvs=KS):
    return vb.lib().vmoba_range_attn_bwd(ctypes.byref(s), plan, q, _st(QS), FAKE, _st(KS), FAKE, _st(KS), o, _st(QS), None, lse, do, _st(dos), dq,
                                         _st(dqs), dk, _st(dks), dv, _st(dvs), FAKE, ws, size, None)


def test_refusals():
    s = _shape()
    for kw in ([{n: None} for n in ("plan", "q", "k", "v", "o", "lse", "status", "ws", "qs", "os_")]
               + [{n: 0x1008} for n in ("plan", "q", "k", "v", "o", "ws", "resid")]
               + [dict(qs=(1, 64, 64)), dict(ks=(2048, 0, 64)), dict(vs=(2048, 128, 66)), dict(os_=(2048, -256, 64)), dict(qs=(2048, 256, 32))]):
        assert _fwd(s, **kw) == vb.ERR_ARG, kw
    for kw in ([{n: None} for n in ("plan", "q", "o", "lse", "do", "dq", "dk", "dv", "ws", "dos", "dqs", "dks", "dvs")]
               + [{n: 0x1008} for n in ("do", "dq", "dk", "dv", "ws")] + [dict(dks=(2048, 64, 0))]):
        assert _bwd(s, **kw) == vb.ERR_ARG, kw
    assert _fwd(s, size=vb.range_workspace_bytes(s) - 1) == vb.ERR_WORKSPACE
    assert _bwd(s, size=vb.range_workspace_bytes(s, True) - 1) == vb.ERR_WORKSPACE
    need = vb.range_plan_bytes(s)
    assert need > 0 and vb.lib().vmoba_range_plan(ctypes.byref(s), FAKE, FAKE, need - 1, None) == vb.ERR_WORKSPACE
    for key_range, plan in ((None, FAKE), (FAKE, None), (0x1004, FAKE), (FAKE, 0x1008)):
        assert vb.lib().vmoba_range_plan(ctypes.byref(s), key_range, plan, need, None) == vb.ERR_ARG
    assert vb.lib().vmoba_range_workspace_bytes(ctypes.byref(s), 2) == 0


def test_scratch_is_a_function_of_the_shape():
    long = _shape(B=1, heads=12, kv_heads=4, head_dim=128, Sq=1, Sk=75600, dtype="bf16")
    assert vb.range_workspace_bytes(long) > 12 * 128 * 4 * 2          # a long cache and one token: split over the SMs
    assert vb.range_workspace_bytes(_shape(B=1, heads=12, kv_heads=12, head_dim=128, Sq=32760, Sk=32760, dtype="bf16")) == 256
