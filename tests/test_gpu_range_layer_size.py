"""Range attention of as many heads and tokens as a layer has, on the tensor cores: one accumulator of dq for many key tiles, several groups of
heads, CTAs that take one item after another; compared head by head with the statement.  Tolerances: test_gpu_range_attn.py."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import RangeAttention, key_ranges
from tests import _plain64 as P
from tests.test_gpu_range_attn import check_all

pytestmark = pytest.mark.gpu
S, D = 1600, 128

CASES = {
    # heads, key heads, ranges, cap, key heads that are compared
    "clips": (132, 132, dict(lens=[700, 1, 499, 300]), 0.0, (0, 15, 16, 65, 66, 131)),
    "frames": (132, 132, dict(lens=[900, 650], frame=100, prefix=130), 0.0, (1, 17, 67, 130)),
    "causal_capped": (132, 132, dict(lens=[1600], frame=1), 30.0, (0, 15, 65, 66, 131)),
    "window": (131, 131, dict(lens=[1590], frame=1, window=333), 0.0, (0, 64, 130)),
    "groups_capped": (132, 44, dict(lens=[1000, 550], frame=50), 30.0, (0, 15, 16, 43)),
    "full_groups": (135, 27, dict(lens=[1600]), 0.0, (0, 16, 26)),
}


@pytest.mark.parametrize("name", CASES)
def test_heads_of_a_layer(name):
    h, hk, r, cap, sel = CASES[name]
    G = h // hk
    ranges = key_ranges(n_tokens=S, device="cpu", **r)
    shape = vb.make_range_shape(1, h, hk, D, S, S, "bf16", softcap=cap)
    one = h * S * D * 4
    assert one < vb.range_workspace_bytes(shape, True) < 2 * one and vb.range_workspace_bytes(shape) == 256
    g = torch.Generator(device="cuda").manual_seed(len(name))
    mk = lambda n: torch.randn((1, S, n, D), generator=g, device="cuda")
    # (capped: heads whose scores pass the polynomial's limit, 3/4 of the cap, in a few places, in many, in none)
    gain = torch.tensor([1.0, 9.0, 25.0, 0.1] if cap else [1.0, 3.0], device="cuda").repeat(h)[:h, None]
    q, k, v, do = (mk(h) * gain).bfloat16(), mk(hk).bfloat16(), mk(hk).bfloat16(), mk(h).bfloat16()
    op = RangeAttention(shape, ranges.cuda(), with_backward=True)

    def once():
        o, grads = torch.full_like(q, 5.0), [torch.full_like(x, 5.0) for x in (q, k, v)]
        op.forward(q, k, v, o)
        op.backward(do, *grads)
        op.check_status()
        return [o, op.lse.clone()] + grads

    got = once()
    for a, b in zip(got, once()):
        assert torch.equal(a, b)
    for j in sel:
        at = slice(j * G, (j + 1) * G)
        kv = slice(j, j + 1)
        qs, ks, vs, ds = (x[:, :, i].cpu() for x, i in ((q, at), (k, kv), (v, kv), (do, at)))
        ref = P.range_attention(qs, ks, vs, ranges, cap, do=ds)
        o, lse, dq, dk, dv = got
        check_all(ref, "bf16", D, cap, o[:, :, at], lse[:, at], [dq[:, :, at], dk[:, :, kv], dv[:, :, kv]])
