"""Weight gradients of linear layers whose input lies by heads: the tiles' columns are channels of several heads, and where a tile of the last
columns is narrow a CTA of the pair may begin inside one.  Against the 64-bit statement, tolerances as in the tests of linear layers."""
import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import Linear
from tests import _block64 as P
from tests.test_gpu_linear import by_heads, check, make

pytestmark = pytest.mark.gpu


# B, S, heads, channels of a head, n_out, act, gate_tokens (-1: no gate); planes of du: one from 65,536 of rows * (n_in + n_out) on, or where
# nothing stands between d_out and du
@pytest.mark.parametrize("B,S,heads,d,N,act,gt", [
    (1, 40, 3, 64, 72, "none", -1),
    (2, 40, 3, 64, 72, "gelu", -1),                # two planes, samples apart
    (1, 90, 3, 64, 136, "none", 0),                # two planes
    (2, 300, 3, 64, 72, "silu", 50),               # one plane
    (1, 700, 7, 64, 72, "none", -1),
    (3, 9, 7, 64, 40, "none", 4),                  # two planes
    (2, 130, 7, 64, 264, "gelu", 0),
    (1, 330, 11, 64, 72, "none", 0),
    (2, 5, 11, 64, 520, "silu", -1),               # two planes
    (2, 2100, 15, 64, 264, "none", -1),            # slices of the summed index
    (2, 300, 1, 64, 72, "none", 0),
    (2, 300, 2, 64, 72, "none", 0),
    (2, 300, 4, 64, 72, "none", 0),
    (2, 300, 5, 64, 72, "none", 0),
    (2, 300, 3, 128, 72, "none", 0),
])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradient_through_heads(B, S, heads, d, N, act, gt, dtype):
    K, tokens, f32 = heads * d, max(gt, 0), dtype == "f32"
    g = torch.Generator().manual_seed(K + S)
    x, w, dout, kept = make(g, dtype, B, S, K), make(g, dtype, N, K, scale=K ** -0.5), make(g, dtype, B, S, N), make(g, dtype, B, S, N)
    gate = torch.randn((B, -(-S // gt) if gt else 1, N), generator=g) if gt >= 0 else None
    order = torch.randperm(S, generator=g)
    apart = act != "none" or gate is not None
    (du, due), _ = P.du_of(dout.double(), kept.double(), act, False, None if gate is None else gate.double(), tokens, f32, order)
    half = torch.finfo(dout.dtype).eps / 2 if apart and not f32 else 0.0
    rounded = due + half * (du.abs() + due)
    op = Linear(vb.make_linear_shape(B, S, K, N, dtype, act, False, heads, tokens))
    xx, dx = by_heads(x, heads).cuda(), torch.empty((B, heads, S, d), dtype=x.dtype, device="cuda")
    dw, db, _ = op.backward(dout.cuda(), xx, w.cuda(), dx, kept=kept.cuda() if apart else None, gate=None if gate is None else gate.cuda(),
                            perm=order.to(torch.int32).cuda(), with_bias=True)
    check(dw, P.weight_grad(du, rounded, x.double()), "dweight")
    check(dx.transpose(1, 2).reshape(B, S, K), P.input_grad(du, rounded, w.double()), "dx")
    check(db, P.column_sums(du, due), "dbias")
    op.check_status()
