"""Linear layers, feed-forward blocks and block norms through the range-checked build, whose workspace slices are followed by guard zones."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = r"""
import torch
from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import BlockNorm, FeedForward, Linear
g = torch.Generator(device="cuda").manual_seed(0)
r = lambda dt, *s: torch.randn(s, generator=g, device="cuda").to(dt)
f = torch.float32
for dtype, dt in (("bf16", torch.bfloat16), ("f32", f)):
    for B, S, K, N, act, gated, heads, gt in ((1, 1, 64, 72, "gelu", False, 0, 0), (2, 33, 256, 136, "none", False, 2, 10), (1, 700, 136, 264, "silu", True, 0, 100),
                                              (2, 2000, 128, 72, "none", False, 1, 0)):
        s = vb.make_linear_shape(B, S, K, N, dtype, act, gated, heads, gt)
        op = Linear(s)
        x = r(dt, B, heads, S, K // heads) if heads else r(dt, B, S, K)
        w, out, kept = r(dt, s.wide, K), torch.empty((B, S, N), dtype=dt, device="cuda"), torch.empty((B, S, s.wide), dtype=dt, device="cuda")
        gate, perm = r(f, B, s.groups, N), torch.randperm(S, device="cuda").to(torch.int32) if heads else None
        # scratch of exactly the stated size
        ws = torch.empty(vb.linear_workspace_bytes(s), dtype=torch.uint8, device="cuda")
        xs = None if heads else (S * K, K)
        vb.vmoba_linear(s, x, xs, w, None, gate, (s.groups * N, N), out, (S * N, N), out, (S * N, N), kept, perm, op.dev_status, ws)
        op.backward(out, x, w, torch.empty_like(x), kept=kept, gate=gate, perm=perm, with_bias=True)
        torch.cuda.synchronize()
        op.check_status()
    for gated, gt in ((True, 30), (False, 0)):
        op = FeedForward(2, 100, 72, 264, dtype, "silu", gated, gt)
        x, w1, w2 = r(dt, 2, 100, 72), r(dt, op.shape.wide, 72), r(dt, 72, 264)
        gate, kept, out = r(f, 2, op.shape.groups, 72), op.keep(), torch.empty((2, 100, 72), dtype=dt, device="cuda")
        op.forward(x, w1, w2, out, gate=gate, residual=x, kept=kept)
        op.backward(out, x, w1, w2, kept, torch.empty_like(x), gate=gate, with_bias=True)
        torch.cuda.synchronize()
        op.check_status()
    for C, post, mod in ((72, "none", 0), (1536, "rms", 7), (5120, "layer", 0)):
        op = BlockNorm(vb.make_norm_shape(2, 40, C, dtype, "f32", "layer", post, mod))
        h, y, d = r(f, 2, 40, C), r(dt, 2, 40, C), r(dt, 2, 40, C)
        p = {n: r(f, 2, op.shape.groups, C) for n in ("gate", "scale", "shift")} | {n: r(f, C) for n in ("weight", "bias")}
        op.forward(h, torch.empty_like(d), y, h, **p)
        op.backward(d, h, torch.empty_like(h), h, y, torch.empty_like(y), **p)
        torch.cuda.synchronize()
        op.check_status()
print("clean")
"""


def test_operators_run_clean_through_the_range_checked_build():
    from paper_2506_23858_b200 import build
    env = dict(os.environ, VMOBA_LIB=build.ensure_built(debug=True))
    r = subprocess.run([sys.executable, "-c", SCRIPT], env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-3000:]
    assert r.stdout.strip().endswith("clean")
