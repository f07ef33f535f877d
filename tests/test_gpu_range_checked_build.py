"""Attention over key ranges and rotary positions through the range-checked build (guard zones behind every slice of the scratch, launches one after
another), with scratch and plans of exactly the size asked for, and from several threads."""
import os
import subprocess
import sys
import threading

import pytest
import torch

from paper_2506_23858_b200 import binding as vb
from paper_2506_23858_b200.layer import key_ranges
from tests.test_gpu_range_attn import CASES, KINDS, make, run
from tests.test_gpu_rotary import case

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_range_and_rotary_cases_run_clean_through_the_range_checked_build():
    from paper_2506_23858_b200 import build
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_range_attn.py", "tests/test_gpu_rotary.py", "-m", "gpu", "-q", "-x",
                        "-p", "no:cacheprovider", "-k", "against_the_statement or forward_and_backward or growing or packed_clips"],
                       env=dict(os.environ, VMOBA_LIB=build.ensure_built(debug=True)), cwd=ROOT, capture_output=True, text=True, timeout=1200)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-1000:]
    assert " passed" in r.stdout


def _snug(n):
    """n bytes followed by a kilobyte that has to stay as it is."""
    room = torch.full((n + 1024,), 0x5a, dtype=torch.uint8, device="cuda")
    return room, room[:n]


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: f"{k[0]}_{k[1]}")
@pytest.mark.parametrize("i", [1, 4, 6, 9, 13, 15, 16, 17])
def test_plan_and_scratch_of_exactly_their_size(i, kind):
    c = CASES[i]
    dtype, d = kind
    ranges = c["r"]()
    shape, op, host, dev, place = make(c["B"], c["Sq"], c["Sk"], c["h"], c["hk"], d, dtype, ranges, c.get("cap", 0.0), seed=i)
    want = run(op, dev, place, host)
    rooms = [_snug(vb.range_plan_bytes(shape)), _snug(vb.range_workspace_bytes(shape)), _snug(vb.range_workspace_bytes(shape, True))]
    vb.vmoba_range_plan(shape, ranges.cuda(), rooms[0][1])
    st = lambda x: tuple(x.stride()[:3])
    q, k, v, do = dev
    o, lse, status = torch.empty_like(q), torch.empty_like(op.lse), torch.zeros(1, dtype=torch.int32, device="cuda")
    resid = torch.empty_like(q) if dtype == "bf16" else None
    grads = [torch.empty_like(x) for x in (q, k, v)]
    args = (q, st(q), k, st(k), v, st(v), o, st(o), resid, lse)
    vb.vmoba_range_attn_fwd(shape, rooms[0][1], *args, status, rooms[1][1])
    vb.vmoba_range_attn_bwd(shape, rooms[0][1], *args, do, st(do), *[x for g in grads for x in (g, st(g))], status, rooms[2][1])
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(o, want[0]) and torch.equal(lse, op.lse) and all(torch.equal(a, b) for a, b in zip(grads, want[1]))
    assert all(bool((room[slice_.numel():] == 0x5a).all()) for room, slice_ in rooms)


@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("heads,tokens", [(3, 7), (12, 900), (100, 40), (401, 9)])
def test_rotary_scratch_of_exactly_its_size(heads, tokens, norm):
    shape, op, x, dy, w, *_ = case(1, heads, 128, (1, 1, tokens), (1, 1, tokens), "bf16", (64,), norm, "interleaved", seed=heads)
    xs, dys, ws = [t.cuda() for t in x], [t.cuda() for t in dy], [t.cuda() for t in w]
    want, dx = [torch.empty_like(t) for t in xs], [torch.empty_like(t) for t in xs]
    dw_want = op.backward(dys, xs, want, ws)
    st = [tuple(t.stride()[:3]) for t in xs]
    dw = [torch.empty_like(t) for t in dw_want]
    need = vb.rotary_workspace_bytes(shape, op.spec, 2)
    room, scratch = _snug(need)
    call = lambda ws_: vb.vmoba_rotary_bwd(shape, op.spec, dys, st, xs, st, ws, dx, st, dw, op.positions, op.freq, op.axis, ws_)
    call(scratch)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(dx + dw, want + dw_want)) and bool((room[need:] == 0x5a).all())
    with pytest.raises(vb.VmobaError, match="workspace"):
        call(room[: need - 256])


def test_calls_from_several_threads():
    """Small and large calls of every path at the same time, each thread on its own stream with its own objects."""
    torch.manual_seed(0)
    jobs = []
    for n, (kind, S, h) in enumerate([(KINDS[0], 200, 2), (KINDS[3], 700, 3), (KINDS[1], 130, 1), (KINDS[2], 257, 2), (KINDS[3], 64, 2)] * 2):
        dtype, d = kind
        ranges = key_ranges([S // 2, S // 3], n_tokens=S, frame=1, device="cpu")
        shape, op, host, dev, place = make(1, S, S, h, 1, d, dtype, ranges, 0.0 if n % 2 else 9.0, seed=n)
        o, grads = run(op, dev, place, host)
        rshape, rot, x, dy, w, *_ = case(1, 5 + 45 * (n % 2), d, (1, 5, 8), (1, 5, 8), dtype, (9,), "row", "half", seed=n)
        x, dy, w = ([t.cuda() for t in y] for y in (x, dy, w))
        dx = [torch.empty_like(t) for t in x]
        dw = rot.backward(dy, x, dx, w)
        jobs.append((op, dev, [t.clone() for t in (o, *grads)], rot, (dy, x, w), [t.clone() for t in dx + dw]))
    torch.cuda.synchronize()
    errors = []

    def work(op, dev, want, rot, args, rot_want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(6):
                    o, grads = torch.empty_like(dev[0]), [torch.empty_like(t) for t in dev[:3]]
                    op.forward(*dev[:3], o)
                    op.backward(dev[3], *grads)
                    dx = [torch.empty_like(t) for t in args[1]]
                    dw = rot.backward(args[0], args[1], dx, args[2])
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(a, b) for a, b in zip([o, *grads], want)) and all(torch.equal(a, b) for a, b in zip(dx + dw, rot_want))
                op.check_status()
        except BaseException as e:      # noqa: BLE001 (handed to the test's own thread)
            errors.append(e)

    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not errors and not any(t.is_alive() for t in threads), errors
