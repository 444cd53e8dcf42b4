"""Rotary positions on the GPU against 64 bits (tests/serving_ref.py derives the bounds)."""
import numpy as np
import pytest

from gpu_util import announce, lib_ready, torch_gpu
from serving_ref import check, rotate, rounding, torch_type

pytestmark = pytest.mark.gpu

CASES = [
    # rows, heads, d, rot, interleaved, in, out, gap, scaling
    (1, 1, 8, 2, False, "f32", "f32", 0, {}),
    (1, 40, 128, 128, False, "bf16", "bf16", 1024, {}),
    (17, 5, 128, 128, True, "f16", "f16", 0, dict(scaling="linear", factor=4.0)),
    (33, 3, 64, 10, False, "f32", "f32", 8, {}),            # pairs off 8
    (33, 3, 64, 10, True, "f32", "f32", 8, {}),
    (16, 2, 96, 42, False, "bf16", "f16", 0, dict(scaling="base", factor=8.0)),
    (15, 7, 256, 64, False, "f16", "bf16", 0, dict(scaling="ramp", factor=8.0, context=8192)),
    (5, 2, 512, 512, False, "f32", "bf16", 0, {}),
    (5, 2, 512, 512, True, "bf16", "f32", 0, {}),
    (300, 9, 64, 32, False, "f32", "f32", 0, {}),
    (2500, 33, 128, 96, False, "bf16", "bf16", 0, {}),
    (4000, 4, 64, 62, False, "f16", "f16", 0, {}),
]


def rows_of(torch, N, H, d, kind, gap, seed=0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn((N, H * d + gap), generator=g).to(torch_type(kind)).cuda()
    return wide[:, :H * d].view(N, H, d) if gap == 0 else wide[:, :H * d].unflatten(1, (H, d))


def positions(torch, N, seed=1):
    p = np.random.default_rng(seed).integers(0, 1 << 20, N)
    p[:6] = [0, 1, -5, 2 ** 31 - 1, -2 ** 31, 131071][:N]
    return p.astype(np.int32)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:8]))
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(case, inverse):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    N, H, d, rot, inter, ti, to, gap, scaling = case
    announce(f"rope {case} inverse {inverse}")
    x, pos = rows_of(torch, N, H, d, ti, gap), positions(torch, N)
    freq = rope_freqs(rot, base=500000.0, **scaling)
    table = RopeTable(freq, interleaved=inter, scale=1.25)
    out = torch.full((N, H * d + gap), 7.0, dtype=torch_type(to), device="cuda")
    view = out[:, :H * d].unflatten(1, (H, d))
    assert rope(x, torch.from_numpy(pos).cuda(), table, inverse=inverse, out=view) is view
    want, tol = rotate(x.double().cpu().numpy(), pos, freq.numpy(), inter, 1.25, inverse)
    check(view.double().cpu().numpy(), want, tol + rounding(np.abs(want) + tol, to), "rope")
    assert (out[:, H * d:] == 7.0).all()                    # what lies between the rows stays


@pytest.mark.parametrize("kind,rot,inter", [("bf16", 128, False), ("f16", 20, False), ("f32", 64, True), ("f32", 128, False)])
def test_rope_in_place(kind, rot, inter):
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce(f"rope in place {kind} {rot}")
    x = rows_of(torch, 50, 6, 128, kind, 2 * 128)
    pos = torch.from_numpy(positions(torch, 50)).cuda()
    table = RopeTable(rope_freqs(rot), interleaved=inter)
    want = rope(x, pos, table)
    assert rope(x, pos, table, out=x) is x
    assert torch.equal(x, want)


@pytest.mark.parametrize("N,H,d,rot", [(1, 1, 8, 6), (1, 1, 64, 2), (1, 2, 128, 126), (3, 1, 16, 14), (7, 40, 96, 30), (2100, 21, 96, 90),
                                       (2051, 5, 512, 500), (2200, 9, 128, 120), (40, 3, 256, 48), (9, 70, 32, 18)])
@pytest.mark.parametrize("kind", ["f16", "f32"])
def test_rope_of_some_channels(N, H, d, rot, kind):
    """Halves that end within the heads, within eight channels: against 64 bits, and the same in place."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce(f"rope of some channels {N} {H} {d} {rot} {kind}")
    x, pos = rows_of(torch, N, H, d, kind, 0), positions(torch, N)
    freq = rope_freqs(rot)
    table = RopeTable(freq, scale=0.5)
    out = rope(x, torch.from_numpy(pos).cuda(), table)
    want, tol = rotate(x.double().cpu().numpy(), pos, freq.numpy(), False, 0.5, False)
    check(out.double().cpu().numpy(), want, tol + rounding(np.abs(want) + tol, kind), "some channels")
    assert torch.equal(out[:, :, rot:], x[:, :, rot:])
    assert rope(x, torch.from_numpy(pos).cuda(), table, out=x) is x
    assert torch.equal(x, out)


def test_rope_reads_only_its_rows():
    """NaN around the rows, in the gaps between them too, reaches nothing."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce("rope between gaps")
    table, pos = RopeTable(rope_freqs(42)), torch.arange(20, dtype=torch.int32, device="cuda")
    wide = torch.full((22, 3 * 64 + 16), float("nan"), device="cuda")
    x = wide[1:21, 8:200].unflatten(1, (3, 64))
    x.copy_(torch.randn((20, 3, 64), generator=torch.Generator().manual_seed(2)))
    assert torch.equal(rope(x, pos, table), rope(x.contiguous(), pos, table))


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (22, False)])
def test_rope_gradient(rot, inter):
    """The map is linear, so a difference is exact up to rounding: R e for each unit vector e, against
    what inverse gives for each output channel."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce(f"rope gradient {rot} {inter}")
    d = 64
    pos = torch.full((d,), 12345, dtype=torch.int32, device="cuda")
    table = RopeTable(rope_freqs(rot), interleaved=inter, scale=0.75)
    eye = torch.eye(d, device="cuda").view(d, 1, d)
    forward = rope(eye, pos, table)[:, 0]                   # row i: dy / dx_i
    back = rope(eye, pos, table, inverse=True)[:, 0]        # row j: the gradient of y_j
    assert torch.equal(forward, back.t().contiguous())
    x, h = torch.randn((d, 1, d), device="cuda"), 0.5 * eye
    diff = (rope(x + h, pos, table) - rope(x - h, pos, table))[:, 0]
    # x +- h and the two results are rounded, each below 8 in size: 6 half steps of 8, and 8 of the products
    assert (diff - forward).abs().max() <= 14 * 8 * 2.0 ** -24
    # and turned back with the scale's inverse it is the input: 2 passes of 4 half steps of |a| + |b|
    undo = RopeTable(rope_freqs(rot), interleaved=inter, scale=1 / 0.75)
    again = rope(rope(x, pos, table), pos, undo, inverse=True)
    assert (again - x).abs().max() <= 2 * 4 * 2.0 ** -24 * 2 * 2 * float(x.abs().max())


def test_rope_on_another_stream_and_captured():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce("rope captured")
    x = rows_of(torch, 40, 4, 128, "bf16", 0)
    pos = torch.arange(40, dtype=torch.int32, device="cuda")
    table = RopeTable(rope_freqs(128))
    out = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        rope(x, pos, table, out=out)
    s.synchronize()
    assert torch.equal(out, rope(x, pos, table))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope(x, pos, table, out=out)
    for k in range(4):
        pos += 1000 * k
        x.mul_(0.5)
        g.replay()
        got = out.clone()
        torch.cuda.synchronize()
        assert torch.equal(got, rope(x, pos, table)), k


def test_rope_without_rows():
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce("rope without rows")
    z = torch.zeros((0, 4, 64), device="cuda")
    assert rope(z, torch.zeros(0, dtype=torch.int32, device="cuda"), RopeTable(rope_freqs(64))).shape == (0, 4, 64)


@pytest.mark.parametrize("kind,to,rot,inter", [("f32", "f32", 64, False), ("bf16", "bf16", 64, True), ("f16", "f32", 22, False), ("f32", "bf16", 64, False)])
def test_rope_gradient_through_autograd(kind, to, rot, inter):
    """The gradient that autograd takes is the formula's: against 64 bits, and bit for bit what inverse gives."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce(f"rope through autograd {kind} {to} {rot} {inter}")
    N, H, d = 50, 6, 64
    pos, freq = positions(torch, N), rope_freqs(rot, base=500000.0)
    at, table = torch.from_numpy(pos).cuda(), RopeTable(freq, interleaved=inter, scale=1.25)
    x, w = rows_of(torch, N, H, d, kind, 0).requires_grad_(), rows_of(torch, N, H, d, to, 0, seed=9)
    y = rope(x, at, table, out=torch.empty((N, H, d), dtype=torch_type(to), device="cuda"))
    with torch.no_grad():
        assert torch.equal(y, rope(x, at, table, out=torch.empty_like(y)))
        back = rope(w, at, table, inverse=True, out=torch.empty_like(x))
    y.backward(w)
    assert x.grad.dtype == x.dtype and torch.equal(x.grad, back)
    want, tol = rotate(w.double().cpu().numpy(), pos, freq.numpy(), inter, 1.25, True)
    check(x.grad.double().cpu().numpy(), want, tol + rounding(np.abs(want) + tol, kind), "gradient")
    # a fused projection's slice in place
    base = rows_of(torch, N, H + 4, d, kind, 0, seed=3).requires_grad_()
    rows = base * 1.0
    rope(rows[:, 2:8], at, table, out=rows[:, 2:8])
    g = rows_of(torch, N, H + 4, d, kind, 0, seed=4)
    rows.backward(g)
    want = g.clone()
    rope(want[:, 2:8], at, table, inverse=True, out=want[:, 2:8])
    assert torch.equal(base.grad, want)


def test_rope_gradient_captured():
    """Forward and backward in one graph, replayed against eager passes."""
    torch = torch_gpu()
    lib_ready()
    from paper_2607_06523_amd import RopeTable, rope, rope_freqs
    announce("rope gradient captured")
    x = rows_of(torch, 40, 4, 128, "bf16", 0).requires_grad_()
    w = rows_of(torch, 40, 4, 128, "bf16", 0, seed=5)
    pos, table = torch.arange(40, dtype=torch.int32, device="cuda"), RopeTable(rope_freqs(128))
    both = lambda: torch.autograd.grad(rope(x, pos, table), x, w)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        both()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = both()
    for k in range(4):
        pos += 1000 * k
        w.mul_(0.5)
        g.replay()
        mine = got.clone()
        torch.cuda.synchronize()
        assert torch.equal(mine, rope(w, pos, table, inverse=True)), k
        assert torch.equal(mine, both()), k
