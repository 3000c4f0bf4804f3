"""Norms of queries and keys with rotary positions, through the binding, against the oracle's float64 definition.

A result is rounded once to the rows' type; before that are fp32 sums over a head (their error a few dozen roundings of
the sum of absolute terms), a root, three products and a rotation whose sine and cosine are off by under 2^-24."""
import numpy as np
import pytest

from oracle import gated as og
from test_gpu_sequence import TINY, U, close, host, strided, up

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24

# rows, heads, kv_heads, dim, rot, axes, layout, pad
SHAPES = [(1, 1, 1, 2, 2, 1, "half", 0), (3, 2, 1, 6, 4, 1, "interleaved", 0), (33, 4, 2, 64, 48, 3, "half", 0),
          (70, 3, 5, 64, 64, 1, "interleaved", 7), (9, 8, 8, 128, 128, 3, "half", 64), (17, 1, 4, 100, 66, 3, "half", 3),
          (40, 5, 1, 33, 30, 2, "interleaved", 1), (5, 2, 2, 256, 254, 3, "half", 0), (6, 1, 1, 255, 2, 1, "half", 0),
          (300, 2, 2, 8, 8, 2, "half", 0), (4, 70, 9, 16, 10, 1, "interleaved", 0), (2, 1024, 3, 32, 32, 1, "half", 0)]


def ladder(mb, rot, axes):
    import torch

    steps, axis = mb.make_rotary(rot, axes, base=500.0)
    return torch.from_numpy(steps).cuda(), torch.from_numpy(axis).cuda(), [int(v) % (1 << 64) for v in steps], axis


def pairs_size(x, rot, layout):
    """For every element the sizes of its pair's two together."""
    x = np.abs(x).copy()
    half = rot // 2
    one = slice(0, half) if layout == "half" else slice(0, rot, 2)
    two = slice(half, rot) if layout == "half" else slice(1, rot, 2)
    both = x[..., one] + x[..., two]
    x[..., one], x[..., two] = both, both
    return x


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,heads,kv,dim,rot,axes,layout,pad", SHAPES)
def test_head_norm_rotary(gpu_lib, rows, heads, kv, dim, rot, axes, layout, pad, dtype):
    import torch

    rng = np.random.default_rng(rows * 31 + dim)
    steps, axis, isteps, iaxis = ladder(gpu_lib, rot, axes)
    pos = rng.integers(-200000, 200000, (rows, axes)).astype(np.int32)
    q, qr = up(rng.standard_normal((rows, heads, dim)) * rng.uniform(0.1, 5, (rows, heads, 1)), dtype)
    k, kr = up(rng.standard_normal((rows, kv, dim)), dtype)
    weights = dtype if rows % 2 else "f32"
    qw, qwr = up(rng.uniform(0.5, 1.5, dim), weights)
    kw, kwr = up(rng.uniform(-1.5, 1.5, dim), weights)
    if rows == 9:
        kw = kwr = None
    if pad:
        q, k = strided(q, pad, 1), strided(k, pad)
    p = torch.from_numpy(pos).cuda()
    got = gpu_lib.head_norm_rotary(q, k, qw, kw, p, steps, axis, eps=1e-4, layout=layout)
    for y, x, w in ((got[0], qr, qwr), (got[1], kr, kwr)):
        ref = og.head_norm_rotary(x, w, pos, isteps, iaxis, 1e-4, layout)
        h = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-4) * (1.0 if w is None else w)
        # sum of up to 256 squares over 64 lanes: 12 roundings; root, quotient, two products, the turn: 10 more
        close(y, ref, U[dtype] * np.abs(ref) + 24 * EPS * pairs_size(h, rot, layout) + TINY[dtype], "out")

    dq, dqr = up(rng.standard_normal((rows, heads, dim)), dtype)
    dk, dkr = up(rng.standard_normal((rows, kv, dim)), dtype)
    grads = gpu_lib.head_norm_rotary_backward(dq, dk, q, k, qw, kw, p, steps, axis, eps=1e-4, layout=layout)
    for dx, dw, dy, x, w in ((grads[0], grads[2], dqr, qr, qwr), (grads[1], grads[3], dkr, kr, kwr)):
        ref, wref = og.head_norm_rotary_backward(dy, x, w, pos, isteps, iaxis, 1e-4, layout)
        r = 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + 1e-4)
        h, d = np.abs(x * r), pairs_size(dy, rot, layout)
        a = d * (1.0 if w is None else np.abs(w))
        close(dx, ref, U[dtype] * np.abs(ref) + 40 * EPS * r * (a + h * (a * h).mean(-1, keepdims=True)) + TINY[dtype], "dx")
        # a thread adds its rows' terms in turn (at most 300 rows x 16 heads here, of at least 256 / 64 groups), then the groups' sums
        close(dw, wref, (40 + rows * x.shape[1]) * EPS * (d * h).sum((0, 1)), "dweight")


def test_in_place_over_a_projection(gpu_lib):
    """Queries and keys side by side in a row, each result in its own place; a bad order of results is refused."""
    import torch

    rng = np.random.default_rng(3)
    steps, axis, _, _ = ladder(gpu_lib, 48, 3)
    rows = torch.from_numpy(rng.standard_normal((50, 6 * 64))).to(torch.bfloat16).cuda()
    q, k, v = (rows[:, i * 128:(i + 1) * 128].unflatten(1, (2, 64)) for i in range(3))
    coords = torch.from_numpy(rng.integers(0, 1440, (50, 4)).astype(np.int32)).cuda()
    kept = v.clone()
    ref = gpu_lib.head_norm_rotary(q, k, None, None, coords[:, 1:], steps, axis)
    with pytest.raises(gpu_lib.MmbevError):
        gpu_lib.head_norm_rotary(q, k, None, None, coords[:, 1:], steps, axis, q_out=k, k_out=q)
    out = gpu_lib.head_norm_rotary(q, k, None, None, coords[:, 1:], steps, axis, q_out=q, k_out=k)
    assert out[0] is q and torch.equal(q, ref[0]) and torch.equal(k, ref[1]) and torch.equal(v, kept)


def test_row_count_on_the_device(gpu_lib):
    import torch

    rng = np.random.default_rng(4)
    steps, axis, _, _ = ladder(gpu_lib, 32, 1)
    q, k, dq, dk = (torch.from_numpy(rng.standard_normal((90, h, 32))).float().cuda() for h in (3, 2, 3, 2))
    w = torch.rand(32, device="cuda") + 0.5
    pos = torch.arange(90, device="cuda", dtype=torch.int32)
    for used, flagged in ((37, False), (0, False), (90, False), (91, True), (-1, True)):
        n = min(max(used, 0), 90)
        count = torch.tensor([used], device="cuda")
        fault = torch.zeros(1, dtype=torch.int32, device="cuda")
        outs = [torch.full_like(t, 7.0) for t in (q, k)]
        gpu_lib.head_norm_rotary(q, k, w, w, pos, steps, axis, row_count=count, q_out=outs[0], k_out=outs[1], fault=fault)
        assert bool(fault.item() & gpu_lib.FAULT_SEQUENCES) == flagged
        grads = [torch.full_like(t, 7.0) for t in (q, k)]
        _, _, dqw, dkw = gpu_lib.head_norm_rotary_backward(dq, dk, q, k, w, w, pos, steps, axis, row_count=count, dq=grads[0], dk=grads[1])
        for t in outs + grads:
            assert bool((t[n:] == 7.0).all())
        if n:
            ref = gpu_lib.head_norm_rotary(q[:n], k[:n], w, w, pos[:n], steps, axis)
            part = gpu_lib.head_norm_rotary_backward(dq[:n], dk[:n], q[:n], k[:n], w, w, pos[:n], steps, axis)
            assert torch.equal(outs[0][:n], ref[0]) and torch.equal(outs[1][:n], ref[1])
            assert torch.equal(grads[0][:n], part[0]) and torch.equal(grads[1][:n], part[1])
            assert torch.allclose(dqw, part[2], rtol=1e-5, atol=1e-5) and torch.allclose(dkw, part[3], rtol=1e-5, atol=1e-5)
        else:
            assert not dqw.any() and not dkw.any()


def test_gradient_against_differences(gpu_lib):
    import torch

    rng = np.random.default_rng(5)
    steps, axis, _, _ = ladder(gpu_lib, 20, 2)
    q, k, dq, dk = (torch.from_numpy(rng.standard_normal((6, 2, 24))).float().cuda() for _ in range(4))
    qw, kw = (torch.rand(24, device="cuda") + 0.5 for _ in range(2))
    pos = torch.from_numpy(rng.integers(0, 99, (6, 2)).astype(np.int32)).cuda()

    def loss(q, k, qw, kw):
        a, b = gpu_lib.head_norm_rotary(q, k, qw, kw, pos, steps, axis)
        return float((a.double() * dq).sum() + (b.double() * dk).sum())

    grads = gpu_lib.head_norm_rotary_backward(dq, dk, q, k, qw, kw, pos, steps, axis)
    args = [q, k, qw, kw]
    for i, g in enumerate(grads):
        at = torch.from_numpy(rng.standard_normal(args[i].shape)).float().cuda()
        h = 2.0 ** -8
        up_, down = ([*args[:i], args[i] + s * h * at, *args[i + 1:]] for s in (1, -1))
        d = (loss(*up_) - loss(*down)) / (2 * h)
        # third derivatives times h^2, and fp32 results of some 300 elements of size 1 over 2 h
        assert abs(d - float((g.double() * at).sum())) < 2e-3 * float((g.double() * at).abs().sum()) + 2e-3


def test_rows_past_one_workgroups_share(gpu_lib):
    """Large calls share an angle among more heads and walk many blocks of rows a workgroup: the same results."""
    import torch

    torch.manual_seed(0)
    steps, axis, _, _ = ladder(gpu_lib, 64, 3)
    q, k = torch.randn(60000, 8, 64, device="cuda").half(), torch.randn(60000, 4, 64, device="cuda").half()
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    pos = torch.randint(0, 1440, (60000, 3), device="cuda", dtype=torch.int32)
    w = torch.rand(64, device="cuda") + 0.5
    out = gpu_lib.head_norm_rotary(q, k, w, None, pos, steps, axis)
    grads = gpu_lib.head_norm_rotary_backward(dq, dk, q, k, w, None, pos, steps, axis)
    total = torch.zeros(2, 64, dtype=torch.float64, device="cuda")
    for lo in range(0, 60000, 20000):
        part = slice(lo, lo + 20000)
        few = [t[part].contiguous() for t in (q, k, dq, dk, pos)]
        a = gpu_lib.head_norm_rotary(few[0], few[1], w, None, few[4], steps, axis)
        g = gpu_lib.head_norm_rotary_backward(few[2], few[3], few[0], few[1], w, None, few[4], steps, axis)
        assert torch.equal(a[0], out[0][part]) and torch.equal(a[1], out[1][part])
        assert torch.equal(g[0], grads[0][part]) and torch.equal(g[1], grads[1][part])
        total += torch.stack([g[2], g[3]]).double()
    # sums of up to 480,000 terms of either sign, in fp32 by some 250 rows a thread
    assert float((total - torch.stack(grads[2:]).double()).abs().max()) < 1e-6 * 480000 ** 0.5 * 20
