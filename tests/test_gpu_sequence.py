"""The sequence operators (layer norm, rotary positions, linear attention with decay), through the binding, against
the oracle's float64 definitions.

Tolerances follow from the number formats.  u is the unit roundoff of the rows' type (2^-24, 2^-11, 2^-8): a result is
rounded once, an error of u times itself.  Sums are taken in fp32, whose error is bounded by a few dozen times 2^-24
times the sum of the absolute terms.  In 16-bit attention each pair of rows (i, j) goes either through a rounded
product q.k or through the rounded state, so its share of an output is off by at most u times its absolute value.
"""
import numpy as np
import pytest

from oracle import sequence as osq

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-30, "f16": 2.0 ** -24, "bf16": 1e-30}  # the smallest step of the type near zero


def torch_type(name):
    import torch

    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def up(a, name="f32"):
    """Values rounded to the type, on the GPU; and the same as float64 for the oracle."""
    import torch

    t = torch.from_numpy(np.asarray(a, np.float64)).to(torch_type(name))
    return t.cuda(), t.double().numpy()


def host(t):
    return t.double().cpu().numpy()


def strided(t, pad, shift=0):
    """The same values in rows `pad` elements further apart, the first `shift` elements into its memory."""
    import torch

    rows, n = t.shape[0], t[0].numel() if t.shape[0] else 0
    room = torch.full((rows * (n + pad) + shift,), 77.0, dtype=t.dtype, device=t.device)
    view = room[shift:].view(rows, n + pad)[:, :n]
    view.copy_(t.reshape(rows, n))
    return view.view(t.shape) if t.dim() == 2 else view.unflatten(1, t.shape[1:])


def close(got, ref, bound, what):
    got = host(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = np.abs(got - ref) > bound
    assert not off.any(), f"{what}: {off.sum()} of {off.size} outside, worst {np.nanmax(np.abs(got - ref) / bound):.3g} of the bound"


# ------------------------------------------------------------------ layer norm

NORM_SHAPES = [(1, 1), (3, 2), (257, 5), (40, 8), (1000, 37), (129, 64), (33, 67), (70, 128), (65, 200), (17, 256), (9, 300),
               (5, 513), (7, 1024), (6, 1031), (3, 2048), (3, 2500), (2, 4097), (2, 8192)]


def norm_bounds(ref, s, rstd, w, dtype):
    # the centred rows carry a few dozen roundings of the largest element; rstd and the rest a few
    spread = np.abs(s).max(1, keepdims=True) * rstd[:, None] * (1.0 if w is None else np.abs(w))
    return U[dtype] * np.abs(ref) + 48 * 2.0 ** -24 * (spread + np.abs(ref)) + TINY[dtype]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", NORM_SHAPES)
def test_layer_norm(gpu_lib, rows, width, dtype):
    rng = np.random.default_rng(rows * 10007 + width)
    x, xr = up(rng.standard_normal((rows, width)) * rng.uniform(0.1, 10, (rows, 1)) + rng.uniform(-5, 5, (rows, 1)), dtype)
    same = rows % 2 == 0
    w, wr = up(rng.uniform(0.5, 1.5, width), dtype if same else "f32")
    b, br = up(rng.standard_normal(width), dtype if same else "f32")
    out, total, mean, rstd = gpu_lib.layer_norm(strided(x, 3, 1) if width % 2 else x, w, b, eps=1e-3, stats=True)
    ref, m, r = osq.layer_norm(xr, wr, br, 1e-3)
    close(out, ref, norm_bounds(ref, xr, r, wr, dtype) + 48 * 2.0 ** -24 * np.abs(br), "out")
    close(mean, m, 48 * 2.0 ** -24 * np.abs(xr).max(1) + 1e-30, "mean")
    close(rstd, r, 1e-5 * r, "rstd")
    assert total.shape == x.shape


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", [(300, 64), (31, 67), (4, 1100)])
def test_layer_norm_residual_and_in_place(gpu_lib, rows, width, dtype):
    import torch

    rng = np.random.default_rng(rows + width)
    x, xr = up(rng.standard_normal((rows, width)), dtype)
    y, yr = up(rng.standard_normal((rows, width)), dtype)
    total = torch.from_numpy(xr + yr).to(torch_type(dtype)).double().numpy()  # one rounding, as the sum's definition
    out, s, _, _ = gpu_lib.layer_norm(strided(x, 5), None, None, residual=y, eps=1e-5)
    assert np.array_equal(host(s), total)
    ref, _, r = osq.layer_norm(total, None, None, 1e-5)
    close(out, ref, norm_bounds(ref, total, r, None, dtype), "out")
    # the sum over the residual's own rows, the result over x's
    gpu_lib.layer_norm(x, None, None, residual=y, eps=1e-5, out=x, out_sum=y)
    assert torch.equal(x, out) and torch.equal(y, s)


def test_layer_norm_rows_without_variance_and_far_from_zero(gpu_lib):
    x, xr = up(np.full((5, 96), 1000.0))
    out, _, mean, rstd = gpu_lib.layer_norm(x, None, None, eps=1e-5, stats=True)
    assert np.array_equal(host(mean), np.full(5, 1000.0)) and np.all(host(out) == 0.0)
    rng = np.random.default_rng(5)
    x, xr = up(rng.standard_normal((64, 128)) * 0.01 + 4096.0)
    out, _, _, rstd = gpu_lib.layer_norm(x, None, None, eps=0.0, stats=True)
    ref, _, r = osq.layer_norm(xr, None, None, 0.0)
    # the mean's error, a few steps of 4096, moves all of a row's elements alike
    close(out, ref, 8 * 4096 * 2.0 ** -24 * r[:, None] + 1e-5, "out")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,width", NORM_SHAPES + [(5000, 64), (3000, 200), (20000, 8)])
def test_layer_norm_backward(gpu_lib, rows, width, dtype):
    rng = np.random.default_rng(rows * 7 + width)
    x, xr = up(rng.standard_normal((rows, width)) * 2 + 1, dtype)
    dy, dr = up(rng.standard_normal((rows, width)), dtype)
    skip, sr = up(rng.standard_normal((rows, width)), dtype) if rows % 2 else (None, None)
    w, wr = up(rng.uniform(0.5, 1.5, width))
    _, _, mean, rstd = gpu_lib.layer_norm(x, w, None, eps=1e-2, stats=True)
    dx, dw, db = gpu_lib.layer_norm_backward(strided(dy, 3, 1) if width % 2 else dy, x, w, mean, rstd, dskip=skip)
    ref, rw, rb = osq.layer_norm_backward(dr, xr, wr, host(mean), host(rstd), sr)
    h = (xr - host(mean)[:, None]) * host(rstd)[:, None]
    big = host(rstd)[:, None] * (np.abs(dr * wr) + np.abs(dr * wr).mean(1, keepdims=True) * (1 + np.abs(h)) *
                                 (1 + np.abs(h).max(1, keepdims=True)))
    close(dx, ref, U[dtype] * np.abs(ref) + 64 * 2.0 ** -24 * (big + np.abs(ref)) + TINY[dtype], "dx")
    # a column's sum: at most (rows in a thread's run + the partial sums) additions, the errors adding up as their root
    terms = 2.0 ** -24 * (8 + 4 * np.sqrt(rows))
    close(dw, rw, terms * np.abs(dr * h).sum(0) + 1e-30, "dweight")
    close(db, rb, terms * np.abs(dr).sum(0) + 1e-30, "dbias")


def test_layer_norm_gradient_against_differences(gpu_lib):
    """The loss sum(out * g) along a random direction, by the library's own forward pass in fp32."""
    import torch

    torch.manual_seed(0)
    x, d, g = (torch.randn(300, 96, device="cuda") for _ in range(3))
    w, b = torch.rand(96, device="cuda") + 0.5, torch.randn(96, device="cuda")
    _, _, mean, rstd = gpu_lib.layer_norm(x, w, b, stats=True)
    dx, dw, db = gpu_lib.layer_norm_backward(g, x, w, mean, rstd)
    eps = 2.0 ** -6

    def loss(x, w, b):
        return (gpu_lib.layer_norm(x, w, b)[0].double() * g.double()).sum().item()

    # central differences: their own error is eps^2 times a third derivative of order one a term
    size = float((dx * d).double().abs().sum())
    assert abs((loss(x + eps * d, w, b) - loss(x - eps * d, w, b)) / (2 * eps) - (dx * d).double().sum().item()) < 2e-3 * size
    e = torch.randn(96, device="cuda")
    size = float((dw * e).double().abs().sum() + (db * e).double().abs().sum())
    assert abs((loss(x, w + e, b) - loss(x, w - e, b)) / 2 - (dw * e).double().sum().item()) < 1e-4 * size + 1e-2
    assert abs((loss(x, w, b + e) - loss(x, w, b - e)) / 2 - (db * e).double().sum().item()) < 1e-4 * size + 1e-2


def test_layer_norm_row_count_on_the_device(gpu_lib):
    import torch

    rng = np.random.default_rng(8)
    x, xr = up(rng.standard_normal((1000, 40)))
    for count, use, fault in ((0, 0, 0), (1, 1, 0), (613, 613, 0), (1000, 1000, 0), (-5, 0, 16), (1001, 1000, 16)):
        n = torch.tensor([count], dtype=torch.int64, device="cuda")
        fw = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = torch.full_like(x, -7.0)
        gpu_lib.layer_norm(x, None, None, out=out, row_count=n, fault=fw)
        ref, _, r = osq.layer_norm(xr, None, None, 1e-5)
        close(out[:use], ref[:use], norm_bounds(ref, xr, r, None, "f32")[:use], count)
        assert bool((out[use:] == -7.0).all()) and int(fw) == fault
        mean, rstd = torch.zeros(1000, device="cuda"), torch.ones(1000, device="cuda")
        bad = torch.where(torch.arange(1000, device="cuda")[:, None] < use, x, float("nan"))
        dx, dw, db = gpu_lib.layer_norm_backward(bad, bad, None, mean, rstd, dx=torch.full_like(x, -7.0), row_count=n)
        assert bool((dx[use:] == -7.0).all())
        close(db, xr[:use].sum(0), 1e-4 + 0 * xr[0], "dbias of the rows in use alone")


# ------------------------------------------------------------------ rotary positions

ROTARY = [  # rows, heads, dim, rotary_dim, axes, layout, pad
    (1, 1, 2, 2, 1, "half", 0), (5, 3, 64, 64, 1, "interleaved", 0), (70, 2, 64, 48, 3, "half", 7), (33, 5, 40, 10, 2, "interleaved", 0),
    (129, 1, 31, 18, 3, "half", 1), (64, 17, 32, 32, 1, "half", 64), (9, 4, 128, 96, 3, "interleaved", 3), (12, 2, 200, 150, 1, "half", 0),
    (3, 300, 8, 6, 1, "interleaved", 0), (2, 1, 1024, 1024, 8, "half", 0)]


def rotary_bound(x, dtype):
    # a pair's two products, sine and cosine off by a few 2^-24 (series, phase's low bits, conversion)
    big = np.abs(x).max(2, keepdims=True)
    return U[dtype] * 2 * big + 16 * 2.0 ** -24 * big + TINY[dtype]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,heads,dim,rot,axes,layout,pad", ROTARY)
def test_rotary(gpu_lib, rows, heads, dim, rot, axes, layout, pad, dtype):
    import torch

    rng = np.random.default_rng(rows + dim)
    x, xr = up(rng.standard_normal((rows, heads, dim)), dtype)
    x = strided(x, pad, pad % 2)
    positions = rng.integers(-2 ** 31, 2 ** 31, (rows, axes))
    positions[: rows // 2] = rng.integers(0, 2000, (rows // 2, axes))
    steps, axis = gpu_lib.make_rotary(rot, axes)
    ds, da = torch.from_numpy(steps).cuda(), torch.from_numpy(axis).cuda()
    dp = torch.from_numpy(positions.astype(np.int32)).cuda()
    out = gpu_lib.rotary(x, dp, ds, da, layout=layout)
    ref = osq.rotary(xr, positions, [int(v) % (1 << 64) for v in steps], axis, layout)
    close(out, ref, rotary_bound(xr, dtype), "out")
    assert torch.equal(out[..., rot:], x[..., rot:])
    back = gpu_lib.rotary(x, dp, ds, da, layout=layout, inverse=True)
    close(back, osq.rotary(xr, positions, [int(v) % (1 << 64) for v in steps], axis, layout, True), rotary_bound(xr, dtype), "inverse")
    gpu_lib.rotary(x, dp, ds, da, layout=layout, out=x)
    assert torch.equal(x, out)


def test_rotary_from_voxel_coordinates_with_a_count(gpu_lib):
    """Positions read out of (b, iz, iy, ix) rows, the rows in use counted by the device."""
    import torch

    rng = np.random.default_rng(4)
    coords = rng.integers(0, 1440, (500, 4)).astype(np.int32)
    x, xr = up(rng.standard_normal((500, 4, 48)), "bf16")
    steps, axis = gpu_lib.make_rotary(48, 3, base=1000.0)
    ds, da = torch.from_numpy(steps).cuda(), torch.from_numpy(axis).cuda()
    n = torch.tensor([321], dtype=torch.int64, device="cuda")
    out = torch.full_like(x, -7.0)
    gpu_lib.rotary(x, torch.from_numpy(coords).cuda()[:, 1:], ds, da, out=out, row_count=n)
    ref = osq.rotary(xr, coords[:, 1:], [int(v) % (1 << 64) for v in steps], axis, "half")
    close(out[:321], ref[:321], rotary_bound(xr, "bf16")[:321], "out")
    assert bool((out[321:] == -7.0).all())


# ------------------------------------------------------------------ linear attention

def attention_case(seed, lengths, H, kv, kd, vd, dtype, spare=0, fused=False, carry=False):
    import torch

    rng = np.random.default_rng(seed)
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    rows = int(offsets[-1]) + spare
    q, k, v, g = (rng.standard_normal(s) for s in ((rows, H, kd), (rows, kv, kd), (rows, kv, vd), (rows, H, vd)))
    c = dict(offsets=offsets, rows=rows, used=int(offsets[-1]), scale=kd ** -0.5, dtype=dtype)
    for name, t in (("q", q), ("k", k), ("v", v), ("g", g)):
        c[name], c[name + "r"] = up(t, dtype)
        if spare:  # what no sequence has may hold anything
            c[name][int(offsets[-1]):] = float("nan")
    if fused:  # side by side in one row, as a projection writes them
        widths = [H * kd, kv * kd, kv * vd]
        room = torch.cat([c[n].flatten(1) for n in "qkv"], 1)
        room = torch.nn.functional.pad(room, (1, 2))
        parts = room[:, 1:-2].split(widths, 1)
        c["q"], c["k"], c["v"] = (p.unflatten(1, (n, -1)) for p, n in zip(parts, (H, kv, kv)))
    decay = -np.exp(rng.uniform(np.log(2e-4), np.log(0.7), H))
    if H > 1:
        decay[0] = 0.0
    if H > 2:
        decay[1] = -30.0
    c["decay"], c["decayr"] = up(decay)
    c["s0"] = c["s0r"] = c["df"] = c["dfr"] = None
    if carry:
        c["s0"], c["s0r"] = up(3 * rng.standard_normal((len(lengths), H, kd, vd)))
        c["df"], c["dfr"] = up(rng.standard_normal((len(lengths), H, kd, vd)))
    c["doff"] = torch.from_numpy(offsets).cuda()
    return c


def share_bound(value, size, dtype):
    """u of the result, and of every pair's absolute share (see the file's head); fp32 sums beside it."""
    return U[dtype] * np.abs(value) + (1.1 * (U[dtype] if dtype != "f32" else 0.0) + 2e-5) * size + \
        (1e-6 if dtype != "f32" else 1e-9) * size.max(initial=0.0) + TINY[dtype]


def check_forward(mb, c, final=True, **kw):
    import torch

    out = torch.full((c["rows"],) + c["q"].shape[1:2] + c["v"].shape[2:], -7.0, dtype=c["q"].dtype, device="cuda")
    fw = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, end = mb.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], scale=c["scale"], initial_state=c["s0"],
                                   final_state=final, out=out, fault=fw, **kw)
    n = c["used"]
    ref, ref_end = osq.linear_attention(c["qr"], c["kr"], c["vr"], c["decayr"], c["offsets"], c["scale"], c["s0r"])
    size, size_end = osq.linear_attention(*(np.abs(c[t + "r"]) for t in "qkv"), c["decayr"], c["offsets"], abs(c["scale"]),
                                          None if c["s0r"] is None else np.abs(c["s0r"]))
    close(out[:n], ref[:n], share_bound(ref, size, c["dtype"])[:n], "out")
    assert bool((out[n:] == -7.0).all()), "rows of no sequence were written"
    if final:
        close(end, ref_end, 2e-6 * size_end + 2e-6 * size_end.max(initial=0.0) * 0.1 + 1e-30, "final state")
    assert int(fw) == 0


def check_backward(mb, c, **kw):
    import torch

    dq, dk, dv = (torch.full(c[t].shape, -7.0, dtype=c[t].dtype, device="cuda") for t in "qkv")
    dq, dk, dv, ds = mb.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"], scale=c["scale"],
                                                  initial_state=c["s0"], dfinal_state=c["df"],
                                                  dinitial_state=c["s0"] is not None, dq=dq, dk=dk, dv=dv, **kw)
    args = ("gr", "qr", "kr", "vr")
    ref = osq.linear_attention_backward(*(c[t] for t in args), c["decayr"], c["offsets"], c["scale"], c["s0r"], c["dfr"])
    size = osq.linear_attention_backward(*(np.abs(c[t]) for t in args), c["decayr"], c["offsets"], abs(c["scale"]),
                                         *(None if t is None else np.abs(t) for t in (c["s0r"], c["dfr"])))
    n = c["used"]
    for name, got, r, s in zip(("dq", "dk", "dv"), (dq, dk, dv), ref, size):
        close(got[:n], r[:n], share_bound(r, s, c["dtype"])[:n], name)
        assert bool((got[n:] == -7.0).all()), "rows of no sequence were written"
    if ds is not None:
        close(ds, ref[3], 2e-6 * size[3] + 2e-7 * size[3].max(initial=0.0) + 1e-30, "dinitial")


ATTENTION = [  # lengths, heads, kv_heads, key_dim, value_dim, spare, fused, carry
    ([1], 1, 1, 1, 1, 0, False, False),
    ([2, 0, 1], 2, 1, 3, 5, 3, False, True),
    ([0], 3, 3, 16, 16, 2, False, True),
    ([63, 64, 65], 2, 2, 32, 32, 0, True, False),
    ([1, 127, 16, 17, 15, 0, 33], 3, 3, 64, 64, 5, True, True),
    ([200], 4, 2, 64, 64, 0, False, False),
    ([130, 70], 4, 1, 40, 24, 1, True, True),
    ([97], 2, 2, 128, 128, 0, False, True),
    ([129, 3], 3, 3, 100, 36, 0, True, False),
    ([66], 2, 1, 31, 127, 0, False, True),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(ATTENTION)))
def test_attention(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, spare, fused, carry = ATTENTION[i]
    c = attention_case(i, lengths, H, kv, kd, vd, dtype, spare, fused, carry)
    check_forward(gpu_lib, c)
    check_forward(gpu_lib, c, final=False)
    check_backward(gpu_lib, c)


LONG = [  # sequences long enough to be cut into segments: one, ragged with empty ones, many short among long
    ([1500], 3, 3, 64, 64, 0, True, True),
    ([700, 0, 64, 1, 900, 0], 2, 1, 32, 32, 7, False, True),
    ([0, 0, 1100], 2, 2, 128, 128, 0, False, False),
    ([3, 2, 1] * 40 + [640] + [5] * 50, 3, 3, 64, 48, 1, True, True),
    ([64 * 13, 64 * 4], 1, 1, 64, 64, 0, False, True),
]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_attention_in_segments(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, spare, fused, carry = LONG[i]
    c = attention_case(100 + i, lengths, H, kv, kd, vd, dtype, spare, fused, carry)
    check_forward(gpu_lib, c)
    check_backward(gpu_lib, c)
    check_forward(gpu_lib, c, max_length=64)  # the same sequences walked whole


def test_attention_gradient_against_differences(gpu_lib):
    """The loss is linear in each of q, k, v and the initial state, so a difference over any distance is its slope."""
    import torch

    torch.manual_seed(1)
    c = attention_case(7, [150, 0, 90], 4, 2, 64, 32, "f32", carry=True)
    dq, dk, dv, ds = gpu_lib.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"], c["scale"],
                                                       c["s0"], c["df"], True)

    def loss(q, k, v, s0):
        out, end = gpu_lib.linear_attention(q, k, v, c["decay"], c["doff"], c["scale"], s0, True)
        return (out.double() * c["g"].double()).sum().item() + (end.double() * c["df"].double()).sum().item()

    base = [c["q"], c["k"], c["v"], c["s0"]]
    for i, grad in enumerate((dq, dk, dv, ds)):
        d = torch.randn_like(base[i])
        ends = [loss(*(t + s * d if j == i else t for j, t in enumerate(base))) for s in (1.0, -1.0)]
        size = float((grad * d).double().abs().sum()) + abs(ends[0]) + abs(ends[1])
        assert abs((ends[0] - ends[1]) / 2 - (grad * d).double().sum().item()) < 2e-5 * size


def test_attention_state_carries_over_calls(gpu_lib):
    """One sequence in two calls, the state handed on, against one call."""
    c = attention_case(9, [900], 2, 2, 64, 64, "bf16")
    import torch

    whole, end = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], final_state=True)
    cut = 333
    off = [torch.tensor([0, n], dtype=torch.int64, device="cuda") for n in (cut, 900 - cut)]
    _, mid = gpu_lib.linear_attention(c["q"][:cut], c["k"][:cut], c["v"][:cut], c["decay"], off[0], final_state=True)
    rest, last = gpu_lib.linear_attention(c["q"][cut:], c["k"][cut:], c["v"][cut:], c["decay"], off[1], initial_state=mid,
                                          final_state=True)
    size, size_end = osq.linear_attention(*(np.abs(c[t + "r"]) for t in "qkv"), c["decayr"], c["offsets"], c["scale"])
    close(rest, host(whole[cut:]), 2 * share_bound(host(whole), size, "bf16")[cut:], "rest")
    close(last, host(end), 4e-6 * size_end + 1e-6 * size_end.max(), "state")


def test_attention_fp16_state_beyond_its_range(gpu_lib):
    """Sums of 3,000 positive rows of size 6: 108,000, past fp16's largest value, in the state but not in the output."""
    import torch

    n = 3000
    q = torch.zeros(n, 1, 32, dtype=torch.float16, device="cuda")
    q[:, :, 0], q[:, :, 1] = 1.0, -1.0
    k = torch.full((n, 1, 32), 6.0, dtype=torch.float16, device="cuda")
    k[:, :, 1] = 5.75
    v = torch.full((n, 1, 32), 6.0, dtype=torch.float16, device="cuda")
    off = torch.tensor([0, n], dtype=torch.int64, device="cuda")
    out, end = gpu_lib.linear_attention(q, k, v, torch.zeros(1, device="cuda"), off, scale=1.0, final_state=True)
    want = 1.5 * torch.arange(1, n + 1, dtype=torch.float64, device="cuda")[:, None, None].expand(n, 1, 32)
    # the state's two columns are rounded to 11 bits of 108,000 before they cancel
    assert float(((out.double() - want).abs() / (want + 2 * 36.0 * torch.arange(1, n + 1, device="cuda")[:, None, None])).max()) < 2.0 ** -10
    assert float((end[0, 0, 0] - 36.0 * n).abs().max()) <= 36.0 * n * 1e-6


def test_attention_bad_offsets_are_clamped_and_reported(gpu_lib):
    import torch

    c = attention_case(11, [100, 100], 2, 2, 32, 32, "f32")
    for bad in ([0, 150, 100], [5, 100, 200], [0, 100, 300], [0, 100, -3], [0, 2 ** 62, 200]):
        fw = torch.zeros(1, dtype=torch.int32, device="cuda")
        room = torch.full((200 + 64, 2, 32), -7.0, device="cuda")
        gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], torch.tensor(bad, dtype=torch.int64, device="cuda"),
                                 out=room[32:232], fault=fw)
        assert int(fw) == gpu_lib.FAULT_SEQUENCES, bad
        assert bool((room[:32] == -7.0).all()) and bool((room[232:] == -7.0).all())


def test_attention_sequences_do_not_see_each_other(gpu_lib):
    """A sequence of NaN beside others, in whole walks and in segments: the others keep their results bit for bit."""
    import torch

    for lengths in ([70, 64, 33], [700, 640, 900]):
        c = attention_case(13, lengths, 2, 2, 64, 64, "bf16")
        clean, end = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], final_state=True)
        lo, hi = int(c["offsets"][1]), int(c["offsets"][2])
        for t in "qkv":
            c[t][lo:hi] = float("nan")
        out, last = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], final_state=True)
        assert torch.equal(out[:lo], clean[:lo]) and torch.equal(out[hi:], clean[hi:])
        assert torch.equal(last[[0, 2]], end[[0, 2]])


STEP = [(1, 1, 1, 1, 1, 1), (5, 4, 2, 64, 64, 9), (3, 2, 2, 128, 128, 3), (17, 3, 3, 31, 40, 17), (9, 8, 1, 96, 33, 20), (0, 2, 2, 8, 8, 4)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,H,kv,kd,vd,slots", STEP)
def test_attention_step(gpu_lib, rows, H, kv, kd, vd, slots, dtype):
    import torch

    rng = np.random.default_rng(rows + kd)
    c = attention_case(rows + kd, [rows], H, kv, kd, vd, dtype, fused=rows > 3)
    state, sr = up(rng.standard_normal((slots, H, kd, vd)))
    order = rng.permutation(slots)[:rows].astype(np.int32)
    if rows > 3:
        order[1] = -1
        order[2] = slots + 5
    fw = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((rows, H, vd), -7.0, dtype=torch_type(dtype), device="cuda")
    gpu_lib.linear_attention_step(c["q"], c["k"], c["v"], c["decay"], state, torch.from_numpy(order).cuda(), c["scale"], out=out,
                                  fault=fw)
    ref, rs = osq.linear_attention_step(c["qr"], c["kr"], c["vr"], c["decayr"], sr, order, c["scale"])
    size, ss = osq.linear_attention_step(*(np.abs(c[t + "r"]) for t in "qkv"), c["decayr"], np.abs(sr), order, c["scale"])
    done = (order >= 0) & (order < slots)
    close(out[torch.from_numpy(done).cuda()], ref[done], U[dtype] * np.abs(ref[done]) + 2e-5 * size[done] + TINY[dtype], "out")
    assert bool((out[torch.from_numpy(~done).cuda()] == -7.0).all())
    close(state, rs, 1e-6 * ss + 1e-30, "state")
    assert int(fw) == (gpu_lib.FAULT_SEQUENCES if rows > 3 else 0)


def test_steps_follow_a_sequence(gpu_lib):
    """A prompt's final state continued row by row, against the sequence walked whole."""
    import torch

    c = attention_case(21, [80], 4, 2, 64, 64, "f32")
    whole, end = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], final_state=True)
    off = torch.tensor([0, 70], dtype=torch.int64, device="cuda")
    _, state = gpu_lib.linear_attention(c["q"][:70], c["k"][:70], c["v"][:70], c["decay"], off, final_state=True)
    for t in range(70, 80):
        out = gpu_lib.linear_attention_step(c["q"][t:t + 1], c["k"][t:t + 1], c["v"][t:t + 1], c["decay"], state)
        assert float((out[0] - whole[t]).abs().max()) < 1e-3 * float(whole[t].abs().max())
    size = float(end.abs().max())
    assert float((state - end).abs().max()) < 1e-5 * size


def test_offsets_past_32_bits_of_elements(gpu_lib):
    """Rows whose element offsets pass 2^32: the last ones are right, in every operator."""
    import torch

    rows, H, d = 40000, 1, 32
    wide = (1 << 32) // rows + 4096  # elements between rows
    room = torch.zeros(rows * wide, dtype=torch.bfloat16, device="cuda")
    assert (rows - 1) * wide > 1 << 32
    x = room.view(rows, wide)[:, :d]
    rng = np.random.default_rng(2)
    t, _ = up(rng.standard_normal((rows, d)), "bf16")
    x.copy_(t)
    assert torch.equal(gpu_lib.layer_norm(x)[0], gpu_lib.layer_norm(t)[0])
    steps, axis = (torch.from_numpy(a).cuda() for a in gpu_lib.make_rotary(d))
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    assert torch.equal(gpu_lib.rotary(x[:, None], pos, steps, axis), gpu_lib.rotary(t[:, None], pos, steps, axis))
    off = torch.tensor([0, rows], dtype=torch.int64, device="cuda")
    g = torch.full((1,), -0.01, device="cuda")
    a, _ = gpu_lib.linear_attention(x[:, None], x[:, None], x[:, None], g, off)
    b, _ = gpu_lib.linear_attention(t[:, None], t[:, None], t[:, None], g, off)
    assert torch.equal(a, b)


def test_operators_on_another_stream_and_in_a_graph(gpu_lib):
    """A block captured on a side stream and replayed over new inputs, against eager calls."""
    import torch

    c = attention_case(31, [700, 0, 333], 4, 2, 64, 64, "bf16", carry=True)
    x = torch.randn(c["rows"], 256, device="cuda").bfloat16()
    steps, axis = (torch.from_numpy(a).cuda() for a in gpu_lib.make_rotary(48, 1))
    pos = torch.arange(c["rows"], dtype=torch.int32, device="cuda")

    def block():
        y, s, m, r = gpu_lib.layer_norm(x, residual=x, stats=True)
        dx, dw, db = gpu_lib.layer_norm_backward(y, s, None, m, r)
        q = gpu_lib.rotary(c["q"], pos, steps, axis)
        out, end = gpu_lib.linear_attention(q, c["k"], c["v"], c["decay"], c["doff"], initial_state=c["s0"], final_state=True)
        grads = gpu_lib.linear_attention_backward(out, q, c["k"], c["v"], c["decay"], c["doff"], initial_state=c["s0"],
                                                  dfinal_state=c["df"], dinitial_state=True)
        return [y, dx, dw, db, q, out, end, *grads]

    eager = block()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = block()
    for k in range(3):
        if k:
            x.copy_(torch.randn_like(x))
            c["v"].copy_(torch.randn_like(c["v"]))
            eager = block()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, held):
            assert torch.equal(a, b), k
