"""Which arrays the sequence operators take to overlap, against sets of addresses.  CPU only: a call that is refused returns
before the library touches the HIP runtime, and one whose arrays are in order ends at its missing workspace."""
import ctypes

import numpy as np
import pytest

from test_abi_host import mb  # noqa: F401  (the loaded library)

BASE = 1 << 40  # never dereferenced


def addresses(at, rows, heads, dim, row, head, size):
    """The bytes of rows of heads: first bytes of elements are enough, all are `size` wide and aligned to it."""
    r, h, c = np.meshgrid(np.arange(rows), np.arange(heads), np.arange(dim), indexing="ij")
    return set((at + size * (r * row + h * head + c)).ravel().tolist())


def layout(rng, rows, heads, dim):
    """Strides of rows of heads, heads inside rows or rows inside heads."""
    if rng.random() < 0.7:
        head = dim + int(rng.integers(0, 2 * dim))
        return (heads - 1) * head + dim + int(rng.integers(0, 3 * dim)), head
    row = dim + int(rng.integers(0, 2 * dim))
    return row, (rows - 1) * row + dim + int(rng.integers(0, 3 * dim))


@pytest.mark.parametrize("seed", range(8))
def test_attention_refuses_shared_elements_and_nothing_else(mb, seed):  # noqa: F811
    L = mb.load()
    rng = np.random.default_rng(seed)
    seen = {True: 0, False: 0}
    for _ in range(600):
        rows, H, kv = int(rng.integers(1, 6)), int(rng.choice([1, 2, 4])), 1
        kd, vd = int(rng.integers(1, 6)), int(rng.integers(1, 6))
        q_row, q_head = layout(rng, rows, H, kd)
        # out like q, or its own layout
        o_row, o_head = (q_row, q_head) if rng.random() < 0.6 else layout(rng, rows, H, vd)
        if rng.random() < 0.5:
            o_row = q_row
        at = int(rng.integers(-40, 40))
        t = mb.mmbev_attention_t(rows=rows, max_length=0, num_sequences=1, heads=H, kv_heads=kv, key_dim=kd, value_dim=vd, dtype=2,
                                 scale=1.0, reserved=0)
        far = mb.mmbev_heads_t(2 * BASE, 64, 64)
        fits = (o_row >= (H - 1) * o_head + vd or o_head >= (rows - 1) * o_row + vd and o_row >= vd or rows == 1) and \
            (H == 1 or o_head >= vd)
        if not fits:
            continue
        got = L.mmbev_linear_attention(ctypes.byref(t), mb.mmbev_heads_t(BASE, q_row, q_head), far, mb.mmbev_heads_t(3 * BASE, 64, 64),
                                       BASE, BASE, None, mb.mmbev_heads_t(BASE + 2 * at, o_row, o_head), None, None, None, 0, None)
        a, b = addresses(0, rows, H, kd, q_row, q_head, 2), addresses(2 * at, rows, H, vd, o_row, o_head, 2)
        shared = bool(a & b)
        spans = max(a) >= min(b) and max(b) >= min(a)
        assert got in (mb.ERR_INVALID_ARG, mb.ERR_WORKSPACE)
        if shared:
            assert got == mb.ERR_INVALID_ARG
        elif not spans or (q_row == o_row and (rows == 1 or q_row >= (H - 1) * q_head + kd and o_row >= (H - 1) * o_head + vd)):
            assert got == mb.ERR_WORKSPACE  # apart, or interleaved in rows of one stride
        seen[shared] += 1
    assert min(seen.values()) > 50


def test_projection_layouts_are_taken(mb):  # noqa: F811
    """out beside q, k and v in one row; q, k and v head by head; heads outside rows."""
    L = mb.load()
    rows, H, d = 1000, 4, 64
    t = mb.mmbev_attention_t(rows=rows, max_length=0, num_sequences=2, heads=H, kv_heads=H, key_dim=d, value_dim=d, dtype=2, scale=1.0,
                             reserved=0)

    def call(*where):
        q, k, v, o = (mb.mmbev_heads_t(BASE + 2 * at, row, head) for at, row, head in where)
        return L.mmbev_linear_attention(ctypes.byref(t), q, k, v, BASE, BASE, None, o, None, None, None, 0, None)

    assert call(*((i * H * d, 4 * H * d, d) for i in range(4))) == mb.ERR_WORKSPACE
    assert call(*((i * d, 4 * H * d, 4 * d) for i in range(4))) == mb.ERR_WORKSPACE
    assert call(*((i * rows * H * d, d, rows * d) for i in range(4))) == mb.ERR_WORKSPACE
    assert call(*((i * rows * d, d, 4 * rows * d) for i in range(4))) == mb.ERR_WORKSPACE
    three = [(i * H * d, 4 * H * d, d) for i in range(3)]
    for at in (0, 1, d, H * d - 1, 2 * H * d + 63, 3 * H * d + 1, 4 * H * d):
        assert call(*three, (at, 4 * H * d, d)) == mb.ERR_INVALID_ARG, at


def test_gradients_may_not_share_memory(mb):  # noqa: F811
    L = mb.load()
    rows, H, d = 100, 2, 8
    t = mb.mmbev_attention_t(rows=rows, max_length=0, num_sequences=1, heads=H, kv_heads=H, key_dim=d, value_dim=d, dtype=2, scale=1.0,
                             reserved=0)
    at = lambda i, off=0: mb.mmbev_heads_t((i + 1) * BASE + 2 * off, H * d, d)  # noqa: E731

    def call(dq=at(4), dk=at(5), dv=at(6)):
        return L.mmbev_linear_attention_backward(ctypes.byref(t), at(0), at(1), at(2), at(3), BASE, BASE, None, None, dq, dk, dv,
                                                 None, None, None, 0, None)

    assert call() == mb.ERR_WORKSPACE
    for kw in (dict(dk=at(4)), dict(dv=at(4)), dict(dv=at(5)), dict(dk=at(4, 8)), dict(dv=at(5, H * d * (rows - 1))),
               dict(dq=at(0)), dict(dq=at(3, 16)), dict(dv=at(2, 4)), dict(dk=at(1, -8))):
        assert call(**kw) == mb.ERR_INVALID_ARG, kw
    side = [mb.mmbev_heads_t(9 * BASE + 2 * i * H * d, 3 * H * d, d) for i in range(3)]
    assert call(*side) == mb.ERR_WORKSPACE


def test_rotary_refuses_shifted_rows_and_heads(mb):  # noqa: F811
    L = mb.load()
    t = mb.mmbev_rotary_t(10, 4, 64, 48, 2, 0, 0)
    x = mb.mmbev_heads_t(BASE, 512, 64)
    for at, row, head in ((64, 512, 64), (512, 512, 64), (-64, 512, 64), (1, 512, 64), (255, 512, 64), (0, 1024, 64), (0, 512, 128),
                          (512 * 9, 512, 64)):
        got = L.mmbev_rotary(ctypes.byref(t), x, 2 * BASE, 3, 3, 2 * BASE, 2 * BASE, None, mb.mmbev_heads_t(BASE + 2 * at, row, head),
                             None, None)
        assert got == mb.ERR_INVALID_ARG, (at, row, head)


def test_layer_norm_refuses_shifted_rows(mb):  # noqa: F811
    L = mb.load()
    n = mb.mmbev_norm_t(10, 64, 2, 0, 1e-5)
    x, none, far = mb.mmbev_rows_t(BASE, 128), mb.mmbev_rows_t(None, 0), mb.mmbev_rows_t(2 * BASE, 64)
    y = mb.mmbev_rows_t(3 * BASE, 64)

    def call(x=x, res=y, out=far, total=none):
        return L.mmbev_layer_norm(ctypes.byref(n), x, res, None, None, None, out, total, None, None, None, None)

    at = lambda base, off, stride: mb.mmbev_rows_t(base + 2 * off, stride)  # noqa: E731
    for kw in (dict(out=at(BASE, 128, 128)), dict(out=at(BASE, 1, 128)), dict(out=at(BASE, -63, 128)), dict(out=at(BASE, 0, 64)),
               dict(out=at(3 * BASE, 64, 64)), dict(total=at(BASE, 63, 128)), dict(total=at(3 * BASE, 8, 64)), dict(total=far),
               dict(total=at(2 * BASE, 32, 64))):
        assert call(**kw) == mb.ERR_INVALID_ARG, kw

    def back(dx, dy=x, s=y, skip=none):
        return L.mmbev_layer_norm_backward(ctypes.byref(n), dy, s, None, BASE, BASE, skip, None, dx, BASE, None, None, None, 0, None)

    for ok in (x, y, far, at(BASE, 64, 128)):
        assert back(ok) == mb.ERR_WORKSPACE
    skip = mb.mmbev_rows_t(5 * BASE, 64)
    assert back(skip, skip=skip) == mb.ERR_WORKSPACE
    for bad in (at(BASE, 128, 128), at(3 * BASE, 64, 64), at(BASE, 0, 64)):
        assert back(bad) == mb.ERR_INVALID_ARG
    assert back(at(5 * BASE, 8, 64), skip=skip) == mb.ERR_INVALID_ARG


def test_step_output_over_shared_keys_and_values_is_refused(mb):  # noqa: F811
    """A step's out may be q's own heads, and k's or v's where no heads share them; refused before anything is launched."""
    L = mb.load()

    def call(q, k, v, out, heads=4, kv=2):
        t = mb.mmbev_attention_t(rows=10, max_length=0, num_sequences=1, heads=heads, kv_heads=kv, key_dim=8, value_dim=8, dtype=2,
                                 scale=1.0, reserved=0)
        return L.mmbev_linear_attention_step(ctypes.byref(t), q, k, v, BASE, None, 10, 9 * BASE, out, None, None)

    at = lambda i, off=0, row=64, head=8: mb.mmbev_heads_t((i + 1) * BASE + 2 * off, row, head)  # noqa: E731
    q, k, v = at(0), at(1), at(2)
    for out in (k, v, at(1, 8), at(2, -8), at(0, 8), at(0, 64), at(0, 4), at(0, 0, 32), at(2, 64 * 9)):
        assert call(q, k, v, out) == mb.ERR_INVALID_ARG
    assert call(q, k, v, at(2, 8), kv=4) == mb.ERR_INVALID_ARG
