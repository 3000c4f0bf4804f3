"""The sequence operators without a GPU: struct layouts, the rotary ladder, workspace sizes, argument refusals.

Every call returns before the library touches the HIP runtime."""
import ctypes
import math

import numpy as np
import pytest

from oracle import sequence as osq
from test_abi_host import mb  # noqa: F401  (the loaded library)

FAKE = 1 << 40  # never dereferenced: validation fails first


def test_struct_layouts(mb):
    for t, n in ((mb.mmbev_rows_t, 16), (mb.mmbev_heads_t, 24), (mb.mmbev_norm_t, 24), (mb.mmbev_rotary_ladder_t, 56),
                 (mb.mmbev_rotary_t, 32), (mb.mmbev_attention_t, 48)):
        assert ctypes.sizeof(t) == n, t


@pytest.mark.parametrize("kw", [dict(), dict(axes=3), dict(base=500.0, axes=2), dict(scaling="linear", factor=4.0),
                                dict(scaling="base", factor=8.0, axes=3),
                                dict(scaling="parts", factor=8.0, length=1000.0, slow=1.0, fast=20.0)])
@pytest.mark.parametrize("rot", [6, 48, 64, 130])
def test_rotary_ladder_matches_oracle(mb, rot, kw):
    steps, axis = mb.make_rotary(rot, **kw)
    turns, ax = osq.rotary_ladder(rot, **kw)
    assert np.array_equal(axis, ax)
    got = np.array([(int(v) % (1 << 64)) / 2.0 ** 64 for v in steps])
    assert np.all(np.abs(got - turns) <= 1e-15 * turns + 2.0 ** -64)  # powers in double, then cut to 64 bits


def test_rotary_ladder_refusals(mb):
    good = dict(rotary_dim=16, axes=2, base=100.0)
    mb.make_rotary(**good)
    for bad in (dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=1026), dict(axes=0), dict(axes=9), dict(axes=4, rotary_dim=6),
                dict(base=1.0), dict(base=math.nan), dict(base=math.inf), dict(scaling="linear", factor=0.5),
                dict(scaling="linear", factor=math.nan), dict(scaling="parts", factor=2.0, length=0.0),
                dict(scaling="parts", factor=2.0, length=10.0, slow=2.0, fast=1.0)):
        with pytest.raises(mb.MmbevError):
            mb.make_rotary(**{**good, **bad})


def norm(mb, rows=10, width=64, dtype=2, weight=0, eps=1e-5):
    return mb.mmbev_norm_t(rows, width, dtype, weight, eps)


def test_layer_norm_refusals(mb):
    L = mb.load()
    ok = mb.mmbev_rows_t(FAKE, 64)
    none = mb.mmbev_rows_t(None, 0)

    def call(desc, x=ok, res=none, w=FAKE, out=ok, s=none):
        return L.mmbev_layer_norm(ctypes.byref(desc), x, res, w, None, None, out, s, None, None, None, None)

    assert call(norm(mb, rows=-1)) == mb.ERR_INVALID_ARG
    assert call(norm(mb, width=0)) == mb.ERR_INVALID_ARG
    assert call(norm(mb, width=8193)) == mb.ERR_UNSUPPORTED
    assert call(norm(mb, rows=1 << 31)) == mb.ERR_UNSUPPORTED
    assert call(norm(mb, dtype=3)) == mb.ERR_INVALID_ARG
    assert call(norm(mb, weight=1)) == mb.ERR_INVALID_ARG  # neither float32 nor the rows' type
    for eps in (-1.0, math.nan, math.inf):
        assert call(norm(mb, eps=eps)) == mb.ERR_INVALID_ARG
    assert call(norm(mb), x=none) == mb.ERR_INVALID_ARG
    assert call(norm(mb), out=none) == mb.ERR_INVALID_ARG
    assert call(norm(mb), x=mb.mmbev_rows_t(FAKE, 63)) == mb.ERR_INVALID_ARG
    assert call(norm(mb), res=mb.mmbev_rows_t(FAKE, 0)) == mb.ERR_INVALID_ARG  # a broadcast row
    assert call(norm(mb), x=mb.mmbev_rows_t(FAKE + 1, 64)) == mb.ERR_INVALID_ARG
    assert call(norm(mb), w=FAKE + 2) == mb.ERR_INVALID_ARG
    need = L.mmbev_layer_norm_backward_workspace_bytes(ctypes.byref(norm(mb)))
    assert need >= 2 * 64 * 4
    assert L.mmbev_layer_norm_backward_workspace_bytes(ctypes.byref(norm(mb, width=9000))) == 0

    def back(desc, dy=ok, mean=FAKE, dx=ok, dw=FAKE, ws=FAKE, nbytes=need):
        return L.mmbev_layer_norm_backward(ctypes.byref(desc), dy, ok, None, mean, FAKE, none, None, dx, dw, None, None, ws,
                                           nbytes, None)

    assert back(norm(mb), nbytes=need - 1) == mb.ERR_WORKSPACE
    assert back(norm(mb), ws=None) == mb.ERR_WORKSPACE
    assert back(norm(mb), ws=FAKE + 128) == mb.ERR_WORKSPACE
    assert back(norm(mb), mean=None) == mb.ERR_INVALID_ARG
    assert back(norm(mb), dy=none) == mb.ERR_INVALID_ARG
    assert back(norm(mb), dx=none) == mb.ERR_INVALID_ARG


def test_rotary_refusals(mb):
    L = mb.load()
    ok = mb.mmbev_heads_t(FAKE, 256, 64)

    def call(x=ok, out=ok, pos=FAKE, stride=3, axes=3, steps=FAKE, axis=FAKE, **kw):
        d = dict(rows=10, heads=4, dim=64, rotary_dim=48, dtype=2, layout=0, inverse=0)
        d.update(kw)
        return L.mmbev_rotary(ctypes.byref(mb.mmbev_rotary_t(**d)), x, pos, stride, axes, steps, axis, None, out, None, None)

    for bad in (dict(rows=-1), dict(heads=0), dict(dim=0), dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=66), dict(dtype=-1),
                dict(layout=2), dict(inverse=2), dict(axes=0), dict(axes=9), dict(stride=2), dict(pos=None), dict(pos=FAKE + 2),
                dict(steps=None), dict(steps=FAKE + 4), dict(axis=None), dict(x=mb.mmbev_heads_t(None, 256, 64)),
                dict(x=mb.mmbev_heads_t(FAKE, 255, 64)), dict(x=mb.mmbev_heads_t(FAKE, 256, 63)),
                dict(out=mb.mmbev_heads_t(FAKE, 512, 64)),  # x's first element, other rows
                dict(out=mb.mmbev_heads_t(FAKE + 1, 256, 64))):
        assert call(**bad) == mb.ERR_INVALID_ARG, bad
    assert call(heads=1025) == mb.ERR_UNSUPPORTED
    assert call(rows=1 << 31) == mb.ERR_UNSUPPORTED


def attention(mb, **kw):
    d = dict(rows=1000, max_length=0, num_sequences=2, heads=4, kv_heads=2, key_dim=64, value_dim=32, dtype=2, scale=0.125,
             reserved=0)
    d.update(kw)
    return mb.mmbev_attention_t(**d)


BAD_ATTENTION = [dict(rows=-1), dict(num_sequences=0), dict(num_sequences=65536), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3),
                 dict(key_dim=0), dict(value_dim=0), dict(dtype=7), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf),
                 dict(reserved=1), dict(max_length=-1)]
LARGE_ATTENTION = [dict(rows=1 << 31), dict(heads=258), dict(key_dim=129), dict(value_dim=129)]


def test_attention_refusals(mb):
    L = mb.load()
    q, k, v = mb.mmbev_heads_t(FAKE, 256, 64), mb.mmbev_heads_t(2 * FAKE, 128, 64), mb.mmbev_heads_t(3 * FAKE, 64, 32)
    o = mb.mmbev_heads_t(4 * FAKE, 128, 32)
    need = mb.linear_attention_workspace_bytes(attention(mb))

    def call(q=q, k=k, v=v, decay=FAKE, off=FAKE, init=None, out=o, final=None, ws=FAKE, nbytes=need, **kw):
        return L.mmbev_linear_attention(ctypes.byref(attention(mb, **kw)), q, k, v, decay, off, init, out, final, None, ws, nbytes, None)

    for bad in BAD_ATTENTION:
        assert call(**bad) == mb.ERR_INVALID_ARG, bad
        assert mb.linear_attention_workspace_bytes(attention(mb, **bad)) == 0
    for bad in LARGE_ATTENTION:
        assert call(**bad) == mb.ERR_UNSUPPORTED, bad
        assert mb.linear_attention_workspace_bytes(attention(mb, **bad), True) == 0
    none = mb.mmbev_heads_t(None, 256, 64)
    for bad in (dict(q=none), dict(k=none), dict(v=none), dict(out=none), dict(decay=None), dict(off=None), dict(off=FAKE + 4),
                dict(decay=FAKE + 2), dict(init=FAKE, final=FAKE + 64), dict(out=mb.mmbev_heads_t(FAKE, 128, 32)),
                dict(k=mb.mmbev_heads_t(2 * FAKE, 127, 64)), dict(k=mb.mmbev_heads_t(2 * FAKE + 1, 128, 64))):
        assert call(**bad) == mb.ERR_INVALID_ARG, bad
    for bad in (dict(ws=None), dict(ws=FAKE + 16), dict(nbytes=need - 1)):
        assert call(**bad) == mb.ERR_WORKSPACE, bad

    back = mb.linear_attention_workspace_bytes(attention(mb), True)
    assert back >= need
    shared = attention(mb, heads=8, kv_heads=1)  # more heads share keys than a workgroup takes: room for parts of their sums
    assert mb.linear_attention_workspace_bytes(shared, True) >= mb.linear_attention_workspace_bytes(shared) + 1000 * 4 * (64 + 32)

    def grad(dout=o, dq=mb.mmbev_heads_t(5 * FAKE, 256, 64), dk=mb.mmbev_heads_t(6 * FAKE, 128, 64),
             dv=mb.mmbev_heads_t(7 * FAKE, 64, 32), init=None, dinit=None, nbytes=back, **kw):
        return L.mmbev_linear_attention_backward(ctypes.byref(attention(mb, **kw)), dout, q, k, v, FAKE, FAKE, init, None, dq, dk, dv,
                                                 dinit, None, FAKE, nbytes, None)

    for bad in BAD_ATTENTION:
        assert grad(**bad) == mb.ERR_INVALID_ARG, bad
    for bad in (dict(dout=none), dict(dq=none), dict(dk=none), dict(dv=none), dict(dq=q), dict(dk=k), dict(dv=o),
                dict(init=FAKE, dinit=FAKE)):
        assert grad(**bad) == mb.ERR_INVALID_ARG, bad
    assert grad(nbytes=back - 1) == mb.ERR_WORKSPACE

    def step(slots=FAKE, num=50, state=FAKE, out=o, **kw):
        return L.mmbev_linear_attention_step(ctypes.byref(attention(mb, **kw)), q, k, v, FAKE, slots, num, state, out, None, None)

    for bad in [b for b in BAD_ATTENTION if not {"num_sequences", "max_length"} & set(b)] + [
            dict(slots=FAKE + 2), dict(num=-1), dict(state=None), dict(state=FAKE + 4), dict(out=none), dict(slots=None, num=999)]:
        assert step(**bad) == mb.ERR_INVALID_ARG, bad
    assert step(num=1 << 31) == mb.ERR_UNSUPPORTED


def test_attention_workspace_does_not_shrink_with_the_rows(mb):
    for back in (False, True):
        last = 0
        for rows in (0, 1, 64, 512, 513, 640, 1000, 5000, 120000, 921997):
            need = mb.linear_attention_workspace_bytes(attention(mb, rows=rows), back)
            assert need >= last and need % 256 == 0
            last = need


def test_binding_refuses_what_the_kernels_cannot_take(mb):
    import torch

    x = torch.zeros(4, 8)
    with pytest.raises(mb.MmbevError, match="GPU"):
        mb.layer_norm(x)
    with pytest.raises(mb.MmbevError, match="next to each other"):
        mb._rows("x", x.t())
    with pytest.raises(mb.MmbevError, match="next to each other"):
        mb._heads("q", torch.zeros(4, 8, 2).transpose(1, 2))
    with pytest.raises(mb.MmbevError, match="float32, float16 or bfloat16"):
        mb._dtype_code(x.double())
    with pytest.raises(mb.MmbevError, match="contiguous"):
        mb._vector("log_decay", torch.zeros(8, dtype=torch.float64), torch.float32, 8)


def test_more_workgroups_than_a_launch_may_have_are_refused(mb):
    assert mb.linear_attention_workspace_bytes(attention(mb, num_sequences=65535, heads=128, kv_heads=128)) == 0
    assert mb.linear_attention_workspace_bytes(attention(mb, num_sequences=65535, heads=64, kv_heads=64)) > 0
    L = mb.load()
    q = mb.mmbev_heads_t(FAKE, 256, 64)
    d = attention(mb, rows=(1 << 21) + 1, kv_heads=4, value_dim=64)
    assert L.mmbev_linear_attention_step(ctypes.byref(d), q, q, q, FAKE, FAKE, 50, FAKE, q, None, None) == mb.ERR_UNSUPPORTED
