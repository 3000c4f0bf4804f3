"""The gated operators without a GPU: struct layout, workspace sizes, argument refusals, what the binding looks at.

Every call returns before the library touches the HIP runtime."""
import ctypes
import math

import pytest
import torch

from test_abi_host import mb  # noqa: F401  (the loaded library)
from test_sequence_binding import gpu, lib, OnOtherGpu  # noqa: F401
from test_sequence_host import BAD_ATTENTION, FAKE, LARGE_ATTENTION, attention


def heads(mb, data=FAKE, row=256, head=64):
    return mb.mmbev_heads_t(data, row, head)


def test_struct_layout(mb):  # noqa: F811
    assert ctypes.sizeof(mb.mmbev_head_norm_t) == 40


def head_norm(mb, **kw):
    d = dict(rows=10, heads=4, kv_heads=2, dim=64, rotary_dim=48, dtype=2, weight_dtype=0, layout=0, eps=1e-6)
    d.update(kw)
    return mb.mmbev_head_norm_t(**d)


BAD_HEAD_NORM = [dict(rows=-1), dict(heads=0), dict(kv_heads=0), dict(dim=1), dict(rotary_dim=0), dict(rotary_dim=7),
                 dict(rotary_dim=66), dict(dtype=3), dict(weight_dtype=1), dict(layout=2), dict(eps=-1.0), dict(eps=math.nan),
                 dict(eps=math.inf)]
LARGE_HEAD_NORM = [dict(rows=1 << 31), dict(heads=1025), dict(kv_heads=1025), dict(dim=257)]
F = 1 << 20  # arrays apart


def test_head_norm_refusals(mb):  # noqa: F811
    L = mb.load()
    q, k = heads(mb), heads(mb, FAKE + F, 128)

    def call(desc, q=q, k=k, qw=FAKE, pos=FAKE, stride=3, axes=3, steps=FAKE, axis=FAKE, qo=heads(mb, FAKE + 2 * F), ko=heads(mb, FAKE + 3 * F, 128)):
        return L.mmbev_head_norm_rotary(ctypes.byref(desc), q, k, qw, None, pos, stride, axes, steps, axis, None, qo, ko, None, None)

    for bad in BAD_HEAD_NORM:
        assert call(head_norm(mb, **bad)) == mb.ERR_INVALID_ARG, bad
        assert L.mmbev_head_norm_rotary_backward_workspace_bytes(ctypes.byref(head_norm(mb, **bad))) == 0
    for bad in LARGE_HEAD_NORM:
        assert call(head_norm(mb, **bad)) == mb.ERR_UNSUPPORTED, bad
    for bad in (dict(q=heads(mb, None)), dict(k=heads(mb, None)), dict(qo=heads(mb, None)), dict(ko=heads(mb, None)), dict(q=heads(mb, row=255)),
                dict(q=heads(mb, head=63)), dict(q=heads(mb, FAKE + 1)), dict(qw=FAKE + 2), dict(pos=None), dict(pos=FAKE + 2), dict(stride=2),
                dict(axes=0), dict(axes=9), dict(steps=None), dict(steps=FAKE + 4), dict(axis=None),
                dict(qo=heads(mb, row=512)),  # q's first element, other rows
                dict(qo=heads(mb, FAKE + F, 256)),  # over the keys
                dict(ko=heads(mb, FAKE + 2 * F + 64, 256)),  # over the other result
                dict(qo=k, ko=q)):
        assert call(head_norm(mb), **bad) == mb.ERR_INVALID_ARG, bad
    need = L.mmbev_head_norm_rotary_backward_workspace_bytes(ctypes.byref(head_norm(mb)))
    assert need >= 2 * 64 * 4

    def back(dq=heads(mb, FAKE + 4 * F), dk=heads(mb, FAKE + 5 * F, 128), dy=heads(mb, FAKE + 2 * F), qdw=FAKE, ws=FAKE, nbytes=need):
        return L.mmbev_head_norm_rotary_backward(ctypes.byref(head_norm(mb)), dy, heads(mb, FAKE + 3 * F, 128), q, k, None, None, FAKE, 3, 3,
                                                 FAKE, FAKE, None, dq, dk, qdw, None, None, ws, nbytes, None)

    assert back(nbytes=need - 1) == mb.ERR_WORKSPACE
    assert back(ws=None) == mb.ERR_WORKSPACE
    assert back(ws=FAKE + 128) == mb.ERR_WORKSPACE
    assert back(qdw=FAKE + 2) == mb.ERR_INVALID_ARG
    assert back(dy=heads(mb, None)) == mb.ERR_INVALID_ARG
    assert back(dq=heads(mb, None)) == mb.ERR_INVALID_ARG
    assert back(dq=heads(mb, FAKE + F)) == mb.ERR_INVALID_ARG  # over k
    assert back(dk=heads(mb, FAKE + 4 * F, 128)) == mb.ERR_INVALID_ARG  # over dq


def arrays(mb):
    """q [1000][4][64], k [1000][2][64], v and gates, apart from each other."""
    G = 1 << 24
    return dict(q=heads(mb, FAKE, 256, 64), k=heads(mb, FAKE + G, 128, 64), v=heads(mb, FAKE + 2 * G, 64, 32),
                g=mb.mmbev_rows_t(FAKE + 3 * G, 4), b=mb.mmbev_rows_t(FAKE + 4 * G, 4), out=heads(mb, FAKE + 5 * G, 128, 32))


def test_delta_refusals(mb):  # noqa: F811
    L = mb.load()
    bytes_of = L.mmbev_gated_delta_workspace_bytes

    def call(desc=attention(mb), off=FAKE, init=None, final=None, ws=FAKE, nbytes=1 << 40, **kw):
        a = {**arrays(mb), **kw}
        return L.mmbev_gated_delta(ctypes.byref(desc), a["q"], a["k"], a["v"], a["g"], a["b"], off, init, a["out"], final, None, ws, nbytes, None)

    for bad in BAD_ATTENTION:
        assert call(attention(mb, **bad)) == mb.ERR_INVALID_ARG, bad
        assert bytes_of(ctypes.byref(attention(mb, **bad)), 0) == 0
    for bad in LARGE_ATTENTION:
        assert call(attention(mb, **bad)) == mb.ERR_UNSUPPORTED, bad
    a = arrays(mb)
    for bad in (dict(off=None), dict(off=FAKE + 4), dict(q=heads(mb, None)), dict(v=heads(mb, None)), dict(out=heads(mb, None)),
                dict(g=mb.mmbev_rows_t(None, 4)), dict(b=mb.mmbev_rows_t(None, 4)), dict(g=mb.mmbev_rows_t(FAKE, 3)),
                dict(b=mb.mmbev_rows_t(FAKE, 0)),  # a broadcast row
                dict(g=mb.mmbev_rows_t(FAKE + 2, 4)), dict(init=FAKE + 2), dict(init=FAKE, final=FAKE + 64), dict(out=a["q"]), dict(out=a["v"]),
                dict(out=heads(mb, a["g"].data, 128, 32)), dict(k=heads(mb, FAKE, 128, 63))):
        assert call(**bad) == mb.ERR_INVALID_ARG, bad
    for bad in (dict(q=heads(mb, FAKE, 1 << 31, 64)), dict(g=mb.mmbev_rows_t(FAKE, 1 << 31))):
        assert call(**bad) == mb.ERR_UNSUPPORTED, bad
    need = bytes_of(ctypes.byref(attention(mb)), 0)
    for bad in (dict(nbytes=need - 1), dict(ws=None), dict(ws=FAKE + 64)):
        assert call(**bad) == mb.ERR_WORKSPACE, bad

    def back(desc=attention(mb), ws=FAKE, nbytes=1 << 40, init=None, dfinal=None, dinit=None, **kw):
        H = 1 << 28
        d = dict(dout=heads(mb, FAKE + H, 128, 32), dq=heads(mb, FAKE + 2 * H, 256, 64), dk=heads(mb, FAKE + 3 * H, 128, 64),
                 dv=heads(mb, FAKE + 4 * H, 64, 32), dg=mb.mmbev_rows_t(FAKE + 5 * H, 4), db=mb.mmbev_rows_t(FAKE + 6 * H, 4))
        d = {**arrays(mb), **d, **kw}
        return L.mmbev_gated_delta_backward(ctypes.byref(desc), d["dout"], d["q"], d["k"], d["v"], d["g"], d["b"], FAKE, init, dfinal, d["dq"],
                                            d["dk"], d["dv"], d["dg"], d["db"], dinit, None, ws, nbytes, None)

    need = bytes_of(ctypes.byref(attention(mb)), 1)
    assert need > bytes_of(ctypes.byref(attention(mb)), 0)
    for bad in (dict(nbytes=need - 1), dict(ws=None)):
        assert back(**bad) == mb.ERR_WORKSPACE, bad
    for bad in (dict(dout=heads(mb, None)), dict(dq=a["q"]), dict(dk=a["k"]), dict(dg=a["g"]), dict(db=a["b"]), dict(dg=mb.mmbev_rows_t(None, 4)),
                dict(dg=mb.mmbev_rows_t(a["v"].data, 4)), dict(dv=heads(mb, a["b"].data, 64, 32)), dict(init=FAKE, dinit=FAKE),
                dict(dfinal=FAKE, dinit=FAKE + 64)):
        assert back(**bad) == mb.ERR_INVALID_ARG, bad
    many = attention(mb, rows=(1 << 31) - 1, kv_heads=4)
    wide = dict(k=heads(mb), v=heads(mb, FAKE, 128, 32), dk=heads(mb), dv=heads(mb, FAKE, 128, 32))
    assert back(many, **wide) == mb.ERR_UNSUPPORTED and bytes_of(ctypes.byref(many), 1) == 0 and bytes_of(ctypes.byref(many), 0) > 0

    def step(desc=attention(mb), slots=FAKE, held=1000, state=FAKE + (1 << 30), **kw):
        d = {**arrays(mb), **kw}
        return L.mmbev_gated_delta_step(ctypes.byref(desc), d["q"], d["k"], d["v"], d["g"], d["b"], slots, held, state, d["out"], None, None)

    for bad in (dict(slots=FAKE + 2), dict(held=-1), dict(state=None), dict(state=FAKE + 4), dict(slots=None, held=999), dict(out=a["v"]),
                dict(g=mb.mmbev_rows_t(None, 4)), dict(out=heads(mb, a["b"].data, 128, 32))):
        assert step(**bad) == mb.ERR_INVALID_ARG, bad
    assert step(held=1 << 31) == mb.ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [0, 2])
def test_gates_inside_the_rows_of_a_projection(mb, dtype):  # noqa: F811
    """fp32 gates in the same fp32 rows as q, k and v; a result between them, or over them."""
    L = mb.load()
    # rows of 1024 elements of the type: q, k, v, gates (fp32: 2 elements each of a 16-bit type), out
    size, per = (4, 1) if dtype == 0 else (2, 2)
    at = lambda e: FAKE + e * size  # noqa: E731
    gate = 1024 // per

    def call(out):
        return L.mmbev_gated_delta(ctypes.byref(attention(mb, dtype=dtype)), heads(mb, at(0), 1024, 64), heads(mb, at(256), 1024, 64),
                                   heads(mb, at(384), 1024, 32), mb.mmbev_rows_t(at(448), gate), mb.mmbev_rows_t(at(456), gate), FAKE * 2, None,
                                   heads(mb, at(out), 1024, 32), None, None, FAKE * 4, 0, None)

    assert call(512) == mb.ERR_WORKSPACE  # all else is right
    assert call(464) == mb.ERR_WORKSPACE
    for out in (0, 330, 447, 456, 463 if dtype else 459, 1000):
        assert call(out) == mb.ERR_INVALID_ARG, out


@pytest.mark.parametrize("kv", [1, 2])
def test_binding_of_the_gated_operators(mb, lib, kv):  # noqa: F811
    q, k, v = gpu(torch.zeros(6, 2, 8)), gpu(torch.zeros(6, kv, 8)), gpu(torch.zeros(6, kv, 4))
    g, beta, off = gpu(torch.zeros(6, 2)), gpu(torch.zeros(6, 2)), gpu(torch.tensor([0, 2, 6]))
    state, dout = gpu(torch.zeros(2, 2, 8, 4)), gpu(torch.zeros(6, 2, 4))
    steps, axis, pos = gpu(torch.zeros(4, dtype=torch.int64)), gpu(torch.zeros(4, dtype=torch.uint8)), gpu(torch.zeros(6, dtype=torch.int32))
    mb.gated_delta(q, k, v, g, beta, off, initial_state=state, final_state=True)
    mb.gated_delta_backward(dout, q, k, v, g, beta, off, dinitial_state=gpu(torch.zeros_like(state)))
    mb.gated_delta_step(q, k, v, g, beta, gpu(torch.zeros(7, 2, 8, 4)))
    mb.head_norm_rotary(q, k, None, None, pos, steps, axis)
    mb.head_norm_rotary_backward(q, k, q, k, None, gpu(torch.ones(8)), pos, steps, axis)
    assert [c[0] for c in lib.calls] == ["mmbev_gated_delta", "mmbev_gated_delta_backward", "mmbev_gated_delta_step", "mmbev_head_norm_rotary",
                                         "mmbev_head_norm_rotary_backward"]
    lib.calls.clear()
    host, other = torch.zeros(6, 2), gpu(torch.zeros(6, 2), OnOtherGpu)
    bad = [lambda: mb.gated_delta(q, k, v, host, beta, off), lambda: mb.gated_delta(q, k, v, g, other, off),
           lambda: mb.gated_delta(q, k, v, g.double(), beta, off), lambda: mb.gated_delta(q, k, v, g[:5], beta, off),
           lambda: mb.gated_delta(q, k, v, g, gpu(torch.zeros(2, 6)).t(), off), lambda: mb.gated_delta(q, k[:, :, :4], v, g, beta, off),
           lambda: mb.gated_delta(q, k, v.half(), g, beta, off), lambda: mb.gated_delta(q, k, v, g, beta, off.int()),
           lambda: mb.gated_delta(q, k, v, g, beta, off, initial_state=state.half()),
           lambda: mb.gated_delta(q, k, v, g, beta, off, out=q), lambda: mb.gated_delta_backward(q, q, k, v, g, beta, off),
           lambda: mb.gated_delta_backward(dout, q, k, v, g, beta, off, dlog_decay=gpu(torch.zeros(6, 1))),
           lambda: mb.gated_delta_step(q, k, v, g, beta, state, slots=gpu(torch.zeros(6, dtype=torch.int64))),
           lambda: mb.head_norm_rotary(q, k.half(), None, None, pos, steps, axis), lambda: mb.head_norm_rotary(q, k[:5], None, None, pos, steps, axis),
           lambda: mb.head_norm_rotary(q, k, gpu(torch.ones(7)), None, pos, steps, axis),
           lambda: mb.head_norm_rotary(q, k, gpu(torch.ones(8)), gpu(torch.ones(8).half()), pos, steps, axis),
           lambda: mb.head_norm_rotary(q, k, None, None, pos.long(), steps, axis), lambda: mb.head_norm_rotary(q, k, None, None, pos, steps, axis[:3]),
           lambda: mb.head_norm_rotary(q, k, None, None, pos, steps, axis, k_out=q if kv == 1 else q.half()),
           lambda: mb.head_norm_rotary_backward(q.half(), k, q, k, None, None, pos, steps, axis),
           lambda: mb.head_norm_rotary_backward(q, k, q, k, None, None, pos, steps, axis, dq_weight=gpu(torch.zeros(4)))]
    for i, call in enumerate(bad):
        with pytest.raises(mb.MmbevError):
            call()
        assert not lib.calls, i


def test_written_tensors_raise_autograds_version(mb, lib):  # noqa: F811
    q, k, o = (gpu(torch.zeros(6, 2, 8)) for _ in range(3))
    g, off, state = gpu(torch.zeros(6, 2)), gpu(torch.tensor([0, 6])), gpu(torch.zeros(6, 2, 8, 8))
    before = q._version, state._version, o._version
    steps, axis, pos = gpu(torch.zeros(4, dtype=torch.int64)), gpu(torch.zeros(4, dtype=torch.uint8)), gpu(torch.zeros(6, dtype=torch.int32))
    mb.head_norm_rotary(q, k, None, None, pos, steps, axis, q_out=q)
    mb.gated_delta_step(q, k, k, g, g, state)
    mb.gated_delta(q, k, k, g, g, off, out=o)
    assert q._version > before[0] and state._version > before[1] and o._version > before[2]
