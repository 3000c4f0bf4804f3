"""Strides that the sequence operators take, refuse as unsupported, or refuse as wrong.  CPU only: every call here returns
before the library touches the HIP runtime."""
import ctypes

import pytest

from test_abi_host import mb  # noqa: F401  (the loaded library)

BASE = 1 << 44  # never dereferenced


def attention(mb, rows=3):  # noqa: F811
    return mb.mmbev_attention_t(rows=rows, max_length=0, num_sequences=1, heads=2, kv_heads=2, key_dim=8, value_dim=8, dtype=2, scale=1.0,
                                reserved=0)


def test_attention_row_strides(mb):  # noqa: F811
    L = mb.load()
    t = attention(mb)

    def call(which, stride, head=8):
        arrays = [mb.mmbev_heads_t((i + 1) * BASE, 16, 8) for i in range(4)]
        arrays[which] = mb.mmbev_heads_t((which + 1) * BASE, stride, head)
        return L.mmbev_linear_attention(ctypes.byref(t), *arrays[:3], BASE, BASE, None, arrays[3], None, None, None, 0, None)

    def back(which, stride):
        arrays = [mb.mmbev_heads_t((i + 1) * BASE, 16, 8) for i in range(7)]
        arrays[which] = mb.mmbev_heads_t((which + 1) * BASE, stride, 8)
        return L.mmbev_linear_attention_backward(ctypes.byref(t), *arrays[:4], BASE, BASE, None, None, *arrays[4:], None, None, None, 0,
                                                 None)

    for stride, want in ((16, mb.ERR_WORKSPACE), ((1 << 31) - 1, mb.ERR_WORKSPACE), (1 << 31, mb.ERR_UNSUPPORTED),
                         ((1 << 40) - 1, mb.ERR_UNSUPPORTED), (1 << 40, mb.ERR_INVALID_ARG), (-16, mb.ERR_INVALID_ARG)):
        for which in range(4):
            assert call(which, stride) == want, (stride, which)
        for which in range(7):
            assert back(which, stride) == want, (stride, which)


@pytest.mark.parametrize("stride", [1 << 31, (1 << 40) - 1])
def test_arrays_past_the_address_space(mb, stride):  # noqa: F811
    """Rows and strides that each are in range and together pass 64 bits."""
    L = mb.load()
    rows = (1 << 31) - 1 if stride > 1 << 32 else 1 << 30
    big, small = mb.mmbev_heads_t(BASE, stride, 8), mb.mmbev_heads_t(2 * BASE, 16, 8)
    t = mb.mmbev_rotary_t(rows, 2, 8, 8, 0, 0, 0)
    for x, out in ((big, small), (small, big)):
        assert L.mmbev_rotary(ctypes.byref(t), x, BASE, 1 << 39, 1, BASE, BASE, None, out, None, None) == mb.ERR_INVALID_ARG
    n = mb.mmbev_norm_t(rows, 16, 0, 0, 1e-5)
    none = mb.mmbev_rows_t(None, 0)
    for x, out in ((stride, 16), (16, stride)):
        got = L.mmbev_layer_norm(ctypes.byref(n), mb.mmbev_rows_t(BASE, x), none, None, None, None, mb.mmbev_rows_t(2 * BASE, out), none,
                                 None, None, None, None)
        assert got == mb.ERR_INVALID_ARG
