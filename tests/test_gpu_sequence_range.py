"""Linear attention in fp16 where values lie far from one: pairs' factors past the type's largest value, gradients and rows
at its smallest ones, columns and rows of different sizes.  Outputs that fit the type are as exact as elsewhere.

Tolerances: those of test_gpu_sequence_precision.py, which follow from the parts of 22 bits that every product takes; near
zero a result is off by at most half the type's smallest step.  States are fp32 and take rows of 22 bits, 2^-22 of each and
the fp32 sums' own rounding: 2e-6 of the absolute terms."""
import numpy as np
import pytest

from oracle import sequence as osq
from test_gpu_sequence import U, attention_case, close, up
from test_gpu_sequence_precision import PARTS

pytestmark = pytest.mark.gpu


def bound(value, size):
    return U["f16"] * np.abs(value) + (PARTS["f16"] + 2e-5) * size + 1e-6 * size.max(initial=0.0) + 1.01 * 2.0 ** -25


def state_bound(size):
    return 2e-6 * size + 1e-45


def times(c, **by):
    """The case with some operands multiplied (by a number or an array that broadcasts)."""
    for name, f in by.items():
        c[name], c[name + "r"] = up(c[name + "r"] * f, "f32" if name in ("s0", "df") else "f16")
    return c


def check(mb, c, what):
    out, end = mb.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], scale=c["scale"], initial_state=c["s0"],
                                   final_state=True)
    ref = osq.linear_attention(c["qr"], c["kr"], c["vr"], c["decayr"], c["offsets"], c["scale"], c["s0r"])
    size = osq.linear_attention(*(np.abs(c[t + "r"]) for t in "qkv"), c["decayr"], c["offsets"], c["scale"],
                                None if c["s0r"] is None else np.abs(c["s0r"]))
    fits = np.abs(ref[0]) < 65000.0
    assert fits.mean() > 0.99, "the case is about results that fit the type"
    close(out[np_mask(fits)], ref[0][fits], bound(ref[0], size[0])[fits], what + ": out")
    close(end, ref[1], state_bound(size[1]), what + ": final state")


def np_mask(m):
    import torch

    return torch.from_numpy(m).cuda()


def check_grads(mb, c, what):
    got = mb.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"], scale=c["scale"],
                                       initial_state=c["s0"], dfinal_state=c["df"], dinitial_state=True)
    args = ("gr", "qr", "kr", "vr")
    ref = osq.linear_attention_backward(*(c[t] for t in args), c["decayr"], c["offsets"], c["scale"], c["s0r"], c["dfr"])
    size = osq.linear_attention_backward(*(np.abs(c[t]) for t in args), c["decayr"], c["offsets"], c["scale"],
                                         *(None if t is None else np.abs(t) for t in (c["s0r"], c["dfr"])))
    for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, size):
        fits = np.abs(r) < 65000.0
        assert fits.mean() > 0.99, "the case is about results that fit the type"
        close(g[np_mask(fits)], r[fits], bound(r, s)[fits], f"{what}: {name}")
    close(got[3], ref[3], state_bound(size[3]), what + ": dinitial")


@pytest.mark.parametrize("lengths,H,kv,kd,vd", [([200, 3], 2, 2, 128, 128), ([1500], 1, 1, 64, 64), ([65, 0, 30], 4, 2, 32, 24)])
def test_pairs_past_the_largest_value(gpu_lib, lengths, H, kv, kd, vd):
    """q and k of one sign and near 100: their products are some 10^4 a dim, far past 65,504 over a head."""
    c = attention_case(700 + kd, lengths, H, kv, kd, vd, "f16")
    c["scale"] = 1.0
    for t in "qk":
        c[t], c[t + "r"] = up(100.0 + c[t + "r"], "f16")
    assert float((c["qr"][0, 0] * c["kr"][0, 0]).sum()) > 2 * 65504.0
    times(c, v=2e-5, g=2e-5)
    check(gpu_lib, c, "large pairs")
    check_grads(gpu_lib, c, "large pairs")


@pytest.mark.parametrize("lengths,H,kv,kd,vd", [([200, 3], 3, 3, 128, 128), ([1500], 3, 3, 64, 64), ([65, 0, 30], 4, 2, 32, 24)])
@pytest.mark.parametrize("small", [1e-2, 1e-4, 1e-6])
def test_small_rows(gpu_lib, lengths, H, kv, kd, vd, small):
    """v and dout of 10^-2 to 10^-6 (where fp16 has a few bits left), the other operands large enough for the results to be
    ordinary numbers."""
    c = attention_case(800 + kd, lengths, H, kv, kd, vd, "f16", carry=True)
    times(c, v=small, g=small, s0=small, k=min(0.1 / small, 1000.0), q=2.0, df=small)
    check(gpu_lib, c, "small rows")
    check_grads(gpu_lib, c, "small rows")


@pytest.mark.parametrize("lengths,H,kv,kd,vd", [([200, 3], 3, 3, 128, 128), ([1500], 3, 3, 64, 64), ([65, 0, 30], 4, 2, 32, 24)])
@pytest.mark.parametrize("small", [1e-2, 1e-4, 1e-6])
def test_small_gradients(gpu_lib, lengths, H, kv, kd, vd, small):
    """The gradients of a loss of that size alone, as training meets them."""
    c = attention_case(850 + kd, lengths, H, kv, kd, vd, "f16", carry=True)
    times(c, g=small, df=small, k=min(0.1 / small, 1000.0), q=2.0)
    check_grads(gpu_lib, c, "small gradients")


def test_pairs_below_the_smallest_value(gpu_lib):
    """Factors of 10^-7 with rows of 10^4."""
    c = attention_case(900, [130], 2, 2, 64, 64, "f16", carry=True)
    times(c, q=1e-4, k=1e-3, v=1e4, g=1.0, s0=10.0, df=1e-3)
    check(gpu_lib, c, "small pairs")
    check_grads(gpu_lib, c, "small pairs")


@pytest.mark.parametrize("lengths", [[130], [900]])
def test_columns_and_rows_of_different_sizes(gpu_lib, lengths):
    """Every column of v a power of two apart over 2^-16 .. 2^4, and a row in ten a thousand times the others."""
    c = attention_case(901, lengths, 2, 2, 64, 64, "f16", carry=True)
    columns = 2.0 ** (4 - np.arange(64) % 21)
    rows = np.where(np.arange(c["rows"]) % 10 == 3, 10.0, 0.01)[:, None, None]
    times(c, v=columns * rows, g=columns[::-1] * rows, s0=columns, df=columns)
    check(gpu_lib, c, "columns")
    check_grads(gpu_lib, c, "columns")
