"""Linear attention in 16-bit types: errors far under the result's own rounding, whatever the call's size says of its rows.

Tolerances.  A result is rounded once (u times itself).  Inside, every factor that a product on the matrix cores takes is
the value's two parts of the type, off by at most u * u = 2^-16 of it in bf16 (fp16: 2^-22): a pair's factor or the state's
copy, and a row on its way into the state, so a pair's share of an output meets at most two of them.  Sums in fp32, decays
as powers of two: the 2e-5 of the absolute terms that test_gpu_sequence.py allows."""
import numpy as np
import pytest

from oracle import sequence as osq
from test_gpu_sequence import TINY, U, attention_case, close, host

pytestmark = pytest.mark.gpu

PARTS = {"f16": 2.0 ** -21, "bf16": 2.0 ** -15}


def tight(value, size, dtype):
    return U[dtype] * np.abs(value) + (PARTS[dtype] + 2e-5) * size + 1e-6 * size.max(initial=0.0) + TINY[dtype]


def forward(mb, c, room=None, **kw):
    """out of the case's rows, in a call whose arrays hold `room` rows."""
    import torch

    q, k, v = (c[t] for t in "qkv")
    if room:
        q, k, v = (torch.cat([t, t.new_full((room - t.shape[0],) + t.shape[1:], float("nan"))]) for t in (q, k, v))
    out, _ = mb.linear_attention(q, k, v, c["decay"], c["doff"], scale=c["scale"], initial_state=c["s0"], **kw)
    return out[:c["used"]]


CASES = [  # lengths, heads, kv_heads, key_dim, value_dim, carry: one part, several, many sequences, each width of the kernels
    ([70], 2, 2, 64, 64, True),
    ([300, 0, 212], 4, 2, 32, 32, False),
    ([1500], 3, 3, 64, 64, True),
    ([700, 0, 64, 1, 900], 2, 1, 128, 128, True),
    ([1100], 2, 2, 100, 36, False),
    ([640, 65], 2, 2, 16, 24, True),
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_outputs_are_rounded_once(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, carry = CASES[i]
    c = attention_case(400 + i, lengths, H, kv, kd, vd, dtype, carry=carry)
    ref, _ = osq.linear_attention(c["qr"], c["kr"], c["vr"], c["decayr"], c["offsets"], c["scale"], c["s0r"])
    size, _ = osq.linear_attention(*(np.abs(c[t + "r"]) for t in "qkv"), c["decayr"], c["offsets"], c["scale"],
                                   None if c["s0r"] is None else np.abs(c["s0r"]))
    bound = tight(ref, size, dtype)
    close(forward(gpu_lib, c), ref, bound, "out")
    # the same rows in a larger buffer, with and without a bound on their number
    close(forward(gpu_lib, c, 4000), ref, bound, "out in a larger buffer")
    close(forward(gpu_lib, c, 4000, max_length=max(lengths)), ref, bound, "out in a larger buffer, lengths bounded")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_gradients_are_rounded_once(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, carry = CASES[i]
    c = attention_case(500 + i, lengths, H, kv, kd, vd, dtype, carry=carry)
    got = gpu_lib.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"], scale=c["scale"],
                                            initial_state=c["s0"], dfinal_state=c["df"])
    args = ("gr", "qr", "kr", "vr")
    ref = osq.linear_attention_backward(*(c[t] for t in args), c["decayr"], c["offsets"], c["scale"], c["s0r"], c["dfr"])
    size = osq.linear_attention_backward(*(np.abs(c[t]) for t in args), c["decayr"], c["offsets"], c["scale"],
                                         *(None if t is None else np.abs(t) for t in (c["s0r"], c["dfr"])))
    for name, g, r, s in zip(("dq", "dk", "dv"), got, ref, size):
        close(g, r, tight(r, s, dtype), name)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_no_further_from_the_definition_than_its_rounding(gpu_lib, dtype):
    """The root mean square error of a long sequence's outputs, against that of the definition rounded to the type: the
    inner errors' share of a result, some 2^-15 of its terms' root sum of squares, is under a tenth of it."""
    import torch

    from test_gpu_sequence import torch_type

    c = attention_case(600, [2000], 2, 2, 64, 64, dtype)
    ref, _ = osq.linear_attention(c["qr"], c["kr"], c["vr"], c["decayr"], c["offsets"], c["scale"])
    once = torch.from_numpy(ref).to(torch_type(dtype)).double().numpy()
    rms = lambda t: float(np.sqrt(np.mean(t * t)))  # noqa: E731
    assert rms(host(forward(gpu_lib, c)) - ref) < 1.1 * rms(once - ref)
