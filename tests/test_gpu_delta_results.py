"""The gated delta rule's results where only they are asked for: the binding's default, a call without a final state.

A result of 16 bits is an fp32 result rounded once, with a final state and without one.  Tolerances: those of
test_gpu_delta.py, and for one element the same bound with its own terms: U of itself and 32 * 2^-24 of the sum of the
absolute values that it adds up."""
import numpy as np
import pytest

from oracle import gated as og
from test_gpu_delta import CASES, DEEP, LONG, check_backward, check_forward, delta_case, near
from test_gpu_sequence import U, close, up

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "log_decay", "beta")
# either side of the middle between two neighbours of 16 bits, 2^-21 apart: in 16 bits they are 2^-16 apart
LESS, MORE = 1 + 2.0 ** -9 + 2.0 ** -17 - 2.0 ** -22, 1 + 2.0 ** -9 + 2.0 ** -17 + 2.0 ** -22


@pytest.mark.parametrize("state", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_sums_that_cancel(gpu_lib, dtype, state):
    """Results that are small beside their terms show what the terms were held in.  Row 0 reads a state whose rows are in turn
    LESS and MORE with a query of 1/8 and -1/8: the terms add up to 8 in size, the bound is 2^-16, rows of 16 bits would be off
    by 32 / 8 * (2^-16 - 2^-21).  Row 31 of the second sequence reads what 32 rows have written, LESS and MORE in turn, under
    keys of their own: terms of 4, a bound of 2^-17, rates or rows of 16 bits off by 16 / 8 * (2^-16 - 2^-21)."""
    dim, rows = 64, 33
    turns = np.where(np.arange(dim) % 2, -0.125, 0.125)
    values = np.where(np.arange(dim) % 2, MORE, LESS)
    q, k, v, initial = (np.zeros(s) for s in ((rows, 1, dim), (rows, 1, dim), (rows, 1, dim), (2, 1, dim, dim)))
    beta = np.zeros((rows, 1))
    q[0, 0], initial[0, 0] = turns, values[:, None]
    k[0, 0, 0] = 1.0
    for i in range(32):
        k[1 + i, 0, i], beta[1 + i] = 1.0, values[i]
    v[1:], q[32, 0, :32] = 1.0, turns[:32]
    offsets = np.array([0, 1, rows])
    import torch

    on, ref = zip(*(up(a, dtype) for a in (q, k, v)))
    gates, gref = zip(*(up(a) for a in (np.zeros((rows, 1)), beta)))
    start, sref = up(initial)
    got = gpu_lib.gated_delta(*on, *gates, torch.from_numpy(offsets).cuda(), scale=1.0, initial_state=start, final_state=state)[0]
    want = og.gated_delta(*ref, *gref, offsets, 1.0, sref)[0]
    size = og.gated_delta(*map(np.abs, ref), *gref, offsets, 1.0, sref)[0]
    # (what 32 rows have written under keys of their own lies side by side: the absolute sum is the rows' own)
    close(got[[0, 32]], want[[0, 32]], U[dtype] * np.abs(want[[0, 32]]) + DEEP * size[[0, 32]], "out")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES) + len(LONG)))
def test_results_alone(gpu_lib, i, dtype):
    """Against the oracle, and the same bits as beside a final state."""
    import torch

    lengths, H, kv, kd, vd, spare, fused, carry = (CASES + LONG)[i]
    c, ref = delta_case(200 + i, lengths, H, kv, kd, vd, dtype, spare, fused, carry)
    out = torch.full((c["q"].shape[0], H, vd), 7.0, dtype=c["q"].dtype, device="cuda")
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, final = gpu_lib.gated_delta(*(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"], out=out, fault=fault)
    used = c["used"]
    assert final is None and fault.item() == 0 and bool((got[used:] == 7.0).all())
    near(got[:used], og.gated_delta(*(ref[n] for n in (*NAMES, "offsets", "scale", "initial")))[0][:used], U[dtype], "out")
    beside = gpu_lib.gated_delta(*(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"], final_state=True)[0]
    assert torch.equal(got[:used], beside[:used])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_more_than_the_caches_hold(gpu_lib, dtype):
    """70 sequences of 500 rows in rows of 4 KiB, 137 MiB: stored past the caches, the same bits as in calls of ten sequences."""
    import torch

    torch.manual_seed(1)
    rows, H = 35000, 8
    q, k, v = (torch.randn(rows, H, 64, device="cuda") for _ in range(3))
    k = torch.nn.functional.normalize(k, dim=-1)
    q, k, v = (t.to(getattr(torch, {"f16": "float16"}.get(dtype, "bfloat16"))) for t in (q, k, v))
    g, beta = -0.1 * torch.rand(rows, H, device="cuda"), 1.9 * torch.rand(rows, H, device="cuda")
    offsets = torch.arange(0, rows + 1, 500, device="cuda")
    for _ in range(2):
        got = gpu_lib.gated_delta(q, k, v, g, beta, offsets, max_length=500)[0]
        for lo in range(0, rows, 5000):
            part = slice(lo, lo + 5000)
            want = gpu_lib.gated_delta(q[part], k[part], v[part], g[part], beta[part], offsets[:11], max_length=500)[0]
            assert torch.equal(got[part], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H", [(200, 2), (256, 2), (65, 4)])
def test_whole_sequences_longest_first(gpu_lib, dtype, B, H):
    """Up to 256 sequences, more with their heads than the chip takes at once, two of them cut: every row of every one."""
    lengths = np.random.default_rng(B).integers(0, 24, B)
    lengths[B // 3:B // 2] = 12  # ties
    lengths[[1, B - 1]] = 1100, 700
    c, ref = delta_case(300 + B, lengths.tolist(), H, 1, 32, 16, dtype, carry=True)
    used = c["used"]
    got, final = gpu_lib.gated_delta(*(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"], final_state=True)
    want, last = og.gated_delta(*(ref[n] for n in (*NAMES, "offsets", "scale", "initial")))
    near(got[:used], want[:used], U[dtype], "out")
    for b in range(B):
        near(final[b], last[b], U["f32"], f"final state {b}")


@pytest.mark.parametrize("H,kv,lengths", [(90, 45, [600, 30]), (64, 64, [520, 0, 40]), (64, 1, [700])])
def test_heads_that_leave_few_shares(gpu_lib, H, kv, lengths):
    """fp32 heads over 64 wide: two shares of the rows and fewer, where no sequence is cut, and three, where one is."""
    c, ref = delta_case(400 + H, lengths, H, kv, 66, 8, "f32", carry=True)
    check_forward(gpu_lib, c, ref)
    check_backward(gpu_lib, c, ref)
