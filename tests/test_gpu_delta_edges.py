"""The gated delta rule where it can go wrong: gates and keys at their limits, ranges that break the contract, NaN beside
other sequences, layouts, sizes of offsets, streams, bounds on the lengths, the same bits twice."""
import numpy as np
import pytest

from oracle import gated as og
from test_gpu_delta import DEEP, check_backward, check_forward, delta_case, near
from test_gpu_sequence import U, up

pytestmark = pytest.mark.gpu

NAMES = ("q", "k", "v", "log_decay", "beta")


def both(mb, c, **kw):
    """Everything that a forward and a backward call write, of a case's tensors."""
    out, final = mb.gated_delta(*(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"], final_state=True, **kw)
    return [out, final, *mb.gated_delta_backward(c["dout"], *(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"],
                                                 dfinal_state=c["dfinal"], dinitial_state=True, **kw)]


def test_gates_at_their_limits(gpu_lib):
    import torch

    c, ref = delta_case(1, [90, 40], 2, 1, 32, 32, "f32", carry=True)
    g = ref["log_decay"]
    g[10] = -np.inf
    g[20:23] = -np.inf
    g[50] = 3.0  # counts as 0
    g[100] = -1e-30
    g[101] = -104.5
    ref["beta"][30] = 2.0
    ref["beta"][31] = -0.5
    c["log_decay"], c["beta"] = torch.from_numpy(g).float().cuda(), torch.from_numpy(ref["beta"]).float().cuda()
    ref["log_decay"], ref["beta"] = c["log_decay"].double().cpu().numpy(), c["beta"].double().cpu().numpy()
    check_forward(gpu_lib, c, ref)
    got = check_backward(gpu_lib, c, ref)
    assert not got[3][50].any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rate", [1.0, 2.0])
def test_one_key_for_all_rows(gpu_lib, dtype, rate):
    """Every row corrects what the row before wrote.  For one key of length 1 the inverse of a chunk's system 1 + beta L
    (L all ones under the diagonal; check: L sum_m (1 - beta)^m steps) has the entries -beta (1 - beta)^(i-j-1) under its
    diagonal: for beta 1 a single -1 beside the diagonal, rows of absolute sum 2; for beta 2 +-2 everywhere, rows of up to
    1 + 31 * 2 = 63.  That is how far a rounding of a row's right side reaches, in any solution of the system, so the
    roundings' bound is multiplied by it."""
    reach = 2 if rate == 1.0 else 63
    c, ref = delta_case(2, [200], 1, 1, 64, 64, dtype, carry=True)
    key = np.zeros(64)
    key[:4] = 0.5  # exact in every type, length 1
    c["k"], ref["k"] = up(np.broadcast_to(key, (200, 1, 64)).copy(), dtype)
    c["beta"], ref["beta"] = up(np.full((200, 1), rate))
    c["log_decay"], ref["log_decay"] = up(np.full((200, 1), -2.0 ** -7))
    out, final = gpu_lib.gated_delta(*(c[n] for n in NAMES), c["offsets"], scale=0.37, initial_state=c["initial"], final_state=True)
    want, last = og.gated_delta(*(ref[n] for n in NAMES), ref["offsets"], 0.37, ref["initial"])
    near(out, want, U[dtype], "out", deep=reach * DEEP)
    near(final, last, 0.0, "final", deep=reach * DEEP)


def test_values_far_from_one(gpu_lib):
    """States beyond fp16's range and gradients under it."""
    for dtype, size in (("f16", 3e4), ("bf16", 1e20), ("f32", 1e15), ("f16", 1e-3)):
        c, ref = delta_case(3, [120], 2, 2, 64, 32, dtype, carry=True)
        c["v"], ref["v"] = up(ref["v"] * size / 4, dtype)
        c["initial"], ref["initial"] = up(ref["initial"] * size)
        c["q"], ref["q"] = up(ref["q"] * (1e-3 if size < 1e5 else 1.0), dtype)
        check_forward(gpu_lib, c, ref)


@pytest.mark.parametrize("offsets,used", [([0, 50, 20, 300], 100), ([5, 60, 100], 100), ([0, -3, 70], 70), ([0, 1 << 40], 100), ([0, 90, 90, 30], 30)])
def test_bad_offsets_are_clamped_and_reported(gpu_lib, offsets, used):
    import torch

    c, _ = delta_case(4, [100], 2, 1, 16, 16, "bf16", spare=40)
    c["offsets"] = torch.tensor(offsets, device="cuda")
    n = len(offsets) - 1
    c["initial"] = c["dfinal"] = None
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    room = torch.full((200, 2, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    gpu_lib.gated_delta(*(c[m][:100] for m in NAMES), c["offsets"], out=room[50:150], fault=fault)
    assert fault.item() & gpu_lib.FAULT_SEQUENCES
    assert bool((room[:50] == 7.0).all()) and bool((room[50 + used:] == 7.0).all())
    fault.zero_()
    dq = torch.full_like(room, 7.0)
    got = gpu_lib.gated_delta_backward(c["dout"][:100], *(c[m][:100] for m in NAMES), c["offsets"], dq=dq[50:150], dinitial_state=True, fault=fault)
    assert fault.item() & gpu_lib.FAULT_SEQUENCES and got[5].shape[0] == n
    assert bool((dq[:50] == 7.0).all()) and bool((dq[50 + used:] == 7.0).all())


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["q", "k", "v", "log_decay", "beta", "dout"])
@pytest.mark.parametrize("lengths", [[40, 70, 33], [1400, 900, 700]])
def test_sequences_do_not_see_each_others_nan(gpu_lib, bad, where, lengths):
    import torch

    c, _ = delta_case(5, lengths, 2, 2, 32, 64, "bf16", carry=True)
    want = both(gpu_lib, c)
    row = lengths[0] + lengths[1] // 2
    x = c[where].clone()
    x[row, 1] = bad
    got = both(gpu_lib, {**c, where: x})
    lo, hi = lengths[0], lengths[0] + lengths[1]
    for i, (a, b) in enumerate(zip(got, want)):
        per_row = i in (0, 2, 3, 4, 5, 6)
        spans = [slice(0, lo), slice(hi, None)] if per_row else [slice(0, 1), slice(2, 3)]
        for s in spans:
            assert torch.equal(a[s], b[s]), i
        middle = slice(lo, hi) if per_row else slice(1, 2)
        assert torch.equal(a[middle, 0], b[middle, 0]), i  # the other head


def test_no_rows_and_many_sequences(gpu_lib):
    import torch

    c, ref = delta_case(6, [0, 0], 2, 1, 16, 24, "f32", carry=True)
    got = both(gpu_lib, c)
    assert torch.equal(got[1], c["initial"]) and torch.equal(got[7], c["dfinal"])
    rng = np.random.default_rng(7)
    lengths = rng.integers(0, 4, 1500).tolist()  # more than are looked through for cuts
    lengths[700] = 600
    c, ref = delta_case(7, lengths, 1, 1, 8, 8, "bf16")
    check_forward(gpu_lib, c, ref)
    check_backward(gpu_lib, c, ref)
    # and 300 that are cut and ordered by their length
    lengths = rng.integers(0, 40, 300).tolist()
    lengths[17] = 3000
    c, ref = delta_case(8, lengths, 2, 2, 16, 16, "f16", carry=True)
    check_forward(gpu_lib, c, ref)
    check_backward(gpu_lib, c, ref)


def test_heads_before_rows(gpu_lib):
    """[heads][rows][dim] arrays seen as [rows][heads][dim], gates as columns of another matrix: the same bits."""
    import torch

    c, _ = delta_case(9, [600, 90], 4, 2, 64, 64, "bf16", carry=True)
    want = both(gpu_lib, c)
    d = {**c, **{n: c[n].transpose(0, 1).contiguous().transpose(0, 1) for n in ("q", "k", "v", "dout")}}
    wide = torch.full((690, 11), 7.0, device="cuda")
    wide[:, 1:5], wide[:, 6:10] = c["log_decay"], c["beta"]
    d["log_decay"], d["beta"] = wide[:, 1:5], wide[:, 6:10]
    for a, b in zip(both(gpu_lib, d), want):
        assert torch.equal(a, b)


def test_the_same_bits_whatever_the_bound_on_lengths_of_a_whole_sequence(gpu_lib):
    """Twice the same; a bound that is too small sizes the launches, and longer sequences are computed too."""
    import torch

    c, ref = delta_case(10, [900, 700], 2, 1, 64, 32, "f32", carry=True)
    one, two = both(gpu_lib, c), both(gpu_lib, c)
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    check_forward(gpu_lib, c, ref, max_length=100)
    check_backward(gpu_lib, c, ref, max_length=100)


def test_offsets_past_32_bits_of_elements(gpu_lib):
    """Rows a million elements apart in one buffer of 2^32.5 elements: the same bits as next to each other."""
    import torch

    rows, apart = 6000, 1 << 20
    c, _ = delta_case(11, [5000, 1000], 1, 1, 32, 32, "bf16")
    want = both(gpu_lib, c)
    room = torch.empty(rows * apart, dtype=torch.bfloat16, device="cuda").view(rows, apart)
    d = dict(c)
    for i, n in enumerate(("q", "k", "v", "dout")):
        d[n] = room[:, 64 * i:64 * i + 32].view(rows, 1, 32)
        d[n].copy_(c[n])
    got = both(gpu_lib, d)
    out = room[:, 512:544].view(rows, 1, 32)
    gpu_lib.gated_delta(*(d[n] for n in NAMES), d["offsets"], scale=0.37, out=out, final_state=True)
    assert torch.equal(out, want[0])
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_on_another_stream_and_with_a_given_workspace(gpu_lib):
    import torch

    c, _ = delta_case(12, [800, 100], 2, 2, 64, 64, "f16", carry=True)
    want = both(gpu_lib, c)
    desc = gpu_lib.mmbev_attention_t(900, 0, 2, 2, 2, 64, 64, gpu_lib.F16, 0.37, 0)
    need = gpu_lib.gated_delta_workspace_bytes(desc, True)
    assert need >= gpu_lib.gated_delta_workspace_bytes(desc)
    side = torch.cuda.Stream()
    workspace = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN and the largest numbers: nothing is taken from it
    torch.cuda.synchronize()
    got = both(gpu_lib, c, workspace=workspace, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_steps_in_slots_out_of_range(gpu_lib):
    import torch

    c, _ = delta_case(13, [4], 2, 1, 16, 16, "f32")
    state = torch.randn(3, 2, 16, 16, device="cuda")
    before, fault = state.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full((4, 2, 16), 7.0, device="cuda")
    gpu_lib.gated_delta_step(*(c[n] for n in NAMES), state, torch.tensor([2, -1, 3, 1 << 30], dtype=torch.int32, device="cuda"), out=out, fault=fault)
    assert fault.item() & gpu_lib.FAULT_SEQUENCES
    assert torch.equal(state[:2], before[:2]) and not torch.equal(state[2], before[2])
    assert bool((out[1:] == 7.0).all()) and not bool((out[0] == 7.0).any())
    # in place: a row's result over its query, its key and its value
    q, k, v = (torch.randn(3, 2, 16, device="cuda") for _ in range(3))
    g, beta = c["log_decay"][:3], c["beta"][:3]
    want = gpu_lib.gated_delta_step(q, k, v, g, beta, before.clone())
    for i in range(3):
        x = [t.clone() for t in (q, k, v)]
        assert torch.equal(gpu_lib.gated_delta_step(*x, g, beta, before.clone(), out=x[i]), want)
