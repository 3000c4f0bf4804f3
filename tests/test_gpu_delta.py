"""The gated delta rule, through the binding, against the oracle's float64 definition.

With keys of length 1 and beta in 0..2 a row's map of the state is a contraction, so errors do not grow from row to row.
Results are rounded once to their type (by at most U of themselves, U half a step); everything before that is as exact
as fp32: sums of up to 128 products, a system of 32 rows, decays, some 32 roundings of 2^-24 deep in all, so an array is
off by at most U + 32 * 2^-24 of its 2-norm.  The gates' gradients are sums of terms of either sign, whose sizes count."""
import numpy as np
import pytest

from oracle import gated as og
from test_gpu_sequence import U, host, strided, up

pytestmark = pytest.mark.gpu

DEEP = 32 * 2.0 ** -24

# lengths, heads, kv_heads, key_dim, value_dim, spare rows, rows in one projection, states carried
CASES = [([1], 1, 1, 1, 1, 0, False, False), ([3, 0, 2], 2, 1, 8, 8, 0, False, True), ([33, 1, 31, 32, 64], 2, 2, 64, 64, 5, True, True),
         ([70, 130], 4, 2, 32, 32, 0, True, False), ([0, 40, 0], 3, 1, 33, 17, 9, False, True), ([100, 7], 2, 2, 128, 128, 1, True, True),
         ([65], 2, 1, 100, 9, 0, False, True), ([48, 17], 1, 1, 5, 120, 3, False, True), ([16, 15], 8, 2, 64, 128, 0, True, False),
         ([90], 2, 2, 128, 48, 0, False, True), ([0], 1, 1, 16, 16, 0, False, True), ([50, 20], 2, 2, 48, 64, 2, True, True),
         ([64, 63], 2, 1, 96, 127, 0, False, False)]
# cut into parts
LONG = [([3000, 40, 900], 2, 1, 64, 64, 10, True, True), ([5000], 1, 1, 33, 40, 0, False, True), ([2100, 700], 4, 4, 128, 128, 0, True, True),
        ([2500], 2, 2, 32, 128, 0, False, False), ([1500, 0, 1200], 3, 3, 128, 64, 0, False, True)]


def delta_case(seed, lengths, H, kv, kd, vd, dtype, spare=0, fused=False, carry=False, most_beta=1.0):
    import torch

    rng = np.random.default_rng(seed)
    rows = sum(lengths) + spare
    offsets = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
    arrays = {"q": rng.standard_normal((rows, H, kd)), "k": rng.standard_normal((rows, kv, kd)), "v": rng.standard_normal((rows, kv, vd)),
              "dout": rng.standard_normal((rows, H, vd))}
    # rounded keys are at most 1 + 2^-8 long: beta under 1.98 keeps the map a contraction
    arrays["k"] /= np.linalg.norm(arrays["k"], axis=-1, keepdims=True)
    c = {"offsets": torch.from_numpy(offsets).cuda(), "lengths": lengths, "used": int(offsets[-1]), "dtype": dtype}
    ref = {"offsets": offsets, "scale": 0.37}
    for name, a in arrays.items():
        c[name], ref[name] = up(a, dtype)
    if fused and rows:  # q, k and v side by side in a row
        row = torch.cat([c[n].flatten(1) for n in ("q", "k", "v")], 1)
        at = 0
        for n in ("q", "k", "v"):
            width = c[n][0].numel()
            c[n] = row[:, at:at + width].view(rows, *c[n].shape[1:])
            at += width
    reach = rng.uniform(1.0, 10.0, H)
    gates = -(2.0 ** -reach) * rng.uniform(0.2, 2.0, (rows, H))
    if rows > 4:
        gates[rows // 2] = -200.0  # nothing left
        gates[rows // 3, 0] = 0.0
    c["log_decay"], ref["log_decay"] = up(gates)
    c["beta"], ref["beta"] = up(rng.uniform(0.0, most_beta, (rows, H)))
    if rows > 3:
        c["beta"][1] = 0.0
        ref["beta"][1] = 0.0
    for name in ("initial", "dfinal"):
        c[name], ref[name] = up(rng.standard_normal((len(lengths), H, kd, vd))) if carry else (None, None)
    return c, ref


def near(got, ref, u, what, more=0.0, deep=DEEP):
    got = host(got)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), what
    off, size = np.linalg.norm(got - ref), np.linalg.norm(ref) + more
    # fp16 has steps of 2^-24 next to zero: half of one an element, whatever its size
    tiny = 2.0 ** -25 * got.size ** 0.5 if u == U["f16"] else 1e-30
    assert off <= (u + deep) * size + tiny, f"{what}: {off / max(size, 1e-300):.3g} of its norm, {(u + deep):.3g} allowed"


def check_forward(mb, c, ref, **kw):
    import torch

    used, u = c["used"], U[c["dtype"]]
    out = torch.full((*c["q"].shape[:2], c["v"].shape[2]), 7.0, dtype=c["q"].dtype, device="cuda")
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    got, final = mb.gated_delta(c["q"], c["k"], c["v"], c["log_decay"], c["beta"], c["offsets"], scale=ref["scale"], initial_state=c["initial"],
                                final_state=True, out=out, fault=fault, **kw)
    want, last = og.gated_delta(*(ref[n] for n in ("q", "k", "v", "log_decay", "beta", "offsets", "scale", "initial")))
    assert fault.item() == 0
    near(got[:used], want[:used], u, "out")
    assert bool((got[used:] == 7.0).all())
    near(final, last, U["f32"], "final state")
    return got, final


def check_backward(mb, c, ref, **kw):
    import torch

    used, u = c["used"], U[c["dtype"]]
    outs = {n: torch.full_like(c[m].contiguous(), 7.0) for n, m in (("dq", "q"), ("dk", "k"), ("dv", "v"), ("dlog_decay", "log_decay"), ("dbeta", "beta"))}
    got = mb.gated_delta_backward(c["dout"], c["q"], c["k"], c["v"], c["log_decay"], c["beta"], c["offsets"], scale=ref["scale"],
                                  initial_state=c["initial"], dfinal_state=c["dfinal"], dinitial_state=True, **outs, **kw)
    want = og.gated_delta_backward(*(ref[n] for n in ("dout", "q", "k", "v", "log_decay", "beta", "offsets", "scale", "initial", "dfinal")))
    for name, x, y in zip(("dq", "dk", "dv"), got, want):
        near(x[:used], y[:used], u, name)
        assert bool((x[used:] == 7.0).all())
    group = ref["q"].shape[1] // ref["k"].shape[1]
    q, k, dq, dk = ref["q"][:used], ref["k"][:used].repeat(group, 1), want[0][:used], want[1][:used].repeat(group, 1)
    terms = np.linalg.norm(np.abs(q * dq).sum(-1) + np.abs(k * dk).sum(-1))
    near(got[3][:used], want[3][:used], U["f32"], "dlog_decay", terms)
    near(got[4][:used], want[4][:used], U["f32"], "dbeta")
    assert bool((got[3][used:] == 7.0).all()) and bool((got[4][used:] == 7.0).all())
    near(got[5], want[5], U["f32"], "dinitial")
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_delta(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, spare, fused, carry = CASES[i]
    check_forward(gpu_lib, *delta_case(i, lengths, H, kv, kd, vd, dtype, spare, fused, carry))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_delta_backward(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, spare, fused, carry = CASES[i]
    check_backward(gpu_lib, *delta_case(50 + i, lengths, H, kv, kd, vd, dtype, spare, fused, carry))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("i", range(len(LONG)))
def test_delta_in_parts(gpu_lib, i, dtype):
    lengths, H, kv, kd, vd, spare, fused, carry = LONG[i]
    c, ref = delta_case(100 + i, lengths, H, kv, kd, vd, dtype, spare, fused, carry, most_beta=1.9)
    check_forward(gpu_lib, c, ref)
    check_backward(gpu_lib, c, ref)


# rows, heads, kv_heads, key_dim, value_dim, states
STEP = [(1, 1, 1, 1, 1, 1), (5, 4, 2, 64, 64, 9), (3, 2, 2, 128, 128, 3), (7, 3, 1, 33, 17, 20), (2, 8, 8, 100, 30, 4), (4, 2, 1, 20, 127, 5),
        (64, 8, 4, 64, 64, 64), (3, 2, 2, 128, 32, 6), (2, 1, 1, 128, 64, 2)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,H,kv,kd,vd,slots", STEP)
def test_delta_step(gpu_lib, rows, H, kv, kd, vd, slots, dtype):
    import torch

    c, ref = delta_case(rows * 7 + kd, [rows], H, kv, kd, vd, dtype)
    state, sref = up(np.random.default_rng(rows).standard_normal((slots, H, kd, vd)))
    names = np.random.default_rng(1).permutation(slots)[:rows].astype(np.int32)
    if rows > 2:
        names[1] = -1
    q = strided(c["q"], 3, 1) if kd % 2 else c["q"]
    out = torch.full((rows, H, vd), 7.0, dtype=c["q"].dtype, device="cuda")
    gpu_lib.gated_delta_step(q, c["k"], c["v"], c["log_decay"], c["beta"], state, torch.from_numpy(names).cuda(), scale=0.37, out=out)
    want, after = og.gated_delta_step(*(ref[n] for n in ("q", "k", "v", "log_decay", "beta")), sref, names, 0.37)
    there = names >= 0
    near(out[torch.from_numpy(there).cuda()], want[there], U[dtype], "out")
    assert bool((out[torch.from_numpy(~there).cuda()] == 7.0).all())
    near(state, after, U["f32"], "state")


def test_delta_gradient_against_differences(gpu_lib):
    import torch

    c, ref = delta_case(7, [45, 30], 2, 1, 24, 16, "f32", carry=True)
    c["log_decay"].clamp_(min=-3.0)
    names = ("q", "k", "v", "log_decay", "beta", "initial")
    rng = np.random.default_rng(8)

    def loss(x):
        out, final = gpu_lib.gated_delta(*(x[n] for n in names[:5]), c["offsets"], scale=0.37, initial_state=x["initial"], final_state=True)
        return float((out.double() * c["dout"]).sum() + (final.double() * c["dfinal"]).sum())

    grads = gpu_lib.gated_delta_backward(c["dout"], *(c[n] for n in names[:5]), c["offsets"], scale=0.37, initial_state=c["initial"],
                                         dfinal_state=c["dfinal"], dinitial_state=True)
    for n, g in zip(names, grads):
        at = torch.from_numpy(rng.standard_normal(c[n].shape)).float().cuda()
        if n == "log_decay":
            at = at * (c[n] < -1e-2)  # the step stays under 0
        h = 2.0 ** -9
        d = (loss({**c, n: c[n] + h * at}) - loss({**c, n: c[n] - h * at})) / (2 * h)
        # third derivatives times h^2, and the roundings of some 4,000 results of size 1 over 2 h
        assert abs(d - float((g.double() * at).sum())) < 1e-3 * float((g.double() * at).norm()) * 40 + 1e-2, n


def test_delta_state_carries_over_calls(gpu_lib):
    """A sequence in two calls is the sequence in one; steps go on from there."""
    import torch

    c, ref = delta_case(9, [200], 2, 2, 64, 64, "f32", carry=True)
    one, last = gpu_lib.gated_delta(c["q"], c["k"], c["v"], c["log_decay"], c["beta"], c["offsets"], initial_state=c["initial"], final_state=True)
    state, parts = c["initial"], []
    for lo, hi in ((0, 77), (77, 190)):
        o, state = gpu_lib.gated_delta(*(c[n][lo:hi] for n in ("q", "k", "v", "log_decay", "beta")), torch.tensor([0, hi - lo]).cuda(),
                                       initial_state=state, final_state=True)
        parts.append(o)
    for t in range(190, 200):
        parts.append(gpu_lib.gated_delta_step(*(c[n][t:t + 1] for n in ("q", "k", "v", "log_decay", "beta")), state))
    near(torch.cat(parts), host(one), 0.0, "out")
    near(state, host(last), 0.0, "state")
