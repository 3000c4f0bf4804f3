"""Decays of linear attention at their ends: powers far below one.

Tolerance: a power of the decay is one exponential and a few products, each off by 2^-24 or so of itself, wherever the
exponent lies; 2e-6, as for states elsewhere."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [3, 40, 200, 2000])
def test_a_single_row_after_many(gpu_lib, rows, dtype):
    """The state that one row (or the initial state) leaves after many rows of zeros: one power of the decay, down to e^-80."""
    import torch

    from test_gpu_sequence import torch_type

    t, H = torch_type(dtype), 16
    rng = np.random.default_rng(rows)
    g = torch.from_numpy(-rng.uniform(20.0, 80.0, H) / rows).float().cuda()
    off = torch.tensor([0, rows], dtype=torch.int64, device="cuda")
    q = torch.ones(rows, H, 8, dtype=t, device="cuda")
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    k[0], v[0] = 2.0, 0.5
    _, end = gpu_lib.linear_attention(q, k, v, g, off, final_state=True)
    want = torch.exp(g.double() * (rows - 1))[:, None, None]
    assert float((end[0].double() / want - 1.0).abs().max()) < 2e-6
    s0 = torch.full((1, H, 8, 8), 3.0, device="cuda")
    _, end = gpu_lib.linear_attention(q, torch.zeros_like(q), v, g, off, initial_state=s0, final_state=True)
    want = 3.0 * torch.exp(g.double() * rows)[:, None, None]
    assert float((end[0].double() / want - 1.0).abs().max()) < 2e-6
    *_, ds = gpu_lib.linear_attention_backward(q, torch.zeros_like(q), k, v, g, off, initial_state=s0, dfinal_state=s0,
                                               dinitial_state=True)
    assert float((ds[0].double() / want - 1.0).abs().max()) < 2e-6


def test_a_step_of_a_far_decay(gpu_lib):
    import torch

    g = -torch.linspace(0.0, 80.0, 32, device="cuda")
    z = torch.zeros(1, 32, 16, device="cuda")
    state = torch.full((1, 32, 16, 16), 3.0, device="cuda")
    gpu_lib.linear_attention_step(z, z, z, g, state)
    want = 3.0 * torch.exp(g.double())[:, None, None]
    assert float((state[0].double() / want - 1.0).abs().max()) < 2e-6


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [5, 1500])
def test_a_decay_of_nan_is_seen_in_its_head_alone(gpu_lib, rows, dtype):
    """S = nan * S + ...: all of the head's outputs and states are nan, the other heads' keep their bits."""
    import torch

    from test_gpu_sequence import torch_type

    torch.manual_seed(rows)
    t = torch_type(dtype)
    q, k, v = (torch.randn(rows, 3, 32, device="cuda").to(t) for _ in range(3))
    off = torch.tensor([0, rows], dtype=torch.int64, device="cuda")
    g = torch.tensor([-0.1, -0.2, -0.3], device="cuda")
    want, end = gpu_lib.linear_attention(q, k, v, g, off, final_state=True)
    bad = g.clone()
    bad[1] = float("nan")
    out, last = gpu_lib.linear_attention(q, k, v, bad, off, final_state=True)
    for got, ref, head in ((out, want, 1), (last, end, 1)):
        assert bool(got.select(head, 1).isnan().all())
        assert torch.equal(got[:, [0, 2]], ref[:, [0, 2]])
    state = torch.zeros(rows, 3, 32, 32, device="cuda")
    out = gpu_lib.linear_attention_step(q, k, v, bad, state)
    assert bool(out[:, 1].isnan().all()) and bool(state[:, 1].isnan().all())
    assert bool(out[:, [0, 2]].isfinite().all()) and bool(state[:, [0, 2]].isfinite().all())
