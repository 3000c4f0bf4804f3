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
