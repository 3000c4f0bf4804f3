"""The differentiable operators of encoder.py in every form that they take, against the same formulas in float64 torch.

Tolerance: in fp32 an operator is off by some 1e-6 of its largest terms; 2e-5 of the largest value leaves room for its sums."""
import pytest

pytestmark = pytest.mark.gpu


def near(got, want, tol=2e-5):
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    assert got.shape == want.shape
    assert float((got - want).abs().max()) <= tol * max(float(want.abs().max()), 1e-30)


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("weight", [True, False])
@pytest.mark.parametrize("bias", [True, False])
def test_norm_forms(gpu_lib, residual, weight, bias):
    import torch

    from paper_2608_15437_amd import encoder

    torch.manual_seed(1)
    shapes = [("x", (70, 40), True), ("r", (70, 40), residual), ("w", (40,), weight), ("b", (40,), bias)]
    here = {n: torch.randn(s, device="cuda", requires_grad=True) if use else None for n, s, use in shapes}
    there = {n: None if t is None else t.detach().double().cpu().requires_grad_(True) for n, t in here.items()}
    g, h = torch.randn(70, 40, device="cuda"), torch.randn(70, 40, device="cuda")
    out, total = encoder.norm(here["x"], here["r"], here["w"], here["b"])
    ((out * g).sum() + (total * h).sum()).backward()
    s = there["x"] + there["r"] if residual else there["x"]
    y = (s - s.mean(1, keepdim=True)) / ((s - s.mean(1, keepdim=True)).square().mean(1, keepdim=True) + 1e-5).sqrt()
    y = y * there["w"] if weight else y
    y = y + there["b"] if bias else y
    ((y * g.double().cpu()).sum() + (s * h.double().cpu()).sum()).backward()
    near(out, y)
    near(total, s)
    for n, t in here.items():
        if t is not None:
            near(t.grad, there[n].grad)


def test_norm_of_a_constant_weight_and_of_one_result(gpu_lib):
    import torch

    from paper_2608_15437_amd import encoder

    x, w = torch.randn(9, 16, device="cuda", requires_grad=True), torch.rand(16, device="cuda")
    encoder.norm(x, None, w, None)[1].sum().backward()  # the sum alone: its gradient passes through
    near(x.grad, torch.ones(9, 16))
    assert w.grad is None
