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


def poison():
    """NaN in the memory that the next tensors will have."""
    import torch

    held = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 8, 1 << 12, 1 << 14, 1 << 16, 1 << 18, 1 << 20) for _ in range(24)]
    torch.cuda.synchronize()
    del held


def test_training_on_rows_counted_by_the_device(gpu_lib):
    """The voxeliser's full buffers, NaN past the count: gradients of every parameter as from the rows in use alone."""
    import torch

    from test_gpu_encoder import build

    net, feats, coords, offsets, rows = build(gpu_lib, torch.float32, [300, 0, 41], spare=100)
    feats[rows:] = float("nan")
    g = torch.randn(rows, 8, device="cuda")
    grads = []
    for use, count in ((slice(None, rows), None), (slice(None), offsets[-1:])):
        poison()
        out, _ = net(feats[use], coords[use], offsets, row_count=count)
        poison()
        (out[:rows] * g).sum().backward()
        grads.append({n: p.grad.clone() for n, p in net.named_parameters()})
        net.zero_grad(set_to_none=True)
    for n, want in grads[0].items():
        near(grads[1][n], want, 1e-4)  # the products between may be taken in another order


def test_rows_of_no_use_have_gradients_of_zero(gpu_lib):
    import torch

    from paper_2608_15437_amd import encoder

    torch.manual_seed(2)
    n, count = 90, torch.tensor([61], dtype=torch.int64, device="cuda")
    x, r = (torch.randn(n, 64, device="cuda", requires_grad=True) for _ in range(2))
    q, k, v = (torch.randn(n, 2, 32, device="cuda", requires_grad=True) for _ in range(3))
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    steps, axis = (torch.from_numpy(t).cuda() for t in gpu_lib.make_rotary(32))
    off = torch.tensor([0, 20, 61], device="cuda")
    for ins, call in (((x, r), lambda: encoder.norm(x, r, None, None, row_count=count)), ((x,), lambda: encoder.norm(x, None, None, None, row_count=count)[:1]),
                      ((q,), lambda: (encoder.rotary(q, pos, steps, axis, row_count=count),)),
                      ((q, k, v), lambda: encoder.linear_attention(q, k, v, torch.full((2,), -0.1, device="cuda"), off)[:1])):
        poison()
        outs = call()
        assert all(bool((t[61:] == 0).all()) for t in outs)
        poison()
        for t, d in zip(ins, torch.autograd.grad(sum((t * torch.randn_like(t)).sum() for t in outs), ins)):
            assert bool((d[61:] == 0).all()) and bool((d[:61] != 0).any())
