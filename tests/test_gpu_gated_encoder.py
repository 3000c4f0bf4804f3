"""The gated operators together, as the encoder uses them: differentiable forms and a training step of gated blocks against
the same network in plain float64 torch with autograd, rows counted by the device, steps after a sequence, the example.

Tolerances: in fp32 every operator is off by some 1e-6 of its terms and a network of two blocks by a few times that; 2e-4 of
the largest value leaves room for the gates' sums.  Two bf16 blocks round about ten times in a row, 2^-8 of a value each:
4 percent of the largest value, errors adding up as their root."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def turned(x, pos, steps, axis):
    import torch

    turns = torch.tensor([[(int(p[a]) * (int(s) % (1 << 64)) % (1 << 64)) / 2.0 ** 64 for s, a in zip(steps, axis)] for p in pos],
                         dtype=torch.float64) * 2 * math.pi
    c, s = turns.cos()[:, None], turns.sin()[:, None]
    h = len(steps)
    a, b = x[..., :h], x[..., h:2 * h]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * h:]], -1)


def headed(x, w, pos, steps, axis):
    return turned(x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w, pos, steps, axis)


def delta(q, k, v, g, beta, bounds, scale, state=None):
    """Row by row."""
    import torch

    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    out, last = [], []
    for b, (lo, hi) in enumerate(zip(bounds, bounds[1:])):
        S = torch.zeros(q.shape[1], q.shape[2], v.shape[2], dtype=torch.float64) if state is None else state[b]
        for t in range(lo, hi):
            S = S * g[t].exp()[:, None, None]
            e = v[t] - torch.einsum("hk,hkv->hv", k[t], S)
            S = S + torch.einsum("hk,hv->hkv", k[t], beta[t][:, None] * e)
            out.append(scale * torch.einsum("hk,hkv->hv", q[t], S))
        last.append(S)
    return torch.stack(out), torch.stack(last)


def reference(net, feats, coords, offsets):
    import torch

    P = {n: p.detach().double().cpu().requires_grad_(True) for n, p in net.named_parameters()}

    def norm(x, i):
        m = x.mean(1, keepdim=True)
        return (x - m) / ((x - m).square().mean(1, keepdim=True) + 1e-5).sqrt() * P[i + "norm_weight"] + P[i + "norm_bias"]

    x = feats.double().cpu() @ P["embed"]
    bounds = offsets.tolist()
    for i, block in enumerate(net.blocks):
        pre = f"blocks.{i}."
        y = norm(x, pre)
        H, K, d = block.heads, block.kv_heads, block.dim
        q, k, v = (t.unflatten(1, (-1, d)) for t in (y @ P[pre + "qkv"]).split([H * d, K * d, K * d], 1))
        where = coords[:, 1:].tolist(), block.steps.tolist(), block.axis.tolist()
        q, k = headed(q, P[pre + "q_weight"], *where), headed(k, block.k_weight.double().cpu(), *where)
        g, beta = (y @ P[pre + "gates"]).chunk(2, 1)
        g = -P[pre + "rate"].exp() * torch.nn.functional.softplus(g) / math.log(2.0)
        out, _ = delta(q, k, v, g, beta.sigmoid(), bounds, d ** -0.5)
        x = x + out.flatten(1) @ P[pre + "out"]
    return norm(x, "") @ P["head"], P


def build(dtype, lengths, spare=0, **kw):
    import torch

    from paper_2608_15437_amd.encoder import VoxelEncoder

    torch.manual_seed(3)
    net = VoxelEncoder(5, width=64, heads=4, depth=2, out_features=8, dtype=dtype, gated=True, **kw)
    offsets = torch.tensor([0] + lengths).cumsum(0)
    rows = int(offsets[-1])
    feats = torch.randn(rows + spare, 5, device="cuda")
    coords = torch.randint(0, 500, (rows + spare, 4), dtype=torch.int32, device="cuda")
    return net, feats, coords, offsets.cuda(), rows


@pytest.mark.parametrize("dtype,tol", [("float32", 2e-4), ("bfloat16", 4e-2)])
@pytest.mark.parametrize("lengths,kv", [([70, 0, 33], 4), ([150, 1], 2)])
def test_training_step_against_float64(gpu_lib, dtype, tol, lengths, kv):
    import torch

    net, feats, coords, offsets, rows = build(getattr(torch, dtype), lengths, kv_heads=kv)
    g = torch.randn(rows, 8, device="cuda")
    out, _ = net(feats, coords, offsets)
    (out * g).sum().backward()
    ref, P = reference(net, feats.to(getattr(torch, dtype)), coords, offsets)
    (ref * g.double().cpu()).sum().backward()
    assert float((out.double().cpu() - ref).abs().max()) < tol * float(ref.abs().max())
    for n, p in net.named_parameters():
        want = P[n].grad
        assert p.grad is not None, n
        off, size = (p.grad.double().cpu() - want).norm(), want.norm()
        assert float(off) < 2 * tol * float(size), (n, float(off / size))


def test_rows_counted_by_the_device(gpu_lib):
    """The voxeliser's whole buffers, garbage past the count: the same gradients as of the rows in use alone."""
    import torch

    net, feats, coords, offsets, rows = build(torch.float32, [100, 41], spare=60)
    feats[rows:] = float("nan")
    g = torch.randn(rows, 8, device="cuda")
    want, states = net(feats[:rows], coords[:rows], offsets)
    wanted = torch.autograd.grad((want * g).sum(), list(net.parameters()))
    got, after = net(feats, coords, offsets, row_count=offsets[-1:])
    grads = torch.autograd.grad((got[:rows] * g).sum(), list(net.parameters()))
    assert float((got[:rows] - want).abs().max()) < 2e-4 * float(want.abs().max())
    for a, b in zip(after + list(grads), states + list(wanted)):
        assert float((a - b).abs().max()) < 2e-4 * float(b.abs().max())


def test_steps_follow_a_frame(gpu_lib):
    import torch

    net, feats, coords, offsets, rows = build(torch.float32, [40])
    with torch.no_grad():
        want, _ = net(feats, coords, offsets)
        _, states = net(feats[:35], coords[:35], torch.tensor([0, 35], device="cuda"))
        for t in range(35, 40):
            got = net.step(feats[t:t + 1], coords[t:t + 1], states)
            assert float((got[0] - want[t]).abs().max()) < 2e-4 * float(want.abs().max())


def test_differentiable_forms(gpu_lib):
    """Constants among the inputs, states that carry gradients, a second derivative refused."""
    import torch

    from paper_2608_15437_amd import encoder

    torch.manual_seed(4)
    q, k, v = (torch.randn(50, h, 16, device="cuda", requires_grad=True) for h in (4, 2, 2))
    g, beta = (-torch.rand(50, 4, device="cuda")).requires_grad_(), torch.rand(50, 4, device="cuda")
    state = torch.randn(2, 4, 16, 16, device="cuda", requires_grad=True)
    off = torch.tensor([0, 20, 50], device="cuda")
    steps, axis = (torch.from_numpy(t).cuda() for t in gpu_lib.make_rotary(12, 1))
    pos = torch.arange(50, device="cuda", dtype=torch.int32)
    w = torch.full((16,), 0.25, device="cuda", requires_grad=True)
    a, b = encoder.head_norm_rotary(q, k, w, w, pos, steps, axis)
    out, final = encoder.gated_delta(a, b, v, g, beta, off, state)
    h = torch.randn_like(out)
    leaves = q, k, v, g, state, w
    got = torch.autograd.grad((out * h).sum() + final.square().sum(), leaves, create_graph=True)
    with pytest.raises(gpu_lib.MmbevError):
        got[0].sum().backward()
    there = [t.detach().double().cpu().requires_grad_(True) for t in leaves]
    where = pos[:, None].tolist(), steps.tolist(), axis.tolist()
    x, y = headed(there[0], there[5], *where), headed(there[1], there[5], *where)
    ref, last = delta(x, y, there[2], there[3], beta.double().cpu(), [0, 20, 50], 0.25, there[4])
    want = torch.autograd.grad((ref * h.double().cpu()).sum() + last.square().sum(), there)
    for x, y in zip(got, want):
        assert float((x.detach().double().cpu() - y).norm()) < 1e-5 * float(y.norm())


def test_backward_pass_in_a_graph(gpu_lib):
    """Both operators and their gradients captured and replayed with other inputs, eager work between the replays."""
    import torch

    torch.manual_seed(6)
    rows, off = 700, torch.tensor([0, 600, 650, 700], device="cuda")
    steps, axis = (torch.from_numpy(t).cuda() for t in gpu_lib.make_rotary(32, 1))
    pos = torch.arange(rows, device="cuda", dtype=torch.int32)
    w = torch.full((32,), 32 ** -0.5, device="cuda")
    ins = [torch.randn(rows, 2, 32, device="cuda").bfloat16() for _ in range(3)] + [-torch.rand(rows, 2, device="cuda"), torch.rand(rows, 2, device="cuda")]

    def work(q, k, v, g, beta):
        a, b = gpu_lib.head_norm_rotary(q, k, w, w, pos, steps, axis)
        out, final = gpu_lib.gated_delta(a, b, v, g, beta, off, final_state=True)
        dq, dk, *rest = gpu_lib.gated_delta_backward(out, a, b, v, g, beta, off, dfinal_state=final, dinitial_state=True)
        return [out, final, *gpu_lib.head_norm_rotary_backward(dq, dk, q, k, w, w, pos, steps, axis), *rest]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(*ins)
    torch.cuda.current_stream().wait_stream(side)
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        kept = work(*ins)
    with torch.cuda.graph(second, pool=first.pool()):  # shares its memory, workspaces among it
        again = work(*ins)
    for i in range(4):
        for t in ins[:3]:
            t.copy_(torch.randn(rows, 2, 32, device="cuda"))
        want = [t.clone() for t in work(*ins)]
        graph, got = (first, kept) if i % 2 == 0 else (second, again)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_gradients_of_the_modules_in_a_graph(gpu_lib):
    """A block's forward and backward pass captured with no eager graph of its leaves alive, replayed with other rows."""
    import torch

    from paper_2608_15437_amd.encoder import GatedBlock

    torch.manual_seed(8)
    off, rows = torch.tensor([0, 90, 90, 700], device="cuda"), 700
    block = GatedBlock(64, 2, dtype=torch.float32)
    # the library's own sums over rows (torch's may clear their scratch memory by a node that a graph should not hold)
    leaves = [block.norm_weight, block.norm_bias, block.q_weight]
    coords = torch.randint(0, 200, (rows, 4), device="cuda", dtype=torch.int32)
    x, weight = torch.randn(rows, 64, device="cuda"), torch.randn(rows, 64, device="cuda")

    def work():
        y, branch, state = block(x, torch.zeros_like(x), coords, off)
        return [t.detach() for t in (branch, state, *torch.autograd.grad([branch, state], leaves, [weight, state.detach()]))]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work()
    for _ in range(3):
        x.copy_(torch.randn(rows, 64, device="cuda"))
        want = work()
        graph.replay()
        torch.cuda.synchronize()
        # torch's own products may take other tiles in the two: fp32 sums over 700 rows of results off by some steps
        for a, b in zip(got, want):
            assert (a - b).norm() <= 700 * 2 ** -24 * b.norm()


def test_example_trains(gpu_lib):
    import torch

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "voxel_encoder.py")
    spec = importlib.util.spec_from_file_location("voxel_encoder_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, encoded, bev = example.main(["--frames", "2", "--steps", "3", "--width", "64", "--gated"])
    assert all(math.isfinite(x) for x in losses)
    assert bool(torch.isfinite(encoded).all()) and int((bev != 0).sum()) > 0
