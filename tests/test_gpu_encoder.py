"""The voxel encoder (paper_2608_15437_amd/encoder.py): a training step's outputs and gradients against the same network in
plain float64 torch with autograd, rows counted by the device, steps after a sequence, and the example.

Tolerances: in fp32 every operator is off by some 1e-6 of its terms and a network of two blocks by a few times that; 1e-4 of
the largest value leaves room.  Two bf16 blocks round about ten times in a row, 2^-8 of a value each: 4 percent of the
largest value, errors adding up as their root."""
import importlib.util
import math
import os

import pytest

pytestmark = pytest.mark.gpu


def reference(net, feats, coords, offsets):
    """The encoder in float64, from its parameters: attention by all pairs of a frame's rows."""
    import torch

    P = {n: p.detach().double().cpu().requires_grad_(True) for n, p in net.named_parameters()}

    def norm(x, i):
        m = x.mean(1, keepdim=True)
        return (x - m) / ((x - m).square().mean(1, keepdim=True) + 1e-5).sqrt() * P[i + "norm_weight"] + P[i + "norm_bias"]

    def turn(x, pos, steps, axis):
        turns = torch.tensor([[(int(p[a]) * (int(s) % (1 << 64)) % (1 << 64)) / 2.0 ** 64 for s, a in zip(steps, axis)] for p in pos],
                             dtype=torch.float64) * 2 * math.pi
        c, s = turns.cos()[:, None], turns.sin()[:, None]
        h = len(steps)
        a, b = x[..., :h], x[..., h:2 * h]
        return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * h:]], -1)

    x = feats.double().cpu() @ P["embed"]
    bounds = offsets.tolist()
    for i, block in enumerate(net.blocks):
        pre = f"blocks.{i}."
        rows = norm(x, pre) @ P[pre + "qkv"]
        H, K, d = block.heads, block.kv_heads, block.dim
        q, k, v = rows.split([H * d, K * d, K * d], 1)
        pos, steps, axis = coords[:, 1:].tolist(), block.steps.tolist(), block.axis.tolist()
        q, k = turn(q.unflatten(1, (H, d)), pos, steps, axis), turn(k.unflatten(1, (K, d)), pos, steps, axis)
        k, v = k.repeat_interleave(H // K, 1), v.unflatten(1, (K, d)).repeat_interleave(H // K, 1)
        g = block.log_decay.double().cpu()
        out = []
        for lo, hi in zip(bounds, bounds[1:]):
            t = torch.arange(hi - lo, dtype=torch.float64)
            w = torch.exp(g[:, None, None] * (t[:, None] - t).clamp(min=0)).tril()
            a = (q[lo:hi].transpose(0, 1) @ k[lo:hi].permute(1, 2, 0)) * w * d ** -0.5
            out.append((a @ v[lo:hi].transpose(0, 1)).transpose(0, 1))
        x = x + torch.cat(out).flatten(1) @ P[pre + "out"]
    return norm(x, "") @ P["head"], P


def build(mb, dtype, lengths, spare=0, **kw):
    import torch

    from paper_2608_15437_amd.encoder import VoxelEncoder

    torch.manual_seed(3)
    net = VoxelEncoder(5, width=64, heads=4, depth=2, out_features=8, dtype=dtype, **kw)
    offsets = torch.tensor([0] + lengths).cumsum(0)
    rows = int(offsets[-1])
    feats = torch.randn(rows + spare, 5, device="cuda")
    coords = torch.randint(0, 500, (rows + spare, 4), dtype=torch.int32, device="cuda")
    return net, feats, coords, offsets.cuda(), rows


@pytest.mark.parametrize("dtype,tol", [("float32", 1e-4), ("bfloat16", 4e-2)])
@pytest.mark.parametrize("lengths,kv", [([70, 0, 33], 4), ([600, 1], 2)])
def test_training_step_against_float64(gpu_lib, dtype, tol, lengths, kv):
    import torch

    net, feats, coords, offsets, rows = build(gpu_lib, getattr(torch, dtype), lengths, kv_heads=kv)
    g = torch.randn(rows, 8, device="cuda")
    out, _ = net(feats, coords, offsets)
    (out * g).sum().backward()
    ref, P = reference(net, feats.to(getattr(torch, dtype)), coords, offsets)
    (ref * g.double().cpu()).sum().backward()
    assert float((out.double().cpu() - ref).abs().max()) < tol * float(ref.abs().max())
    for n, p in net.named_parameters():
        want = P[n].grad
        assert p.grad is not None, n
        assert float((p.grad.double().cpu() - want).abs().max()) < tol * float(want.abs().max()), n


def test_rows_counted_by_the_device(gpu_lib):
    """The voxeliser's whole buffers, garbage past the count, against the rows in use alone."""
    import torch

    net, feats, coords, offsets, rows = build(gpu_lib, torch.bfloat16, [300, 41], spare=100)
    feats[rows:] = float("nan")
    with torch.no_grad():
        want, states = net(feats[:rows], coords[:rows], offsets)
        got, after = net(feats, coords, offsets, row_count=offsets[-1:])
    # the products between the operators may be taken in another order for another number of rows
    assert float((got[:rows] - want).abs().max()) < 4e-2 * float(want.abs().max())
    for a, b in zip(after, states):
        assert float((a - b).abs().max()) < 4e-2 * float(b.abs().max())


def test_steps_follow_a_frame(gpu_lib):
    import torch

    net, feats, coords, offsets, rows = build(gpu_lib, torch.float32, [40])
    with torch.no_grad():
        want, _ = net(feats, coords, offsets)
        _, states = net(feats[:35], coords[:35], torch.tensor([0, 35], device="cuda"))
        for t in range(35, 40):
            got = net.step(feats[t:t + 1], coords[t:t + 1], states)
            assert float((got[0] - want[t]).abs().max()) < 1e-4 * float(want.abs().max())


def test_example_trains(gpu_lib):
    import torch

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "voxel_encoder.py")
    spec = importlib.util.spec_from_file_location("voxel_encoder_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    losses, encoded, bev = example.main(["--frames", "3", "--steps", "12", "--width", "64"])
    assert losses[-1] < 0.5 * losses[0]
    assert bool(torch.isfinite(encoded).all()) and int((bev != 0).sum()) > 0


def test_a_state_updated_in_place_is_not_differentiated_as_it_was(gpu_lib):
    import torch

    from paper_2608_15437_amd import encoder

    torch.manual_seed(5)
    q, k, v = (torch.randn(9, 2, 16, device="cuda", requires_grad=True) for _ in range(3))
    decay, off = torch.full((2,), -0.1, device="cuda"), torch.tensor([0, 9], device="cuda")
    state = torch.randn(1, 2, 16, 16, device="cuda")
    out, _ = encoder.linear_attention(q, k, v, decay, off, state)
    with torch.no_grad():
        gpu_lib.linear_attention_step(q[:1], k[:1], v[:1], decay, state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
