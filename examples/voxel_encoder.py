"""From points to an encoded bird's-eye-view map: voxelise a batch of frames, train a small voxel encoder on them, encode
the voxeliser's buffers without waiting for their counts, and scatter the result.

    python examples/voxel_encoder.py [--frames 4] [--steps 20] [--width 128] [--heads 4] [--depth 2] [--gated]

The frames are synthetic; the target is each voxel's mean intensity, smoothed over the voxels before it in its frame.
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import synth  # noqa: E402
from paper_2608_15437_amd import mmbev  # noqa: E402
from paper_2608_15437_amd.encoder import VoxelEncoder  # noqa: E402


def inputs(frames, seed=1):
    """A voxeliser that has run, its features scaled, and the rows in use."""
    vz = mmbev.voxelizer_for_workload(synth.small(seed, frames=frames, max_voxels=4000, dims=(96, 96, 12)), "cuda:0")
    vz.run()
    scale = torch.tensor([0.05, 0.05, 0.5] + [1.0 / 255.0] + [1.0] * (vz.out_feats.shape[1] - 4), device="cuda")[:vz.out_feats.shape[1]]
    return vz, vz.out_feats * scale, int(vz.out_voxel_offsets[-1])


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("frames", 4), ("steps", 20), ("width", 128), ("heads", 4), ("depth", 2)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--gated", action="store_true", help="blocks with the gated delta rule")
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    vz, feats, rows = inputs(a.frames)
    coords, offsets = vz.out_coords, vz.out_voxel_offsets
    print(f"{a.frames} frames, {rows} voxels of {feats.shape[1]} features", flush=True)

    net = VoxelEncoder(feats.shape[1], a.width, a.heads, a.depth, gated=a.gated)
    opt = torch.optim.AdamW(net.parameters(), lr=2e-3)
    frame = coords[:rows, 0].long()
    total = feats[:rows, 3].cumsum(0)
    before = torch.where(frame > 0, total[(offsets[frame] - 1).clamp(min=0)], 0.0)
    target = (total - before) / (torch.arange(rows, device="cuda") - offsets[frame] + 1)
    losses = []
    for step in range(a.steps):
        t = time.perf_counter()
        out, _ = net(feats[:rows], coords[:rows], offsets, max_length=vz.grid.max_voxels)
        loss = (out[:, 0] - target).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.item())
        if step % 5 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {losses[-1]:.4f}, {1e3 * (time.perf_counter() - t):.2f} ms", flush=True)

    with torch.no_grad():
        # the whole buffers, their rows counted by the device
        encoded, states = net(feats, coords, offsets, max_length=vz.grid.max_voxels, row_count=offsets[-1:])
        bev = torch.empty(mmbev.bev_map_shape(vz.grid, encoded.shape[1]), device="cuda")
        mmbev.scatter_to_bev(coords, encoded.contiguous(), offsets, vz.grid, bev)
        # one more voxel for every frame, from the frames' states
        last = (offsets[1:] - 1).clamp(min=0)
        more = net.step(feats[last], coords[last], states)
    torch.cuda.synchronize()
    print(f"map {tuple(bev.shape)}, {int((bev != 0).sum())} values; one more row for {more.shape[0]} frames", flush=True)
    return losses, encoded[:rows], bev


if __name__ == "__main__":
    main()
