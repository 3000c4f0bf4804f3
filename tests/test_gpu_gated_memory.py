"""The gated operators at their largest: the last of 2^31 - 1 rows, head norms past one launch and past 2^32 elements.  What
small calls give for the same rows is compared bit by bit (those are checked against the oracle elsewhere)."""
import pytest

from test_gpu_sequence_memory import MOST, whole_of

pytestmark = pytest.mark.gpu


def test_the_last_rows_that_a_call_may_have(gpu_lib):
    """2^31 - 1 rows of one head of dim 1: a sequence of nearly all of them, and two that end with the last rows, beginning in
    the middle of a chunk.  (The backward call refuses so many.)"""
    import torch

    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB of memory")
    rows, few = (1 << 31) - 1, 70
    q, k, v = (torch.zeros(rows, 1, 1, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    g, beta = (torch.zeros(rows, 1, device="cuda") for _ in range(2))
    torch.manual_seed(2)
    for t in (q, v):
        t[-few:] = torch.randn(few, 1, 1, device="cuda").bfloat16()
    k[-few:], beta[-few:], g[-few:] = 1.0, torch.rand(few, 1, device="cuda"), -torch.rand(few, 1, device="cuda")
    out = torch.full_like(q, 7.0)
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, rows - few, rows - 5, rows], device="cuda")
    gpu_lib.gated_delta(q, k, v, g, beta, offsets, out=out, fault=fault)
    ends = [t[-few:].contiguous() for t in (q, k, v, g, beta)]
    want = gpu_lib.gated_delta(*ends, torch.tensor([0, few - 5, few], device="cuda"))[0]
    assert int(fault) == 0 and torch.equal(out[-few:], want) and bool(want.any())
    assert not bool(out[:-few].any())  # written, every row: zeros
    with pytest.raises(gpu_lib.MmbevError, match="-3"):
        gpu_lib.gated_delta_backward(out, q, k, v, g, beta, offsets, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"), dq=q, dk=k,
                                     dv=v, dlog_decay=g, dbeta=beta)


@pytest.mark.parametrize("rows,heads,kv,dim", [((MOST << 5) + 5, 1, 1, 2), (MOST + 5, 8, 1, 64)])
def test_head_norms_past_one_launch_and_32_bits_of_elements(gpu_lib, rows, heads, kv, dim):
    """Heads of 2: 32 rows a workgroup, so 2^28 rows are a launch.  8 heads of 64: 2^32 elements of queries.  In place, and
    so are the gradients; the last two rows are past the count."""
    import torch

    if torch.cuda.mem_get_info()[0] < 60e9:
        pytest.skip("needs 60 GB of memory")
    n, used = 1 << 18, rows - 2
    torch.manual_seed(3)
    tiles = [torch.randn(n, h, dim, device="cuda").bfloat16() for h in (heads, kv, heads, kv)]
    steps, axis = (torch.from_numpy(a).cuda() for a in gpu_lib.make_rotary(dim))
    pos = torch.arange(n, dtype=torch.int32, device="cuda").repeat((rows + n - 1) // n)[:rows].contiguous()
    w = torch.rand(dim, device="cuda") + 0.5
    count = torch.tensor([used], device="cuda")
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")

    def spread(tile):
        x = torch.empty(rows, *tile.shape[1:], dtype=tile.dtype, device="cuda")
        for a in range(0, rows, n):
            x[a:a + n] = tile[:min(n, rows - a)]
        return x

    def rest(x, tile):  # as it was
        return torch.equal(x[used:], torch.cat([tile, tile])[used % n:used % n + 2])

    q, k = spread(tiles[0]), spread(tiles[1])
    dq, dk = spread(tiles[2]), spread(tiles[3])
    want = gpu_lib.head_norm_rotary_backward(tiles[2], tiles[3], tiles[0], tiles[1], w, w, pos[:n], steps, axis, weight_grads=False)
    got = gpu_lib.head_norm_rotary_backward(dq, dk, q, k, w, w, pos, steps, axis, row_count=count, fault=fault, dq=dq, dk=dk)
    assert whole_of(dq, want[0], used) and whole_of(dk, want[1], used) and rest(dq, tiles[2]) and rest(dk, tiles[3])
    assert bool(torch.isfinite(got[2]).all()) and bool(torch.isfinite(got[3]).all())
    want = gpu_lib.head_norm_rotary(tiles[0], tiles[1], w, w, pos[:n], steps, axis)
    gpu_lib.head_norm_rotary(q, k, w, w, pos, steps, axis, row_count=count, fault=fault, q_out=q, k_out=k)
    assert whole_of(q, want[0], used) and whole_of(k, want[1], used) and rest(q, tiles[0]) and rest(k, tiles[1])
    assert int(fault) == 0
    del q, k, dq, dk, pos
    torch.cuda.empty_cache()
