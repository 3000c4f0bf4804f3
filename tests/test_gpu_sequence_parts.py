"""Linear attention over many sequences: which workgroup takes which part of which sequence.

Sequences longer than two shares of the rows are cut; where there are more sequences and heads than the chip takes at
once, the others go longest first (up to 256 sequences) or in order; among more than 1,024 none is cut.  Every output row
and final state is checked, so a part left out or taken twice shows.  Tolerances: those of test_gpu_sequence.py."""
import numpy as np
import pytest

from test_gpu_sequence import attention_case, check_backward, check_forward

pytestmark = pytest.mark.gpu


def lengths(seed, B, most, long=()):
    rng = np.random.default_rng(seed)
    n = rng.integers(0, most, B)
    n[rng.integers(0, B, B // 4)] = most // 2  # ties
    n[rng.integers(0, B, B // 8)] = 0
    for i, x in long:
        n[i] = x
    return n.tolist()


CASES = [  # sequences, heads, kv_heads, dim, lengths
    (200, 8, 8, 32, lengths(1, 200, 30)),                                   # longest first, none cut
    (200, 8, 2, 16, lengths(2, 200, 20, [(0, 700), (77, 1500), (199, 900)])),  # some cut, the rest longest first
    (64, 16, 16, 8, lengths(3, 64, 40, [(63, 800)])),                       # one round of lanes
    (65, 16, 4, 16, lengths(4, 65, 40, [(64, 600), (0, 601)])),             # one lane of a second
    (256, 4, 4, 32, lengths(5, 256, 16, [(255, 640)])),                     # the most that are ordered
    (257, 4, 4, 32, lengths(6, 257, 16, [(256, 640), (3, 530)])),           # in order from here
    (1024, 1, 1, 16, lengths(7, 1024, 6, [(1023, 1100), (512, 700)])),      # the most that are cut
    (1025, 1, 1, 16, lengths(8, 1025, 6, [(1024, 700)])),                   # none is
    (1, 1, 1, 64, [5000]),                                                  # one sequence over all of the chip
    (2, 200, 200, 8, [400, 300]),                                           # more heads than half the workgroups
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_every_row_once(gpu_lib, i, dtype):
    B, H, kv, d, n = CASES[i]
    assert len(n) == B
    c = attention_case(200 + i, n, H, kv, d, d, dtype, spare=5, carry=i % 2 == 1)
    check_forward(gpu_lib, c)
    check_backward(gpu_lib, c)


def test_bad_offsets_of_cut_sequences_stay_inside(gpu_lib):
    """Sequences that overlap add up to more parts than there is room for: reported, and nothing outside out is written."""
    import torch

    c = attention_case(300, [2000, 0, 0, 0, 0], 2, 2, 32, 32, "bf16")
    for bad in ([0, 2000, 0, 2000, 0, 2000], [0, 2000, 2000, 0, 0, 2000], [2000, 0, 2000, 0, 2000, 2000],
                [0, -2 ** 62, 2 ** 62, 5, 2000, 2000]):
        fw = torch.zeros(1, dtype=torch.int32, device="cuda")
        room = torch.full((2000 + 64, 2, 32), -7.0, device="cuda", dtype=torch.bfloat16)
        off = torch.tensor(bad, dtype=torch.int64, device="cuda")
        gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], off, out=room[32:2032], fault=fw)
        assert int(fw) == gpu_lib.FAULT_SEQUENCES, bad
        assert bool((room[:32] == -7.0).all()) and bool((room[2032:] == -7.0).all())
        gpu_lib.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], off)
    torch.cuda.synchronize()


def test_the_same_bits_every_time(gpu_lib):
    """Gradients of shared heads and of cut sequences, twice."""
    import torch

    c = attention_case(301, lengths(9, 40, 200, [(7, 3000)]), 8, 2, 64, 64, "bf16", carry=True)
    runs = [gpu_lib.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"], initial_state=c["s0"],
                                              dfinal_state=c["df"], dinitial_state=True) for _ in range(2)]
    for a, b in zip(*runs):
        assert torch.equal(a, b)


def test_calls_on_a_given_stream(gpu_lib):
    """The stream argument: outputs and workspaces belong to it, and it may run beside the current one."""
    import torch

    c = attention_case(302, [900, 30], 4, 4, 64, 64, "bf16")
    x = torch.randn(c["rows"], 64, device="cuda").bfloat16()
    want = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"])[0]
    normed = gpu_lib.layer_norm(x, stats=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        got = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], stream=side)[0]
        again = gpu_lib.layer_norm(x, stats=True, stream=side)
        noise = torch.randn(1 << 22, device="cuda") * 2  # the current stream goes on
        side.synchronize()
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(again, normed))
    del noise


def test_head_major_rows(gpu_lib):
    """q, k, v and out as [heads][rows][dim], seen as rows of heads."""
    import torch

    c = attention_case(303, [700, 0, 65], 3, 3, 64, 40, "f16")
    want = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"])[0]
    q, k, v = (c[t].transpose(0, 1).contiguous().transpose(0, 1) for t in "qkv")
    out = torch.empty(3, c["rows"], 40, device="cuda", dtype=torch.float16).transpose(0, 1)
    gpu_lib.linear_attention(q, k, v, c["decay"], c["doff"], out=out)
    assert torch.equal(out, want)


def test_infinite_and_positive_decays(gpu_lib):
    """-inf forgets everything at once; more than 0 counts as 0."""
    import torch

    c = attention_case(304, [130], 2, 2, 32, 32, "f32")
    odd = torch.tensor([-float("inf"), 0.5], device="cuda")
    got, end = gpu_lib.linear_attention(c["q"], c["k"], c["v"], odd, c["doff"], final_state=True)
    c["decay"], c["decayr"] = torch.tensor([-1e4, 0.0], device="cuda"), np.array([-1e4, 0.0])
    check_forward(gpu_lib, c)
    want, last = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"], final_state=True)
    assert torch.equal(got, want) and torch.equal(end, last)
