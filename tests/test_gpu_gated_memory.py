"""The gated operators at their largest: the last of 2^31 - 1 rows.  What small calls give for the same rows is compared bit
by bit (those are checked against the oracle elsewhere)."""
import pytest

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
