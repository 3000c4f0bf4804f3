"""Where the sequence operators' arrays lie: outputs over inputs where that is allowed, and arrays interleaved in one buffer."""
import pytest

from test_gpu_sequence import attention_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_step_in_place(gpu_lib, dtype):
    """out over q (shared heads), and over v where no heads share it."""
    import torch

    for kv, over in ((2, "q"), (4, "q"), (4, "k"), (4, "v")):
        c = attention_case(40, [37], 4, kv, 64, 64, dtype)
        state = torch.randn(37, 4, 64, 64, device="cuda")
        again = state.clone()
        want = gpu_lib.linear_attention_step(c["q"], c["k"], c["v"], c["decay"], state)
        got = gpu_lib.linear_attention_step(c["q"], c["k"], c["v"], c["decay"], again, out=c[over])
        assert torch.equal(got, want) and torch.equal(again, state)


def test_arrays_interleaved_in_rows_of_one_buffer(gpu_lib):
    """q, k, v and out, and then the gradients, side by side in rows and head by head."""
    import torch

    c = attention_case(41, [700, 0, 65], 3, 3, 64, 64, "bf16")
    want = gpu_lib.linear_attention(c["q"], c["k"], c["v"], c["decay"], c["doff"])[0]
    grads = gpu_lib.linear_attention_backward(c["g"], c["q"], c["k"], c["v"], c["decay"], c["doff"])
    R = c["rows"]
    for shape, pick in (((R, 4, 3, 64), lambda t, i: t[:, i]), ((R, 3, 4, 64), lambda t, i: t[:, :, i])):
        room = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
        for i, t in enumerate("qkv"):
            pick(room, i).copy_(c[t])
        q, k, v, out = (pick(room, i) for i in range(4))
        gpu_lib.linear_attention(q, k, v, c["decay"], c["doff"], out=out)
        assert torch.equal(out, want) and torch.equal(q, c["q"]) and torch.equal(k, c["k"]) and torch.equal(v, c["v"])
        back = torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda")
        dq, dk, dv, rest = (pick(back, i) for i in range(4))
        gpu_lib.linear_attention_backward(c["g"], q, k, v, c["decay"], c["doff"], dq=dq, dk=dk, dv=dv)
        assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), grads)) and bool((rest == 7.0).all())
