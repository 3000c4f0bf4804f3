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


def test_rows_more_than_31_bits_apart(gpu_lib):
    """Two rows 2^31 + 64 elements apart: norm, rotary and the step take them; attention says that it does not."""
    import torch

    wide = (1 << 31) + 64
    room = torch.zeros(wide + 64, dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((2, 64), (wide, 1))
    t = torch.randn(2, 64, device="cuda").bfloat16()
    x.copy_(t)
    assert torch.equal(gpu_lib.layer_norm(x)[0], gpu_lib.layer_norm(t)[0])
    steps, axis = (torch.from_numpy(a).cuda() for a in gpu_lib.make_rotary(32))
    pos = torch.tensor([7, 9], dtype=torch.int32, device="cuda")
    h, ht = x.unflatten(1, (2, 32)), t.unflatten(1, (2, 32))
    assert torch.equal(gpu_lib.rotary(h, pos, steps, axis), gpu_lib.rotary(ht, pos, steps, axis))
    g = torch.full((2,), -0.1, device="cuda")
    a, b = torch.zeros(2, 2, 2, 32, 32, device="cuda").unbind(0)
    assert torch.equal(gpu_lib.linear_attention_step(h, h, h, g, a), gpu_lib.linear_attention_step(ht, ht, ht, g, b))
    assert torch.equal(a, b)
    with pytest.raises(gpu_lib.MmbevError, match="-3"):
        gpu_lib.linear_attention(h, h, h, g, torch.tensor([0, 2], device="cuda"))


MOST = 1 << 23  # workgroups of a launch: more rows take more launches


def whole_of(view, tile, rows):
    """Every row of a large tensor against a tile that repeats, some of it at a time."""
    import torch

    n = tile.shape[0]
    return all(torch.equal(view[a:min(a + n, rows)], tile[:min(n, rows - a)]) for a in range(0, rows, n))


@pytest.mark.parametrize("operator", ["layer_norm", "rotary"])
def test_rows_past_one_launch(gpu_lib, operator):
    """A row a workgroup, 2^23 + 5 of them with 2^23 + 2 in use, in place: every row is right and those past the count are as
    they were."""
    import torch

    rows, used, n = MOST + 5, MOST + 2, 1 << 17
    if torch.cuda.mem_get_info()[0] < 45e9:
        pytest.skip("needs 45 GB of memory")
    count = torch.tensor([used], dtype=torch.int64, device="cuda")
    if operator == "layer_norm":
        tile = torch.randn(n, 2050, device="cuda").bfloat16()  # past 2,048 a row takes a whole workgroup
        run = lambda x, **kw: gpu_lib.layer_norm(x, **kw)[0]  # noqa: E731
    else:
        tile = torch.randn(n, 1024, device="cuda")  # 256 packs of two pairs
        steps, axis = (torch.from_numpy(a).cuda() for a in gpu_lib.make_rotary(1024))
        pos = (torch.arange(rows, dtype=torch.int32, device="cuda") % n).contiguous()
        run = lambda x, **kw: gpu_lib.rotary(x[:, None], pos[:x.shape[0]], steps, axis, "interleaved",  # noqa: E731
                                             **{k: v[:, None] if k == "out" else v for k, v in kw.items()})[:, 0]
    want = run(tile)
    x = torch.empty(rows, tile.shape[1], dtype=tile.dtype, device="cuda")
    for a in range(0, rows, n):
        x[a:a + n] = tile[:min(n, rows - a)]
    fault = torch.zeros(1, dtype=torch.int32, device="cuda")
    run(x, out=x, row_count=count, fault=fault)
    assert whole_of(x, want, used) and torch.equal(x[used:], tile[used - MOST:rows - MOST]) and int(fault) == 0
    del x
    torch.cuda.empty_cache()
