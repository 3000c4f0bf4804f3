"""The binding of the sequence operators without a GPU: what it looks at before it hands addresses to the library.

Tensors here say that they are on GPU 0 and lie in host memory; the library is the real one for sizes, and a recorder for
calls, which run nothing."""
import pytest
import torch

from test_abi_host import mb  # noqa: F401  (the loaded library)


class OnGpu(torch.Tensor):
    where = 0

    def get_device(self):
        return self.where


class OnOtherGpu(OnGpu):
    where = 1


def gpu(t, where=OnGpu):
    return t.as_subclass(where)


class Recorder:
    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("workspace_bytes"):
            return getattr(self.real, name)
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def lib(mb, monkeypatch):
    rec = Recorder(mb.load())
    monkeypatch.setattr(mb, "_lib", rec)
    monkeypatch.setattr(mb, "load", lambda: rec)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    return rec


def attention_tensors(rows=6, heads=2, dim=4, sequences=2):
    q, k, v, g = (gpu(torch.zeros(rows, heads, dim)) for _ in range(4))
    decay = gpu(torch.zeros(heads))
    off = gpu(torch.tensor([0, 2, rows]))
    state = gpu(torch.zeros(sequences, heads, dim, dim))
    return q, k, v, g, decay, off, state


@pytest.mark.parametrize("wrong", [lambda t: t.as_subclass(torch.Tensor), lambda t: gpu(t, OnOtherGpu)], ids=["host", "other"])
def test_states_to_write_must_be_on_the_gpu(mb, lib, wrong):  # noqa: F811
    q, k, v, g, decay, off, state = attention_tensors()
    mb.linear_attention(q, k, v, decay, off, final_state=state)
    mb.linear_attention_backward(g, q, k, v, decay, off, initial_state=state, dinitial_state=gpu(torch.zeros_like(state)))
    assert [c[0] for c in lib.calls] == ["mmbev_linear_attention", "mmbev_linear_attention_backward"]
    lib.calls.clear()
    with pytest.raises(mb.MmbevError, match="one GPU"):
        mb.linear_attention(q, k, v, decay, off, final_state=wrong(state))
    with pytest.raises(mb.MmbevError, match="one GPU"):
        mb.linear_attention_backward(g, q, k, v, decay, off, initial_state=state, dinitial_state=wrong(state))
    assert not lib.calls


def test_a_first_call_with_its_own_workspace_loads_the_library(mb, lib, monkeypatch):  # noqa: F811
    q, k, v, g, decay, off, state = attention_tensors()
    room = gpu(torch.zeros(1 << 20, dtype=torch.uint8))
    monkeypatch.setattr(mb, "_lib", None)
    mb.linear_attention(q, k, v, decay, off, workspace=room)
    mb.linear_attention_backward(g, q, k, v, decay, off, workspace=room)
    assert len(lib.calls) == 2


def norm_tensors():
    x, y = (gpu(torch.zeros(5, 8)) for _ in range(2))
    w, mean, rstd = gpu(torch.ones(8)), gpu(torch.zeros(5)), gpu(torch.ones(5))
    return x, y, w, mean, rstd


def test_writes_raise_the_version_that_autograd_checks(mb, lib):  # noqa: F811
    x, y, w, mean, rstd = norm_tensors()
    q, k, v, g, decay, off, state = attention_tensors()
    pos, steps, axis = gpu(torch.zeros(6, dtype=torch.int32)), gpu(torch.zeros(2, dtype=torch.int64)), gpu(torch.zeros(2, dtype=torch.uint8))
    out, dq, dk, dv, end = (gpu(torch.zeros_like(t)) for t in (q, q, k, v, state))

    def check(call, written, read):
        before = [t._version for t in written + read]
        call()
        after = [t._version for t in written + read]
        assert [a > b for a, b in zip(after, before)] == [True] * len(written) + [False] * len(read)

    total, dw, db = gpu(torch.zeros(5, 8)), gpu(torch.zeros(8)), gpu(torch.zeros(8))
    check(lambda: mb.layer_norm(x, w, residual=y, out=x, out_sum=total), [x, total], [y, w])
    check(lambda: mb.layer_norm_backward(y, x, w, mean, rstd, dx=total, dweight=dw, dbias=db), [total, dw, db], [x, y, w, mean, rstd])
    check(lambda: mb.rotary(q, pos, steps, axis, out=q), [q], [pos, steps])
    check(lambda: mb.linear_attention(q, k, v, decay, off, initial_state=state, final_state=end, out=out), [end, out], [q, k, v, state])
    check(lambda: mb.linear_attention_backward(g, q, k, v, decay, off, initial_state=state, dinitial_state=end, dq=dq, dk=dk, dv=dv),
          [end, dq, dk, dv], [g, q, k, v, state])
    check(lambda: mb.linear_attention_step(q, k, v, decay, gpu(torch.zeros(6, 2, 4, 4)), out=out), [out], [q, k, v])
    held = gpu(torch.zeros(6, 2, 4, 4))
    check(lambda: mb.linear_attention_step(q, k, v, decay, held), [held], [q, k, v])
    with torch.inference_mode():
        held = gpu(torch.zeros(6, 2, 4, 4))
        mb.linear_attention_step(q, k, v, decay, held)
    mb.linear_attention_step(q, k, v, decay, held)  # a tensor without a version


@pytest.fixture
def anywhere(mb, lib, monkeypatch):
    """The binding without its look at where tensors are, for what autograd makes by itself."""
    mb._with_torch()
    monkeypatch.setattr(mb, "_issue_on", lambda *a: None)


@pytest.mark.parametrize("residual", [True, False])
@pytest.mark.parametrize("weight", [True, False])
@pytest.mark.parametrize("bias", [True, False])
def test_every_form_of_the_norm_has_a_gradient(mb, anywhere, residual, weight, bias):  # noqa: F811
    from paper_2608_15437_amd import encoder

    x, y, w, b = (torch.ones(*s, requires_grad=use) for s, use in (((5, 8), True), ((5, 8), residual), ((8,), weight), ((8,), bias)))
    out, total = encoder.norm(x, y if residual else None, w if weight else None, b if bias else None)
    (out.sum() + total.sum()).backward()
    assert all((t.grad is not None) == t.requires_grad for t in (x, y, w, b))


def test_second_derivatives_are_refused(mb, anywhere):  # noqa: F811
    from paper_2608_15437_amd import encoder

    rows = lambda *s: torch.ones(*s, requires_grad=True)  # noqa: E731
    x = rows(5, 8)
    q, k, v = (rows(6, 2, 4) for _ in range(3))
    pos, steps, axis = torch.zeros(6, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.uint8)
    for t, out in ((x, encoder.norm(x, None, None, None)[0]), (q, encoder.rotary(q, pos, steps, axis)),
                   (q, encoder.linear_attention(q, k, v, torch.zeros(2), torch.tensor([0, 6]))[0])):
        (d,) = torch.autograd.grad(out.square().sum(), t, create_graph=True)  # the gradient that comes in depends on t
        with pytest.raises(mb.MmbevError, match="second derivative"):
            (d * t).sum().backward()
    out, total = encoder.norm(x, None, None, None)  # what was saved does
    (d,) = torch.autograd.grad(out.sum(), x, create_graph=True)
    with pytest.raises(mb.MmbevError, match="second derivative"):
        (d * x).sum().backward()
    # a rotation's gradient does not depend on what was turned
    (d,) = torch.autograd.grad(encoder.rotary(q, pos, steps, axis).sum(), q, create_graph=True)
    assert not d.requires_grad


def test_a_decay_that_wants_a_gradient_is_refused(mb, anywhere):  # noqa: F811
    from paper_2608_15437_amd import encoder

    q, k, v = (torch.ones(6, 2, 4, requires_grad=True) for _ in range(3))
    decay, off = torch.zeros(2, requires_grad=True), torch.tensor([0, 6])
    with pytest.raises(mb.MmbevError, match="log_decay"):
        encoder.linear_attention(q, k, v, decay, off)
    with torch.no_grad():
        encoder.linear_attention(q, k, v, decay, off)
    encoder.linear_attention(q, k, v, decay.detach(), off)


def test_the_library_shares_torchs_hip_runtime(mb):  # noqa: F811
    """A host helper called before torch is imported must not bring a second HIP runtime: launches on torch's memory and
    streams then fail."""
    import os
    import subprocess
    import sys

    code = ("from paper_2608_15437_amd import mmbev; mmbev.make_rotary(16); import torch; "
            "print(len({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}))")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=110)
    assert r.returncode == 0 and r.stdout.split()[-1] == "1", r.stdout + r.stderr


def test_rows_are_zeroed_only_where_a_gradient_is_wanted(mb, anywhere, monkeypatch):  # noqa: F811
    """Inference with the module's parameters, over buffers whose rows the device counts, fills nothing."""
    from paper_2608_15437_amd import encoder

    zeroed = []
    for name in ("layer_norm", "rotary", "linear_attention"):
        real = getattr(mb, name)
        monkeypatch.setattr(mb, name, lambda *a, real=real, **kw: zeroed.append(kw.get("out") is not None) or real(*a, **kw))
    x, y, w, b = torch.ones(5, 8), torch.ones(5, 8), torch.ones(8, requires_grad=True), torch.zeros(8, requires_grad=True)
    q, k, v = (torch.ones(6, 2, 4, requires_grad=True) for _ in range(3))
    pos, steps, axis = torch.zeros(6, dtype=torch.int32), torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.uint8)
    count = torch.tensor([3])

    def run():
        zeroed.clear()
        encoder.norm(x, y, w, b, row_count=count)
        encoder.rotary(q, pos, steps, axis, row_count=count)
        encoder.linear_attention(q, k, v, torch.zeros(2), torch.tensor([0, 6]))
        return list(zeroed)

    assert run() == [True] * 3
    with torch.no_grad():
        assert run() == [False] * 3
