"""The oracle of the gated operators: closed forms, its other definitions, and its gradients against central differences
of its forward passes.  CPU only."""
import numpy as np
import pytest

from oracle import gated as og
from oracle import sequence as osq


def differences(f, x, g, eps=1e-5):
    """Central differences of sum(f(x) * g) with respect to x."""
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += eps
        down[i] -= eps
        d[i] = ((f(up) - f(down)) * g).sum() / (2 * eps)
    return d


def test_head_norm_closed_form():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    steps, axis = [1 << 62], [0]  # a quarter of a turn a position
    out = og.head_norm_rotary(x, np.array([1.0, 2.0, 1.0, 1.0]), [[1]], steps, axis, 0.0, "interleaved")
    assert np.allclose(out[0, 0], [-3.2, 1.2, 0.0, 0.0])  # root of the mean square 2.5


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_head_norm_gradients_against_differences(layout):
    rng = np.random.default_rng(1)
    x, g, w = rng.standard_normal((3, 2, 9)), rng.standard_normal((3, 2, 9)), rng.uniform(0.5, 1.5, 9)
    steps, axis = [1 << 60, 3 << 57, 1 << 55], [0, 1, 1]
    pos = rng.integers(-50, 50, (3, 2))
    f = lambda x, w: og.head_norm_rotary(x, w, pos, steps, axis, 1e-2, layout)  # noqa: E731
    dx, dw = og.head_norm_rotary_backward(g, x, w, pos, steps, axis, 1e-2, layout)
    assert np.allclose(dx, differences(lambda t: f(t, w), x, g), atol=1e-8)
    assert np.allclose(dw, differences(lambda t: f(x, t), w, g), atol=1e-8)


def case(seed, rows=7, H=2, kv=1, kd=4, vd=3, B=2):
    rng = np.random.default_rng(seed)
    k = rng.standard_normal((rows, kv, kd))
    return dict(q=rng.standard_normal((rows, H, kd)), k=k / np.linalg.norm(k, axis=-1, keepdims=True), v=rng.standard_normal((rows, kv, vd)),
                log_decay=-rng.uniform(0.05, 1.0, (rows, H)), beta=rng.uniform(0.1, 1.5, (rows, H)), offsets=[0, 3, rows], scale=0.5,
                initial=rng.standard_normal((B, H, kd, vd)))


def test_no_keys_in_common_is_linear_attention():
    # keys along different axes never correct each other: with beta 1 the rule adds k v like linear attention
    rng = np.random.default_rng(2)
    q, v = rng.standard_normal((4, 1, 4)), rng.standard_normal((4, 1, 3))
    k = np.eye(4)[:, None, :]
    g = np.full((4, 1), -0.3)
    out, final = og.gated_delta(q, k, v, g, np.ones((4, 1)), [0, 4], 0.7)
    ref, last = osq.linear_attention(q, k, v, g[0], [0, 4], 0.7)
    assert np.allclose(out, ref) and np.allclose(final, last)


def test_a_whole_correction_holds_the_last_value():
    c = case(3)
    c["beta"][:] = 1.0
    _, final = og.gated_delta(**c)
    got = np.einsum("k,hkv->hv", c["k"][-1, 0], final[1])
    assert np.allclose(got, c["v"][-1].repeat(2, 0))


def test_delta_gradients_against_differences():
    c = case(4)
    rng = np.random.default_rng(5)
    dout, dfinal = rng.standard_normal((7, 2, 3)), rng.standard_normal((2, 2, 4, 3))

    def loss(name):
        def f(x):
            out, final = og.gated_delta(**{**c, name: x})
            return np.concatenate([(out * dout).ravel(), (final * dfinal).ravel()])

        return differences(f, c[name], 1.0)

    got = og.gated_delta_backward(dout, dfinal=dfinal, **c)
    for name, d in zip(("q", "k", "v", "log_decay", "beta", "initial"), got):
        assert np.allclose(d, loss(name), atol=1e-8), name


def test_steps_follow_a_sequence():
    c = case(6)
    out, final = og.gated_delta(**c)
    state = c["initial"].copy()
    for t in range(7):
        b = 0 if t < 3 else 1
        one = {n: c[n][t:t + 1] for n in ("q", "k", "v", "log_decay", "beta")}
        o, state = og.gated_delta_step(**one, state=state, slots=[b], scale=0.5)
        assert np.allclose(o[0], out[t])
    assert np.allclose(state, final)
