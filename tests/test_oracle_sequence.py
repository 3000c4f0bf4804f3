"""The oracle of the sequence operators: closed forms, a definition by all pairs of rows, and its gradients against
central differences of its forward passes.  CPU only."""
import math

import numpy as np
import pytest

from oracle import sequence as osq


def test_layer_norm_closed_form():
    out, mean, rstd = osq.layer_norm([[1.0, 3.0], [5.0, 5.0]], np.array([2.0, 2.0]), np.array([1.0, 0.0]), 0.0 + 1e-30)
    assert mean.tolist() == [2.0, 5.0]
    assert np.allclose(out[0], [-1.0, 2.0]) and rstd[0] == 1.0
    assert np.allclose(out[1], [1.0, 0.0])  # no variance: the bias alone


def differences(f, x, g, eps=1e-5):
    """Central differences of sum(f(x) * g) with respect to x."""
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += eps
        down[i] -= eps
        d[i] = ((f(up) - f(down)) * g).sum() / (2 * eps)
    return d


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(0)
    x, w, b, g, skip = (rng.standard_normal(s) for s in ((4, 7), 7, 7, (4, 7), (4, 7)))
    _, mean, rstd = osq.layer_norm(x, w, b, 1e-3)
    dx, dw, db = osq.layer_norm_backward(g, x, w, mean, rstd, skip)
    assert np.allclose(dx - skip, differences(lambda t: osq.layer_norm(t, w, b, 1e-3)[0], x, g), atol=1e-8)
    assert np.allclose(dw, differences(lambda t: osq.layer_norm(x, t, b, 1e-3)[0], w, g), atol=1e-8)
    assert np.allclose(db, differences(lambda t: osq.layer_norm(x, w, t, 1e-3)[0], b, g), atol=1e-8)


def test_rotary_turns_a_quarter_and_keeps_relative_angles():
    steps, axis = [1 << 62, 1 << 61], [0, 0]  # a quarter and an eighth of a turn a position
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    out = osq.rotary(x, [[1]], steps, axis, "half")
    r = math.sqrt(0.5)
    assert np.allclose(out[0, 0], [-3.0, 2 * r - 4 * r, 1.0, 2 * r + 4 * r, 9.0])
    out = osq.rotary(x, [[1]], steps, axis, "interleaved")
    assert np.allclose(out[0, 0], [-2.0, 1.0, 3 * r - 4 * r, 3 * r + 4 * r, 9.0])
    # 2^20 + 1 positions of a quarter turn are a quarter turn; the inverse takes it back
    far = osq.rotary(x, [[(1 << 20) + 1]], steps[:1], axis[:1], "half")
    assert np.allclose(far, osq.rotary(x, [[1]], steps[:1], axis[:1], "half"), atol=1e-15)
    assert np.allclose(osq.rotary(out, [[1]], steps, axis, "interleaved", inverse=True), x)


def test_rotary_ladders():
    plain, axis = osq.rotary_ladder(16, axes=3)
    assert axis.tolist() == [0, 0, 1, 1, 1, 2, 2, 2]
    assert np.allclose(plain[[0, 2, 5]], 1 / (2 * math.pi))
    slow = osq.rotary_ladder(16, scaling="base", factor=4.0)[0]
    ref = osq.rotary_ladder(16)[0]
    assert np.isclose(slow[0], ref[0]) and np.isclose(slow[-1], ref[-1] / 4)
    parts = osq.rotary_ladder(16, scaling="parts", factor=8.0, length=1000.0, slow=1.0, fast=20.0)[0]
    turns = ref * 1000.0
    assert np.allclose(parts[turns >= 20], ref[turns >= 20]) and np.allclose(parts[turns <= 1], ref[turns <= 1] / 8)


def attention_inputs(rng, rows=9, H=4, kv=2, kd=3, vd=5, B=3):
    q, k, v, g = (rng.standard_normal(s) for s in ((rows, H, kd), (rows, kv, kd), (rows, kv, vd), (rows, H, vd)))
    return q, k, v, g, -rng.uniform(0, 1, H), rng.standard_normal((B, H, kd, vd)), rng.standard_normal((B, H, kd, vd))


def test_attention_against_all_pairs():
    rng = np.random.default_rng(1)
    q, k, v, _, decay, s0, _ = attention_inputs(rng)
    offsets = [0, 4, 4, 9]
    out, final = osq.linear_attention(q, k, v, decay, offsets, 0.7, s0)
    for b in range(3):
        lo, hi = offsets[b], offsets[b + 1]
        for h in range(4):
            end = s0[b, h] * math.exp(decay[h] * (hi - lo))
            for i in range(lo, hi):
                ref = math.exp(decay[h] * (i - lo + 1)) * q[i, h] @ s0[b, h]
                for j in range(lo, i + 1):
                    ref = ref + math.exp(decay[h] * (i - j)) * (q[i, h] @ k[j, h // 2]) * v[j, h // 2]
                assert np.allclose(out[i, h], 0.7 * ref)
                end = end + math.exp(decay[h] * (hi - 1 - i)) * np.outer(k[i, h // 2], v[i, h // 2])
            assert np.allclose(final[b, h], end)


@pytest.mark.parametrize("carry", [False, True])
def test_attention_gradients_against_differences(carry):
    rng = np.random.default_rng(2)
    q, k, v, g, decay, s0, gf = attention_inputs(rng, rows=7)
    offsets = [0, 3, 3, 7]
    s0, gf = (s0, gf) if carry else (None, None)
    dq, dk, dv, ds = osq.linear_attention_backward(g, q, k, v, decay, offsets, 0.7, s0, gf)
    weight = np.concatenate([g.ravel(), (gf if carry else np.zeros((3, 4, 3, 5))).ravel()])

    def both(*a):
        return np.concatenate([t.ravel() for t in osq.linear_attention(*a)])

    assert np.allclose(dq, differences(lambda t: both(t, k, v, decay, offsets, 0.7, s0), q, weight), atol=1e-7)
    assert np.allclose(dk, differences(lambda t: both(q, t, v, decay, offsets, 0.7, s0), k, weight), atol=1e-7)
    assert np.allclose(dv, differences(lambda t: both(q, k, t, decay, offsets, 0.7, s0), v, weight), atol=1e-7)
    if carry:
        assert np.allclose(ds, differences(lambda t: both(q, k, v, decay, offsets, 0.7, t), s0, weight), atol=1e-7)


def test_attention_steps_are_the_sequence():
    rng = np.random.default_rng(3)
    q, k, v, _, decay, s0, _ = attention_inputs(rng, rows=6, B=1)
    out, final = osq.linear_attention(q, k, v, decay, [0, 6], 0.5, s0)
    state = s0.copy()
    for t in range(6):
        got, state = osq.linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], decay, state, [0], 0.5)
        assert np.allclose(got[0], out[t])
    assert np.allclose(state, final)
