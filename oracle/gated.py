"""Oracle of the gated operators (norms of queries and keys with rotary positions, the gated delta rule): their
definitions in include/mmbev.h, row by row in float64 numpy.  Shares no code with the library; test infrastructure only."""
import numpy as np

from . import sequence as osq


def head_norm_rotary(x, weight, positions, steps, axis, eps, layout):
    """One array of rows of heads [rows][heads][dim]; steps: Python integers below 2^64."""
    x = np.asarray(x, np.float64)
    y = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    return osq.rotary(y * (1.0 if weight is None else weight), positions, steps, axis, layout)


def head_norm_rotary_backward(dy, x, weight, positions, steps, axis, eps, layout):
    """(dx, dweight)."""
    x = np.asarray(x, np.float64)
    d = osq.rotary(dy, positions, steps, axis, layout, inverse=True)
    r = 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    a = d * (1.0 if weight is None else weight)
    dx = r * a - r ** 3 * x * (a * x).mean(-1, keepdims=True)
    return dx, (d * x * r).sum((0, 1))


def _heads(q, k, v):
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    group = q.shape[1] // k.shape[1]
    return q, k.repeat(group, 1), v.repeat(group, 1), group


def _row(S, k, v, a, beta):
    """One row of every head: the decayed state, what the row's rule left over, the state after it."""
    faded = a[:, None, None] * S
    error = v - np.einsum("hk,hkv->hv", k, faded)
    return faded, error, faded + k[:, :, None] * (beta[:, None] * error)[:, None, :]


def gated_delta(q, k, v, log_decay, beta, offsets, scale, initial=None):
    """(out [rows][heads][value_dim], final [B][heads][key_dim][value_dim]); rows of no sequence are zero."""
    q, k, v, _ = _heads(q, k, v)
    a, beta = np.exp(np.minimum(np.asarray(log_decay, np.float64), 0.0)), np.asarray(beta, np.float64)
    rows, H, kd = q.shape
    vd, B = v.shape[2], len(offsets) - 1
    out, final = np.zeros((rows, H, vd)), np.zeros((B, H, kd, vd))
    for b in range(B):
        S = np.zeros((H, kd, vd)) if initial is None else np.array(initial[b], np.float64)
        for t in range(offsets[b], offsets[b + 1]):
            S = _row(S, k[t], v[t], a[t], beta[t])[2]
            out[t] = scale * np.einsum("hk,hkv->hv", q[t], S)
        final[b] = S
    return out, final


def gated_delta_backward(dout, q, k, v, log_decay, beta, offsets, scale, initial=None, dfinal=None):
    """(dq, dk, dv, dlog_decay, dbeta, dinitial): the rows' recurrence differentiated by hand, backwards."""
    kv = np.asarray(k).shape[1]
    q, k, v, group = _heads(q, k, v)
    dout = np.asarray(dout, np.float64)
    g = np.asarray(log_decay, np.float64)
    a, beta = np.exp(np.minimum(g, 0.0)), np.asarray(beta, np.float64)
    rows, H, kd = q.shape
    vd, B = v.shape[2], len(offsets) - 1
    dq, dk, dv = np.zeros((rows, H, kd)), np.zeros((rows, H, kd)), np.zeros((rows, H, vd))
    dg, dbeta, dinitial = np.zeros((rows, H)), np.zeros((rows, H)), np.zeros((B, H, kd, vd))
    for b in range(B):
        S = np.zeros((H, kd, vd)) if initial is None else np.array(initial[b], np.float64)
        before = []
        for t in range(offsets[b], offsets[b + 1]):
            before.append(S)
            S = _row(S, k[t], v[t], a[t], beta[t])[2]
        D = np.zeros((H, kd, vd)) if dfinal is None else np.array(dfinal[b], np.float64)
        for t in reversed(range(offsets[b], offsets[b + 1])):
            faded, error, after = _row(before[t - offsets[b]], k[t], v[t], a[t], beta[t])
            dq[t] = scale * np.einsum("hv,hkv->hk", dout[t], after)
            D = D + scale * q[t][:, :, None] * dout[t][:, None, :]
            du = np.einsum("hk,hkv->hv", k[t], D)
            dbeta[t] = (du * error).sum(-1)
            dv[t] = beta[t][:, None] * du
            dk[t] = np.einsum("hkv,hv->hk", D, beta[t][:, None] * error) - np.einsum("hkv,hv->hk", faded, dv[t])
            dfaded = D - k[t][:, :, None] * dv[t][:, None, :]
            dg[t] = np.where(g[t] > 0, 0.0, (dfaded * faded).sum((-1, -2)))
            D = a[t][:, None, None] * dfaded
        dinitial[b] = D
    return (dq, dk.reshape(rows, kv, group, kd).sum(2), dv.reshape(rows, kv, group, vd).sum(2), dg, dbeta, dinitial)


def gated_delta_step(q, k, v, log_decay, beta, state, slots, scale):
    """(out, state): skipped rows' outputs are NaN."""
    q, k, v, _ = _heads(q, k, v)
    a, beta, state = np.exp(np.asarray(log_decay, np.float64)), np.asarray(beta, np.float64), np.array(state, np.float64)
    out = np.full((q.shape[0], q.shape[1], v.shape[2]), np.nan)
    for r, s in enumerate(slots):
        if 0 <= s < len(state):
            state[s] = _row(state[s], k[r], v[r], a[r], beta[r])[2]
            out[r] = scale * np.einsum("hk,hkv->hv", q[r], state[s])
    return out, state
