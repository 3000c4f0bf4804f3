"""Oracle of the sequence operators (layer norm, rotary positions, linear attention with decay): their definitions in
include/mmbev.h, row by row in float64 numpy.  Shares no code with the library; test infrastructure only."""
import math

import numpy as np


def layer_norm(s, weight, bias, eps):
    """(out, mean, rstd) of rows s [rows][width]."""
    s = np.asarray(s, np.float64)
    mean = np.array([math.fsum(r) / len(r) for r in s])
    var = np.array([math.fsum((r - m) ** 2) / len(r) for r, m in zip(s, mean)])
    rstd = 1.0 / np.sqrt(var + eps)
    h = (s - mean[:, None]) * rstd[:, None]
    out = h * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    return out, mean, rstd


def layer_norm_backward(dy, s, weight, mean, rstd, dskip=None):
    """(dx, dweight, dbias)."""
    dy, s = np.asarray(dy, np.float64), np.asarray(s, np.float64)
    h = (s - np.asarray(mean, np.float64)[:, None]) * np.asarray(rstd, np.float64)[:, None]
    a = dy * (1.0 if weight is None else weight)
    dx = (a - a.mean(1, keepdims=True) - h * (a * h).mean(1, keepdims=True)) * np.asarray(rstd, np.float64)[:, None]
    return dx + (0.0 if dskip is None else dskip), (dy * h).sum(0), dy.sum(0)


def rotary_ladder(rotary_dim, axes=1, base=10000.0, scaling="plain", factor=1.0, length=0.0, slow=1.0, fast=32.0):
    """Turns per position (float64) and axis of each pair."""
    pairs = rotary_dim // 2
    turns, axis = [], []
    for a in range(axes):
        n = pairs * (a + 1) // axes - pairs * a // axes
        for j in range(n):
            b = base * factor ** (n / (n - 1)) if scaling == "base" and n > 1 else base
            t = b ** (-j / n) / (2 * math.pi)
            if scaling == "linear":
                t /= factor
            if scaling == "parts":
                keep = min(1.0, max(0.0, (t * length - slow) / (fast - slow)))
                t = keep * t + (1 - keep) * t / factor
            turns.append(t)
            axis.append(a)
    return np.array(turns), np.array(axis)


def rotary(x, positions, steps, axis, layout, inverse=False):
    """x [rows][heads][dim]; steps: Python integers below 2^64 (turns per position in 2^-64)."""
    x = np.array(x, np.float64)
    half = len(steps)
    for r in range(x.shape[0]):
        for j in range(half):
            phase = (int(positions[r][axis[j]]) * int(steps[j])) % (1 << 64)
            t = 2 * math.pi * (phase / 2.0 ** 64)
            c, s = math.cos(t), math.sin(t) * (-1 if inverse else 1)
            i, k = (j, j + half) if layout == "half" else (2 * j, 2 * j + 1)
            a, b = x[r, :, i].copy(), x[r, :, k].copy()
            x[r, :, i], x[r, :, k] = a * c - b * s, a * s + b * c
    return x


def linear_attention(q, k, v, log_decay, offsets, scale, initial=None):
    """(out [rows][heads][value_dim], final [B][heads][key_dim][value_dim]); rows of no sequence are zero."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    rows, H, kd = q.shape
    group, vd, B = H // k.shape[1], v.shape[2], len(offsets) - 1
    k, v = k.repeat(group, 1), v.repeat(group, 1)
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    out = np.zeros((rows, H, vd))
    final = np.zeros((B, H, kd, vd))
    for b in range(B):
        S = np.zeros((H, kd, vd)) if initial is None else np.array(initial[b], np.float64)
        for t in range(offsets[b], offsets[b + 1]):
            S = lam * S + k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * np.einsum("hk,hkv->hv", q[t], S)
        final[b] = S
    return out, final


def linear_attention_backward(dout, q, k, v, log_decay, offsets, scale, initial=None, dfinal=None):
    """(dq, dk, dv, dinitial), the rows' recurrence differentiated by hand: forwards for dq, backwards for the rest."""
    dout, q, k, v = (np.asarray(t, np.float64) for t in (dout, q, k, v))
    rows, H, kd = q.shape
    kv, vd, B = k.shape[1], v.shape[2], len(offsets) - 1
    group = H // kv
    kr, vr = k.repeat(group, 1), v.repeat(group, 1)
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    dq, dk, dv = np.zeros((rows, H, kd)), np.zeros((rows, H, kd)), np.zeros((rows, H, vd))
    dinitial = np.zeros((B, H, kd, vd))
    for b in range(B):
        S = np.zeros((H, kd, vd)) if initial is None else np.array(initial[b], np.float64)
        for t in range(offsets[b], offsets[b + 1]):
            S = lam * S + kr[t][:, :, None] * vr[t][:, None, :]
            dq[t] = scale * np.einsum("hv,hkv->hk", dout[t], S)
        D = np.zeros((H, kd, vd)) if dfinal is None else np.array(dfinal[b], np.float64)
        for t in reversed(range(offsets[b], offsets[b + 1])):
            D = D + scale * q[t][:, :, None] * dout[t][:, None, :]  # the gradient of S_t
            dk[t] = np.einsum("hkv,hv->hk", D, vr[t])
            dv[t] = np.einsum("hkv,hk->hv", D, kr[t])
            D = lam * D
        dinitial[b] = D
    return dq, dk.reshape(rows, kv, group, kd).sum(2), dv.reshape(rows, kv, group, vd).sum(2), dinitial


def linear_attention_step(q, k, v, log_decay, state, slots, scale):
    """(out, state): skipped rows' outputs are NaN."""
    q, k, v, state = (np.array(t, np.float64) for t in (q, k, v, state))
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat(group, 1), v.repeat(group, 1)
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    out = np.full((q.shape[0], q.shape[1], v.shape[2]), np.nan)
    for r, s in enumerate(slots):
        if s < 0 or s >= len(state):
            continue
        state[s] = lam * state[s] + k[r][:, :, None] * v[r][:, None, :]
        out[r] = scale * np.einsum("hk,hkv->hv", q[r], state[s])
    return out, state
