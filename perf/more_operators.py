"""Cases of the voxel encoder's gated operators: norms of queries and keys with rotary positions, and the gated delta rule.

They stand where layer norm, rotary and linear attention do: over the rows that the voxelisation writes, one row per
voxel in key order, one range of rows per frame.  Row counts are those of the voxeliser's own workloads (one frame, a
keyframe at its cap, a robot frame, 8 crowded frames, 128 frames of a log); widths and heads are generic.
"""
import math
import types

import torch

own = False
DEV = "cuda"
_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_EPS = 1e-6
_CHUNK = 64  # rows of a chunk in the plain form

# ------------------------------------------------------------------ the cases

_QK = dict(kind="qk", rows=5442, heads=8, kv_heads=8, dim=64, rot=48, axes=3, dtype="bf16", layout="half", far=1440)
_DELTA = dict(kind="delta", frames=1, rows=5442, heads=8, kv_heads=8, key_dim=64, value_dim=64, dtype="bf16", carry=False)
_STEP = dict(kind="step", streams=64, heads=8, kv_heads=8, key_dim=64, value_dim=64, dtype="bf16")


def listed():
    return [
        # Queries and keys of one frame, normalised and turned by their voxel coordinates: a small call, latency counts.
        dict(_QK, name="qk_frame"),
        # The same over 128 frames of a log, keys of two query heads each, the whole head turned along the key order.
        dict(_QK, name="qk_batch", rows=921997, kv_heads=4, rot=64, axes=1, layout="interleaved", far=160000),
        # Its gradients on a robot frame in half precision: few wide heads of an odd width.
        dict(_QK, name="qk_grad_robot", kind="qk_grad", rows=18608, heads=4, kv_heads=4, dim=100, rot=66, dtype="f16", far=400),
        # Its gradients in a training step over 8 crowded frames, in full precision.
        dict(_QK, name="qk_grad_crowded", kind="qk_grad", rows=213879, dtype="f32"),
        # One new row for each of 64 streams: the recurrent form, states updated in place, the smallest call.
        dict(_STEP, name="delta_step"),
        # The same for 1,024 streams of wide heads, pairs of query heads sharing keys and values.
        dict(_STEP, name="delta_step_many", streams=1024, kv_heads=4, key_dim=128, value_dim=128, dtype="f16"),
        # One frame's voxels.
        dict(_DELTA, name="delta_frame"),
        # A keyframe at the voxel cap that continues from a state and leaves one: a single long sequence.
        dict(_DELTA, name="delta_keyframe", rows=120000, carry=True),
        # 128 frames of a log, ragged.
        dict(_DELTA, name="delta_batch", frames=128, rows=921997),
        # A robot frame in full precision, heads of unlike key and value widths.
        dict(_DELTA, name="delta_robot", rows=18608, heads=4, kv_heads=4, key_dim=96, value_dim=120, dtype="f32", carry=True),
        # The gradients for one robot frame: few wide heads in half precision.
        dict(_DELTA, name="delta_grad_robot", kind="delta_grad", rows=18608, heads=4, kv_heads=4, key_dim=128, value_dim=128,
             dtype="f16", carry=True),
        # The gradients over 8 crowded frames, pairs of query heads sharing keys and values.
        dict(_DELTA, name="delta_grad_crowded", kind="delta_grad", frames=8, rows=213879, kv_heads=4),
    ]


def draw(rng):
    """One more case of the same ranges: from a single row to 128 frames, odd sizes, every type and direction."""
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))

    kind = rng.choice(["qk", "qk_grad", "delta", "delta", "delta_grad", "delta_grad", "step"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    wide = 2 if dtype == "f32" else 1
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 1, 2, 4])
    if kind in ("qk", "qk_grad"):
        dim = rng.choice([32, 48, 64, 64, 96, 128, 128, rng.randint(6, 160)])
        rot = 2 * rng.randint(3, dim // 2)
        rows = spread(1, 921997 * 768 // ((heads + kv_heads) * dim) // wide // (2 if kind == "qk_grad" else 1))
        return dict(kind=kind, rows=min(rows, 921997), heads=heads, kv_heads=kv_heads, dim=dim, rot=rot, axes=rng.choice([1, 3]),
                    dtype=dtype, layout=rng.choice(["half", "interleaved"]), far=spread(16, 2000000))
    key_dim = rng.choice([32, 64, 64, 128, rng.randint(8, 128)])
    value_dim = key_dim if rng.random() < 0.6 else rng.choice([32, 64, 128, rng.randint(8, 128)])
    if kind == "step":
        return dict(kind=kind, streams=spread(1, 1024 * 8 // heads), heads=heads, kv_heads=kv_heads, key_dim=key_dim,
                    value_dim=value_dim, dtype=dtype)
    width = 32 if max(key_dim, value_dim) <= 32 else 64 if max(key_dim, value_dim) <= 64 else 128
    most = (921997 if kind == "delta" else 213879) * 512 // (heads * width) // (1 if width <= 64 else 2) // wide
    rows = min(spread(1, most), 921997)
    frames = min(spread(1, 128), rows)
    # few frames hold few rows: the longest sequence is a keyframe at its cap
    rows = min(rows, frames * 120000)
    return dict(kind=kind, frames=frames, rows=rows, heads=heads, kv_heads=kv_heads, key_dim=key_dim, value_dim=value_dim,
                dtype=dtype, carry=rng.random() < 0.5)


def work(case):
    c = types.SimpleNamespace(**case)
    size = 4 if c.dtype == "f32" else 2
    if c.kind in ("qk", "qk_grad"):
        n = c.rows * (c.heads + c.kv_heads) * c.dim
        more = 4 * c.rows * c.axes + 9 * c.rot // 2 + 8 * c.dim
        if c.kind == "qk":
            return {"bytes": 2 * n * size + more, "flops": 4 * n + n * 3 * c.rot // c.dim}
        return {"bytes": 3 * n * size + more + 8 * c.dim, "flops": 11 * n + n * 3 * c.rot // c.dim}
    state = c.heads * c.key_dim * c.value_dim
    token = (c.heads + c.kv_heads) * (c.key_dim + c.value_dim)
    if c.kind == "step":
        return {"bytes": c.streams * (8 * state + token * size + 8 * c.heads), "flops": c.streams * state * 7}
    carried = c.frames * state * 4 * 2 if c.carry else 0
    if c.kind == "delta":
        return {"bytes": c.rows * (token * size + 8 * c.heads) + carried, "flops": c.rows * state * 7}
    dout = c.heads * c.value_dim  # the gradients are those of q, k, v and the gates
    return {"bytes": c.rows * ((2 * token - dout) * size + 16 * c.heads) + 1.5 * carried, "flops": c.rows * state * 20}


# ------------------------------------------------------------------ inputs

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def rotary_ladder(rot, axes, base=10000.0):
    """Steps (fractions of a turn in 64 bits) and axis of each pair: the pairs shared out among the axes, each with a
    geometric ladder of its own."""
    pairs = rot // 2
    steps, axis = [], []
    for a in range(axes):
        n = pairs * (a + 1) // axes - pairs * a // axes
        for j in range(n):
            step = int(math.ldexp(base ** (-j / n) / (2.0 * math.pi), 64)) % (1 << 64)
            steps.append(step - (1 << 64) if step >> 63 else step)
            axis.append(a)
    return torch.tensor(steps, dtype=torch.int64), torch.tensor(axis, dtype=torch.uint8)


def _offsets(gen, frames, rows):
    """Ragged ranges of rows that add up to `rows`; with several frames one of them may be empty."""
    share = torch.rand(frames, generator=gen, dtype=torch.float64) + 0.25
    if frames > 2 and frames % 2 == 0:
        share[int(torch.randint(frames, (1,), generator=gen))] = 0.0
    ends = (share.cumsum(0) / share.sum() * rows).round().to(torch.int64)
    ends[-1] = rows
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends]).to(DEV)


def prepare(case, seed):
    s = types.SimpleNamespace(**case)
    gen = torch.Generator(device=DEV).manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    t = _TYPES[s.dtype]
    if s.kind in ("qk", "qk_grad"):
        # queries, keys and values side by side in a projection's rows
        widths = [s.heads * s.dim, s.kv_heads * s.dim, s.kv_heads * s.dim]
        x = _normal(gen, s.rows, sum(widths)) * (0.5 + torch.rand(s.rows, 1, generator=gen, device=DEV))
        q, k, _ = x.to(t).split(widths, dim=1)
        s.q, s.k = q.unflatten(1, (s.heads, s.dim)), k.unflatten(1, (s.kv_heads, s.dim))
        s.q_weight = 1.0 + 0.2 * _normal(gen, s.dim)
        s.k_weight = 1.0 + 0.2 * _normal(gen, s.dim)
        s.positions = torch.randint(0, s.far, (s.rows, s.axes), generator=gen, device=DEV, dtype=torch.int32)
        s.steps, s.axis = (v.to(DEV) for v in rotary_ladder(s.rot, s.axes))
        if s.kind == "qk_grad":
            s.dq = _normal(gen, s.rows, s.heads, s.dim).to(t)
            s.dk = _normal(gen, s.rows, s.kv_heads, s.dim).to(t)
        return s
    n = s.streams if s.kind == "step" else s.rows
    # queries and keys of length 1, as a norm for each head leaves them; values as they lie behind the keys' projection
    s.q = torch.nn.functional.normalize(_normal(gen, n, s.heads, s.key_dim), dim=-1).to(t)
    widths = [s.kv_heads * s.key_dim, s.kv_heads * s.value_dim]
    k = torch.nn.functional.normalize(_normal(gen, n, s.kv_heads, s.key_dim), dim=-1)
    kv = torch.cat([k.flatten(1), _normal(gen, n, widths[1])], dim=1).to(t)
    k, v = kv.split(widths, dim=1)
    s.k, s.v = k.unflatten(1, (s.kv_heads, -1)), v.unflatten(1, (s.kv_heads, -1))
    # the gates: heads that remember from a few rows to a few thousand, each row a little more or less; rates of writing
    # from next to none to a whole correction
    reach = 3.0 + 9.0 * torch.rand(s.heads, generator=gen, device=DEV)
    gate = torch.nn.functional.softplus(_normal(gen, n, s.heads)) / math.log(2.0)
    s.log_decay = -torch.exp2(-reach) * gate
    s.beta = torch.sigmoid(1.5 * _normal(gen, n, s.heads))
    s.scale = s.key_dim ** -0.5
    if s.kind == "step":
        s.state = 0.5 * _normal(gen, n, s.heads, s.key_dim, s.value_dim)
        return s
    s.offsets = _offsets(host, s.frames, s.rows)
    s.initial = s.dfinal = None
    if s.carry:
        s.initial = 0.5 * _normal(gen, s.frames, s.heads, s.key_dim, s.value_dim)
    if s.kind == "delta_grad":
        s.dout = _normal(gen, n, s.heads, s.value_dim).to(t)
        if s.carry:
            s.dfinal = _normal(gen, s.frames, s.heads, s.key_dim, s.value_dim)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2608_15437_amd import mmbev

    if s.kind == "qk":
        q, k = mmbev.head_norm_rotary(s.q, s.k, s.q_weight, s.k_weight, s.positions, s.steps, s.axis, eps=_EPS, layout=s.layout)
        return {"q": q, "k": k}
    if s.kind == "qk_grad":
        dq, dk, dqw, dkw = mmbev.head_norm_rotary_backward(s.dq, s.dk, s.q, s.k, s.q_weight, s.k_weight, s.positions, s.steps,
                                                           s.axis, eps=_EPS, layout=s.layout)
        return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
    if s.kind == "step":
        out = mmbev.gated_delta_step(s.q, s.k, s.v, s.log_decay, s.beta, s.state, scale=s.scale)
        return {"out": out, "state": s.state}
    if s.kind == "delta":
        out, final = mmbev.gated_delta(s.q, s.k, s.v, s.log_decay, s.beta, s.offsets, scale=s.scale, initial_state=s.initial,
                                       final_state=s.carry)
        return {"out": out, **({"final": final} if s.carry else {})}
    dq, dk, dv, dg, dbeta, dinitial = mmbev.gated_delta_backward(
        s.dout, s.q, s.k, s.v, s.log_decay, s.beta, s.offsets, scale=s.scale, initial_state=s.initial, dfinal_state=s.dfinal,
        dinitial_state=s.carry)
    return {"dq": dq, "dk": dk, "dv": dv, "dlog_decay": dg, "dbeta": dbeta, **({"dinitial": dinitial} if s.carry else {})}


def _turn(x, s, back):
    """The first `rot` elements of every head turned by the row's position, in 32 bits."""
    # a wrapping product of whole numbers: the phase is exact at any position
    phase = s.positions[:, s.axis.long()].long() * s.steps
    angle = (phase >> 40).float() * (2.0 * math.pi / (1 << 24))
    cos, sin = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    if back:
        sin = -sin
    turned, rest = x[..., :s.rot], x[..., s.rot:]
    if s.layout == "half":
        a, b = turned.chunk(2, dim=-1)
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    else:
        a, b = turned[..., 0::2], turned[..., 1::2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    return torch.cat([turned, rest], dim=-1)


def _plain(s):
    t = _TYPES[s.dtype]
    if s.kind in ("qk", "qk_grad"):
        out = {}
        for name in ("q", "k"):
            x, w = getattr(s, name).float(), getattr(s, name + "_weight")
            r = torch.rsqrt(x.square().mean(-1, keepdim=True) + _EPS)
            if s.kind == "qk":
                out[name] = _turn(x * r * w, s, False).to(t)
                continue
            h, dy = x * r, _turn(getattr(s, "d" + name).float(), s, True)
            a = dy * w
            out["d" + name] = (r * (a - h * (a * h).mean(-1, keepdim=True))).to(t)
            out["d" + name + "_weight"] = (dy * h).sum((0, 1))
        return out if s.kind == "qk" else {n: out[n] for n in ("dq", "dk", "dq_weight", "dk_weight")}
    group = s.heads // s.kv_heads
    if s.kind == "step":
        q, k, v = s.q.float(), s.k.float().repeat_interleave(group, 1), s.v.float().repeat_interleave(group, 1)
        state = s.state * torch.exp(s.log_decay)[..., None, None]
        u = s.beta[..., None] * (v - (k[..., None, :] @ state)[..., 0, :])
        s.state.copy_(state + k[..., :, None] * u[..., None, :])
        return {"out": ((q[..., None, :] @ s.state)[..., 0, :] * s.scale).to(t), "state": s.state}
    return _chunked(s, t, group)


def _chunked(s, t, group):
    """The gated delta rule in chunks of rows: what a chunk's rows do to each other solved at once, the states carried
    from chunk to chunk; its gradients in the same chunks, backwards."""
    C, frames, heads = _CHUNK, s.frames, s.heads
    length = s.offsets[1:] - s.offsets[:-1]
    count = -(-int(length.max()) // C)
    place = torch.arange(count * C, device=DEV)
    there = place < length[:, None]
    source = (s.offsets[:-1, None] + place).clamp(max=s.rows - 1)

    def cut(x):  # [frames][heads][chunks][C][...], zeros past a sequence's end
        x = torch.where(there.view(*there.shape, *[1] * (x.dim() - 1)), x[source].float(), 0.0)
        x = x.transpose(1, 2).unflatten(2, (count, C))
        return x if x.shape[1] == heads else x.repeat_interleave(group, 1)

    def join(x, like):  # back to rows, the heads that share an operand added up
        x = x.flatten(2, 3).transpose(1, 2)[there]
        if like.shape[1] != heads:
            x = x.unflatten(1, (like.shape[1], group)).sum(2)
        return x.to(like.dtype)

    q, k, v, beta = cut(s.q), cut(s.k), cut(s.v), cut(s.beta)[..., None]
    total = cut(s.log_decay).cumsum(-1)
    last = total[..., -1:, None]
    fade, left, whole = torch.exp(total)[..., None], torch.exp(last - total[..., None]), torch.exp(last)
    at = torch.arange(C, device=DEV)
    gap = total[..., :, None] - total[..., None, :]
    upto = torch.where(at[:, None] >= at, torch.exp(gap.clamp(max=0.0)), 0.0)
    del gap
    lower = (k @ k.transpose(-1, -2) * upto).tril(-1) * beta
    pairs = (q @ k.transpose(-1, -2)) * upto * s.scale
    # the inverse of 1 + lower, row by row
    solve = torch.eye(C, device=DEV).expand_as(lower).contiguous()
    for i in range(1, C):
        solve[..., i, :i] = -(lower[..., i:i + 1, :i] @ solve[..., :i, :i])[..., 0, :]
    u = solve @ (beta * v)
    into = solve @ (beta * fade * k)
    state = torch.zeros(frames, heads, s.key_dim, s.value_dim, device=DEV)
    if s.initial is not None:
        state = state + s.initial
    before = torch.empty(frames, heads, count, s.key_dim, s.value_dim, device=DEV)
    late = (k * left).transpose(-1, -2)
    for c in range(count):
        before[:, :, c] = state
        u[:, :, c] -= into[:, :, c] @ state
        state = whole[:, :, c] * state + late[:, :, c] @ u[:, :, c]
    if s.kind == "delta":
        out = join((q * fade * s.scale) @ before + pairs @ u, torch.empty(0, heads, dtype=t))
        return {"out": out, **({"final": state} if s.carry else {})}

    dout = cut(s.dout)
    du = pairs.transpose(-1, -2) @ dout
    dstate = torch.zeros_like(state) if s.dfinal is None else s.dfinal
    after = torch.empty_like(before)
    z = torch.empty_like(u)
    read_q, read_k, back = (q * fade * s.scale).transpose(-1, -2), (k * fade).transpose(-1, -2), solve.transpose(-1, -2)
    ends = torch.empty(frames, heads, count, device=DEV)
    for c in reversed(range(count)):
        after[:, :, c] = dstate
        ends[:, :, c] = (dstate * (before[:, :, c + 1] if c + 1 < count else state)).sum((-1, -2))
        z[:, :, c] = back[:, :, c] @ (du[:, :, c] + late[:, :, c].transpose(-1, -2) @ dstate)
        dstate = whole[:, :, c] * dstate + read_q[:, :, c] @ dout[:, :, c] - read_k[:, :, c] @ (beta[:, :, c] * z[:, :, c])
    y = beta * z
    dpairs = dout @ u.transpose(-1, -2) * upto * s.scale
    dlower = (y @ u.transpose(-1, -2) * upto).tril(-1)
    dq = fade * s.scale * (dout @ before.transpose(-1, -2)) + dpairs @ k
    dk_read = -fade * (y @ before.transpose(-1, -2)) - dlower @ k
    dk_write = left * (u @ after.transpose(-1, -2)) - dlower.transpose(-1, -2) @ k + dpairs.transpose(-1, -2) @ q
    # what a row's rule left over: its values less what the state and the rows before it hold for its key
    error = v - fade * (k @ before) - (k @ k.transpose(-1, -2) * upto).tril(-1) @ u
    dbeta = (z * error).sum(-1)
    dtotal = (q * dq).sum(-1) + (k * (dk_read - dk_write)).sum(-1)
    dgate = dtotal.flip(-1).cumsum(-1).flip(-1) + ends[..., None]
    return {"dq": join(dq, s.q), "dk": join(dk_read + dk_write, s.k), "dv": join(y, s.v), "dlog_decay": join(dgate, s.log_decay),
            "dbeta": join(dbeta, s.beta), **({"dinitial": dstate} if s.carry else {})}


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if s.kind in ("qk", "qk_grad"):
        # unit complex numbers from the phase's two halves of 32 bits
        phase = s.positions.long()[:, s.axis.long()] * s.steps
        turns = (phase >> 32).double() / 2.0 ** 32 + (phase & 0xFFFFFFFF).double() / 2.0 ** 64
        unit = torch.polar(torch.ones_like(turns), turns * 2.0 * math.pi)[:, None]
        half = s.rot // 2
        one = slice(0, half) if s.layout == "half" else slice(0, s.rot, 2)
        two = slice(half, s.rot) if s.layout == "half" else slice(1, s.rot, 2)
        out = {}
        for name in ("q", "k"):
            x, w = getattr(s, name).double(), getattr(s, name + "_weight").double()
            norm = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / s.dim + _EPS)
            y = x / norm * w if s.kind == "qk" else getattr(s, "d" + name).double()
            z = torch.complex(y[..., one], y[..., two]) * (unit if s.kind == "qk" else unit.conj())
            y = y.clone()
            y[..., one], y[..., two] = z.real, z.imag
            if s.kind == "qk":
                out[name] = y
                continue
            out["d" + name + "_weight"] = torch.einsum("rhd,rhd,rhu->d", y, x, 1.0 / norm)
            dot = torch.einsum("rhd,rhd,d->rh", y, x, w)[..., None]
            out["d" + name] = y * w / norm - x * dot / (s.dim * norm ** 3)
        return out if s.kind == "qk" else {n: out[n] for n in ("dq", "dk", "dq_weight", "dk_weight")}
    return _recurrent(s)


def _recurrent(s):
    """Row after row, all sequences and heads at once."""
    if s.kind == "step":
        s.rows, s.frames, s.carry, s.initial = s.streams, s.streams, True, s.state
        s.offsets = torch.arange(s.streams + 1, device=DEV)
    back = s.kind == "delta_grad"
    bounds = s.offsets.tolist()
    most = max(y - x for x, y in zip(bounds, bounds[1:]))
    n = s.frames * s.heads
    size = 8 * n * s.key_dim * s.value_dim
    if most * (2 if back else 1) * (5e-5 + size * 1e-11) > 12.0 or size * most / (s.key_dim if s.key_dim < s.value_dim else s.value_dim) > 2e10:
        return None  # too many rows one after the other
    which = torch.zeros(most, s.frames, dtype=torch.long)
    inside = torch.zeros(most, s.frames, dtype=torch.bool)
    for f, (x, y) in enumerate(zip(bounds, bounds[1:])):
        which[:y - x, f] = torch.arange(x, y)
        inside[:y - x, f] = True
    which, inside = which.to(DEV), inside.to(DEV)

    def rows(x):  # [row of its sequence][sequence and head][...]
        x = x.double().repeat_interleave(s.heads // x.shape[1], 1)[which]
        return (x * inside.view(most, s.frames, *[1] * (x.dim() - 2))).flatten(1, 2)

    def spread(x, like):
        x = x.unflatten(1, (s.frames, s.heads))
        y = torch.zeros(s.rows, *x.shape[2:], dtype=x.dtype, device=DEV)
        y[which[inside]] = x[inside]
        return y if like.shape[1] == s.heads else y.unflatten(1, (like.shape[1], -1)).sum(2)

    q, k, v = rows(s.q), rows(s.k), rows(s.v)
    a, beta = torch.exp(rows(s.log_decay))[..., None, None], rows(s.beta)[..., None, None]
    state = torch.zeros(n, s.key_dim, s.value_dim, dtype=torch.float64, device=DEV)
    if s.initial is not None:
        state += s.initial.double().flatten(0, 1)
    kc, kr, vr = k[..., None], k[..., None, :], v[..., None, :]

    def step(x, i, u_out):
        """The state after row i from the one before it, and what the row adds along its key."""
        x = x * a[i]
        torch.mul(torch.baddbmm(vr[i], kr[i], x, alpha=-1.0), beta[i], out=u_out)
        return x.baddbmm_(kc[i], u_out)

    u = torch.zeros(most, n, 1, s.value_dim, dtype=torch.float64, device=DEV)
    if not back:
        out = torch.zeros_like(u)
        for i in range(most):
            state = step(state, i, u[i])
            torch.bmm(q[i][:, None], state, out=out[i])
        out = spread(out[:, :, 0] * s.scale, s.q)
        state = state.unflatten(0, (s.frames, s.heads))
        return {"out": out, "state": state} if s.kind == "step" else {"out": out, **({"final": state} if s.carry else {})}

    block = max(1, min(256, int(2e9 // size)))
    marks = []
    for i in range(most):
        if i % block == 0:
            marks.append(state)
        state = step(state, i, u[i])
    dout = rows(s.dout) * s.scale
    dstate = torch.zeros_like(state) if s.dfinal is None else s.dfinal.double().flatten(0, 1)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    dg, dbeta = torch.zeros_like(q[..., 0]), torch.zeros_like(q[..., 0])
    for first in reversed(range(0, most, block)):
        m = min(block, most - first)
        at = slice(first, first + m)
        kept = torch.empty(m + 1, *state.shape, dtype=torch.float64, device=DEV)
        kept[0] = marks[first // block]
        for i in range(m):
            kept[i + 1] = step(kept[i], first + i, u[first + i])
        grads = torch.empty(m, *state.shape, dtype=torch.float64, device=DEV)
        for i in reversed(range(m)):
            torch.baddbmm(dstate, q[first + i][..., None], dout[first + i][:, None], out=grads[i])
            rate = torch.bmm(kr[first + i], grads[i]) * beta[first + i]
            dv[first + i] = rate[:, 0]
            dstate = torch.baddbmm(grads[i], kc[first + i], rate, alpha=-1.0) * a[first + i]
        dq[at] = (kept[1:] @ dout[at][..., None])[..., 0]
        faded = kept[:-1] * a[at]
        due = kr[at] @ grads
        dk[at] = (grads @ u[at].transpose(-1, -2) - faded @ dv[at][..., None])[..., 0]
        dbeta[at] = (due * (vr[at] - kr[at] @ faded)).sum((-1, -2))
        dg[at] = ((grads - kc[at] * dv[at][..., None, :]) * faded).sum((-1, -2))
    dinitial = dstate.unflatten(0, (s.frames, s.heads))
    return {"dq": spread(dq, s.q), "dk": spread(dk, s.k), "dv": spread(dv, s.v), "dlog_decay": spread(dg, s.log_decay),
            "dbeta": spread(dbeta, s.beta), **({"dinitial": dinitial} if s.carry else {})}
