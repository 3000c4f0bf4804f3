"""A learned VoxelFeatureEncoder (Alg. 1) over the voxeliser's rows: the sequence operators as torch modules.

The voxeliser writes one row per voxel in key order, one range of rows per frame.  A block of the encoder norms the
rows, turns queries and keys by their voxel coordinates, mixes each frame's rows by linear attention with a decay per
head and adds the result to the rows; the projections between are plain matrix products of torch.  A gated block
takes the gated delta rule instead, over queries and keys that are normed for each head as they are turned.  Gradients
come from the library's backward calls, which have none themselves: a second derivative is refused.  A trained block can
also go on row by row (`step`), its state kept between rows.

The rows' number and ranges stay on the device: pass `row_count` (voxel_offsets[-1:]) to encode the voxeliser's full
buffers without waiting for the count.  Results past it hold nothing of meaning; where gradients are wanted they are
zeros, and so are the gradients of those rows.

The operators and the gradients that they sum themselves (of rows, norms' weights and biases) may be captured into a graph.
As with all torch modules, no eager autograd graph of the same parameters may be alive meanwhile: drop the results of
earlier passes first.  The other parameters' gradients are torch's own products and sums over rows (a gated block's
`rate` is one), which may clear scratch memory by nodes of the graph: compare replays of such a step with eager ones.
"""
from __future__ import annotations

import functools
import math

import torch
from torch import nn

from . import mmbev


class _Refusal(torch.autograd.Function):
    """A gradient that depends on `sources` in ways that autograd does not know of."""

    @staticmethod
    def forward(ctx, grad, *sources):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *grads):
        raise mmbev.MmbevError("the sequence operators have no second derivatives")


def _once(backward):
    """A backward pass whose results cannot be differentiated: neither by the gradients that come in nor by what it saved."""

    @functools.wraps(backward)
    def call(ctx, *grads):
        with torch.no_grad():
            results = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return results
        sources = [t for t in (*grads, *ctx.saved_tensors) if t is not None and t.requires_grad]
        return tuple(_Refusal.apply(t, *sources) if t is not None and sources else t for t in results)

    return call


# The library writes the rows in use.  Where a gradient is wanted the others are zeros: they reach the weights' gradients
# in the products of torch between the operators.

def _wanted(*inputs):
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs)


def _rows_like(x, zeros):
    return torch.zeros_like(x) if zeros else None


class _Norm(torch.autograd.Function):
    """layer_norm of x + residual, and the sum itself."""

    @staticmethod
    def forward(ctx, x, residual, weight, bias, eps, row_count, wanted):
        part = row_count is not None and wanted
        out, total, mean, rstd = mmbev.layer_norm(x, weight, bias, eps=eps, residual=residual, stats=True, row_count=row_count,
                                                  out=_rows_like(x, part), out_sum=_rows_like(x, part and residual is not None))
        ctx.save_for_backward(total, weight, mean, rstd, row_count)
        ctx.types = [None if t is None else t.dtype for t in (weight, bias)]
        return out, total

    @staticmethod
    @_once
    def backward(ctx, dout, dtotal):
        total, weight, mean, rstd, row_count = ctx.saved_tensors
        needed = ctx.needs_input_grad  # False where there is no such input
        dx, *sums = mmbev.layer_norm_backward(dout.contiguous(), total, weight, mean, rstd, dskip=dtotal.contiguous(),
                                              row_count=row_count, weight_grads=needed[2] or needed[3],
                                              dx=_rows_like(total, row_count is not None))
        dweight, dbias = (t.to(kind) if need else None for t, kind, need in zip(sums, ctx.types, needed[2:4]))
        return dx if needed[0] else None, dx if needed[1] else None, dweight, dbias, None, None, None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, steps, axis, layout, row_count, wanted):
        ctx.save_for_backward(positions, steps, axis, row_count)
        ctx.layout = layout
        part = row_count is not None and wanted
        return mmbev.rotary(x, positions, steps, axis, layout=layout, row_count=row_count, out=_rows_like(x, part))

    @staticmethod
    @_once
    def backward(ctx, dout):
        positions, steps, axis, row_count = ctx.saved_tensors
        dout = dout.contiguous()
        dx = mmbev.rotary(dout, positions, steps, axis, layout=ctx.layout, inverse=True, row_count=row_count,
                          out=_rows_like(dout, row_count is not None))
        return dx, None, None, None, None, None, None


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, offsets, initial_state, max_length, wanted):
        # the offsets alone know where the rows in use end
        out = q.new_zeros(*q.shape[:2], v.shape[2]) if wanted else None
        out, final = mmbev.linear_attention(q, k, v, log_decay, offsets, initial_state=initial_state, final_state=True,
                                            max_length=max_length, out=out)
        ctx.save_for_backward(q, k, v, log_decay, offsets, initial_state)
        ctx.max_length = max_length
        return out, final

    @staticmethod
    @_once
    def backward(ctx, dout, dfinal):
        q, k, v, log_decay, offsets, initial_state = ctx.saved_tensors
        dq, dk, dv, dinitial = mmbev.linear_attention_backward(
            dout.contiguous(), q, k, v, log_decay, offsets, initial_state=initial_state, dfinal_state=dfinal.contiguous(),
            dinitial_state=initial_state is not None, max_length=ctx.max_length, dq=torch.zeros_like(q), dk=torch.zeros_like(k),
            dv=torch.zeros_like(v))
        return dq, dk, dv, None, None, dinitial, None, None


class _HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, q_weight, k_weight, positions, steps, axis, eps, layout, row_count, wanted):
        ctx.save_for_backward(q, k, q_weight, k_weight, positions, steps, axis, row_count)
        ctx.form = eps, layout
        part = row_count is not None and wanted
        return mmbev.head_norm_rotary(q, k, q_weight, k_weight, positions, steps, axis, eps=eps, layout=layout, row_count=row_count,
                                      q_out=_rows_like(q, part), k_out=_rows_like(k, part))

    @staticmethod
    @_once
    def backward(ctx, dq_out, dk_out):
        q, k, q_weight, k_weight, positions, steps, axis, row_count = ctx.saved_tensors
        eps, layout = ctx.form
        needed, part = ctx.needs_input_grad, row_count is not None
        dq, dk, *sums = mmbev.head_norm_rotary_backward(
            dq_out.contiguous(), dk_out.contiguous(), q, k, q_weight, k_weight, positions, steps, axis, eps=eps, layout=layout,
            row_count=row_count, dq=_rows_like(q, part), dk=_rows_like(k, part), weight_grads=needed[2] or needed[3])
        dqw, dkw = (t.to(w.dtype) if need else None for t, w, need in zip(sums, (q_weight, k_weight), needed[2:4]))
        return dq if needed[0] else None, dk if needed[1] else None, dqw, dkw, None, None, None, None, None, None, None


class _GatedDelta(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay, beta, offsets, initial_state, max_length, wanted):
        # the offsets alone know where the rows in use end
        out = q.new_zeros(*q.shape[:2], v.shape[2]) if wanted else None
        out, final = mmbev.gated_delta(q, k, v, log_decay, beta, offsets, initial_state=initial_state, final_state=True,
                                       max_length=max_length, out=out)
        ctx.save_for_backward(q, k, v, log_decay, beta, offsets, initial_state)
        ctx.max_length = max_length
        return out, final

    @staticmethod
    @_once
    def backward(ctx, dout, dfinal):
        q, k, v, log_decay, beta, offsets, initial_state = ctx.saved_tensors
        *grads, dinitial = mmbev.gated_delta_backward(
            dout.contiguous(), q, k, v, log_decay, beta, offsets, initial_state=initial_state, dfinal_state=dfinal.contiguous(),
            dinitial_state=initial_state is not None, max_length=ctx.max_length, dq=torch.zeros_like(q), dk=torch.zeros_like(k),
            dv=torch.zeros_like(v), dlog_decay=torch.zeros_like(log_decay), dbeta=torch.zeros_like(beta))
        return *grads, None, dinitial, None, None


def norm(x, residual, weight, bias, eps=1e-5, row_count=None):
    """(layer_norm(x + residual), x + residual), differentiable."""
    return _Norm.apply(x, residual, weight, bias, eps, row_count, _wanted(x, residual, weight, bias))


def rotary(x, positions, steps, axis, layout="half", row_count=None):
    """mmbev.rotary, differentiable in x."""
    return _Rotary.apply(x, positions, steps, axis, layout, row_count, _wanted(x))


def linear_attention(q, k, v, log_decay, offsets, initial_state=None, max_length=None):
    """mmbev.linear_attention's (out, final state), differentiable in q, k, v and the initial state; log_decay is a constant."""
    if log_decay.requires_grad and torch.is_grad_enabled():
        raise mmbev.MmbevError("log_decay has no gradient: detach it")
    return _Attention.apply(q, k, v, log_decay, offsets, initial_state, max_length, _wanted(q, k, v, initial_state))


def head_norm_rotary(q, k, q_weight, k_weight, positions, steps, axis, eps=1e-6, layout="half", row_count=None):
    """mmbev.head_norm_rotary, differentiable in q, k and the weights."""
    return _HeadNorm.apply(q, k, q_weight, k_weight, positions, steps, axis, eps, layout, row_count, _wanted(q, k, q_weight, k_weight))


def gated_delta(q, k, v, log_decay, beta, offsets, initial_state=None, max_length=None):
    """mmbev.gated_delta's (out, final state), differentiable in all but the offsets."""
    return _GatedDelta.apply(q, k, v, log_decay, beta, offsets, initial_state, max_length,
                             _wanted(q, k, v, log_decay, beta, initial_state))


class Block(nn.Module):
    """Norm, attention over each frame's rows, and the residual sum (which the next norm takes in)."""

    def __init__(self, width, heads, kv_heads=None, head_dim=None, axes=3, base=1000.0, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.heads, self.kv_heads = heads, kv_heads or heads
        self.dim = head_dim or width // heads
        self.norm_weight = nn.Parameter(torch.ones(width, device=device))
        self.norm_bias = nn.Parameter(torch.zeros(width, device=device))
        rows = (self.heads + 2 * self.kv_heads) * self.dim
        self.qkv = nn.Parameter(torch.randn(width, rows, device=device, dtype=dtype) * width ** -0.5)
        self.out = nn.Parameter(torch.randn(self.heads * self.dim, width, device=device, dtype=dtype) * (self.heads * self.dim) ** -0.5)
        steps, axis = mmbev.make_rotary(self.dim - self.dim % 2, axes, base=base)
        self.register_buffer("steps", torch.from_numpy(steps).to(device))
        self.register_buffer("axis", torch.from_numpy(axis).to(device))
        # from some ten rows' memory to some ten thousand
        reach = torch.linspace(3.0, 13.0, heads, device=device)
        self.register_buffer("log_decay", torch.log1p(-torch.exp2(-reach)))

    def _project(self, x, branch, positions, row_count):
        y, x = norm(x, branch, self.norm_weight, self.norm_bias, row_count=row_count)
        rows = y @ self.qkv
        turned = self.heads + self.kv_heads  # queries and keys lie side by side: one call turns both
        qk = rotary(rows[:, :turned * self.dim].unflatten(1, (turned, self.dim)), positions, self.steps, self.axis,
                    row_count=row_count)
        v = rows[:, turned * self.dim:].unflatten(1, (self.kv_heads, self.dim))
        return x, qk[:, :self.heads], qk[:, self.heads:], v

    def forward(self, x, branch, coords, offsets, state=None, max_length=None, row_count=None):
        """x, branch [rows][width]: the rows and what the block before adds to them.  coords int32 [rows][4] and offsets
        int64 [frames+1] as the voxeliser writes them.  Returns (rows, branch to add, state after each frame)."""
        x, q, k, v = self._project(x, branch, coords[:, 1:], row_count)
        out, state = linear_attention(q, k, v, self.log_decay, offsets, state, max_length)
        return x, out.flatten(1) @ self.out, state

    @torch.no_grad()
    def step(self, x, branch, coords, state, slots=None):
        """One new row for each of many streams, whose states are updated in place."""
        x, q, k, v = self._project(x, branch, coords[:, 1:], None)
        out = mmbev.linear_attention_step(q, k, v, self.log_decay, state, slots)
        return x, out.flatten(1) @ self.out


class GatedBlock(Block):
    """The same with the gated delta rule: queries and keys normed for each head (keys to length 1, as the rule wants them)
    and turned in one pass; decays and rates of writing per row and head from the normed rows."""

    def __init__(self, width, heads, kv_heads=None, head_dim=None, axes=3, base=1000.0, dtype=torch.bfloat16, device="cuda"):
        super().__init__(width, heads, kv_heads, head_dim, axes, base, dtype, device)
        self.q_weight = nn.Parameter(torch.full((self.dim,), self.dim ** -0.5, device=device))
        self.register_buffer("k_weight", torch.full((self.dim,), self.dim ** -0.5, device=device))
        self.gates = nn.Parameter(torch.randn(width, 2 * heads, device=device) * width ** -0.5)
        # the decays that Block's heads have, times softplus(gate) / ln 2, which is 1 at a gate of 0
        self.rate = nn.Parameter((-self.log_decay).log())

    def _project(self, x, branch, positions, row_count):
        y, x = norm(x, branch, self.norm_weight, self.norm_bias, row_count=row_count)
        rows = y @ self.qkv
        q, k, v = (t.unflatten(1, (-1, self.dim)) for t in
                   rows.split([self.heads * self.dim, self.kv_heads * self.dim, self.kv_heads * self.dim], dim=1))
        q, k = head_norm_rotary(q, k, self.q_weight, self.k_weight, positions, self.steps, self.axis, row_count=row_count)
        decay, beta = (y.float() @ self.gates).chunk(2, dim=1)
        log_decay = -self.rate.exp() * nn.functional.softplus(decay) / math.log(2.0)
        return x, q, k, v, log_decay, torch.sigmoid(beta)

    def forward(self, x, branch, coords, offsets, state=None, max_length=None, row_count=None):
        """As Block's."""
        x, q, k, v, log_decay, beta = self._project(x, branch, coords[:, 1:], row_count)
        out, state = gated_delta(q, k, v, log_decay, beta, offsets, state, max_length)
        return x, out.flatten(1) @ self.out, state

    @torch.no_grad()
    def step(self, x, branch, coords, state, slots=None):
        """One new row for each of many streams, whose states are updated in place."""
        x, q, k, v, log_decay, beta = self._project(x, branch, coords[:, 1:], None)
        out = mmbev.gated_delta_step(q, k, v, log_decay, beta, state, slots)
        return x, out.flatten(1) @ self.out


class VoxelEncoder(nn.Module):
    """Voxel features [rows][features] to encoded ones [rows][out_features], fp32, as mmbev.scatter_to_bev takes them.
    gated: its blocks are GatedBlocks."""

    def __init__(self, features, width=128, heads=4, depth=2, out_features=32, dtype=torch.bfloat16, device="cuda", gated=False,
                 **block):
        super().__init__()
        self.dtype = dtype
        self.embed = nn.Parameter(torch.randn(features, width, device=device, dtype=dtype) * features ** -0.5)
        kind = GatedBlock if gated else Block
        self.blocks = nn.ModuleList(kind(width, heads, dtype=dtype, device=device, **block) for _ in range(depth))
        self.norm_weight = nn.Parameter(torch.ones(width, device=device))
        self.norm_bias = nn.Parameter(torch.zeros(width, device=device))
        self.head = nn.Parameter(torch.randn(width, out_features, device=device, dtype=dtype) * width ** -0.5)

    def _finish(self, x, branch, row_count):
        y, _ = norm(x, branch, self.norm_weight, self.norm_bias, row_count=row_count)
        return (y @ self.head).float()

    def forward(self, feats, coords, offsets, states=None, max_length=None, row_count=None):
        """Returns (encoded features, the blocks' states after each frame)."""
        if row_count is not None and torch.is_grad_enabled():  # what lies past the count would enter the weights' gradients
            feats = torch.where(torch.arange(feats.shape[0], device=feats.device)[:, None] < row_count, feats, 0.0)
        x = feats.to(self.dtype) @ self.embed
        branch, after = torch.zeros_like(x), []
        for i, block in enumerate(self.blocks):
            x, branch, state = block(x, branch, coords, offsets, states[i] if states else None, max_length, row_count)
            after.append(state)
        return self._finish(x, branch, row_count), after

    @torch.no_grad()
    def step(self, feats, coords, states, slots=None):
        """One new voxel row for each of many streams; `states` (as forward returns them) are updated in place."""
        x = feats.to(self.dtype) @ self.embed
        branch = torch.zeros_like(x)
        for block, state in zip(self.blocks, states):
            x, branch = block.step(x, branch, coords, state, slots)
        return self._finish(x, branch, None)
