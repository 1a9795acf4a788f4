"""The operators of a trained layer as functions with gradients (``torch.autograd``): rotary positions, attention over packed
sequences, dropout with bias and residual.  Each call allocates its outputs and hands them to the binding, which runs the
library's kernels; there is no fallback.  A program that owns its buffers calls the binding itself."""
from __future__ import annotations

import dataclasses
import functools
from typing import Optional, Tuple

import torch

from . import binding as ps


@dataclasses.dataclass(frozen=True)
class Sequences:
    """Which rows of packed tensors belong together, and what they see (``include/preserve.h``, ps_attention_seqs)."""
    q_offsets: torch.Tensor
    k_offsets: torch.Tensor
    max_q: int
    max_k: int
    k_lengths: Optional[torch.Tensor] = None
    q_start: Optional[torch.Tensor] = None
    prefix: Optional[torch.Tensor] = None
    q_docs: Optional[torch.Tensor] = None
    k_docs: Optional[torch.Tensor] = None
    status: Optional[torch.Tensor] = None      # raised by faulty sequences, in both directions (``binding.new_status``, ``ps_status_read``)

    def arguments(self) -> dict:
        return {n: getattr(self, n) for n in ("k_lengths", "q_start", "prefix", "q_docs", "k_docs", "status")}


def _constant(t: Optional[torch.Tensor], where: str, name: str) -> None:
    if t is not None and t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{where}: {name} have no gradient; detach them")


class _NoSecond(torch.autograd.Function):
    @staticmethod
    def forward(ctx, grad):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the layer functions have no second derivatives")


def _first_only(backward):
    """A backward pass whose gradients, where a graph of them is asked for (``create_graph=True``), raise an error when differentiated.
    (torch's ``once_differentiable`` does so only if the incoming gradient has a graph of its own, and a sum's has none.)"""
    @functools.wraps(backward)
    def run(ctx, *grads):
        with torch.no_grad():
            got = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return got
        return tuple(None if g is None else _NoSecond.apply(g.detach().requires_grad_()) for g in got)
    return run


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, seqs, scale, softcap, causal, slopes):
        train = any(ctx.needs_input_grad[:3])
        out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)             # (the kernels leave rows that no sequence has alone)
        lse = torch.empty(q.shape[1], q.shape[0], device=q.device)
        rest = torch.empty_like(out) if train and q.dtype == torch.bfloat16 else None
        shape = (seqs.q_offsets.numel() - 1, q.shape[0], k.shape[0], seqs.max_q, seqs.max_k, q.shape[1], k.shape[1], q.shape[2], q.dtype)
        ws = ps.alloc_workspace(ps.ps_attention_workspace_bytes(*shape), q.device)
        masks = dict(seqs.arguments(), slopes=slopes)
        ctx.how = dict(scale=scale, softcap=softcap, causal=causal, status=masks.pop("status"))
        ctx.bounds, ctx.shape, ctx.masks = (seqs.max_q, seqs.max_k), shape, tuple(masks)
        ps.ps_attention_forward(q, k, v, seqs.q_offsets, seqs.k_offsets, *ctx.bounds, out, lse, ws, out_rest=rest, **masks, **ctx.how)
        # (all that the gradients depend on, so that what is written again in between does not go unnoticed)
        ctx.save_for_backward(q, k, v, out, lse, rest, seqs.q_offsets, seqs.k_offsets, *masks.values())
        return out

    @staticmethod
    @_first_only
    def backward(ctx, dout):
        q, k, v, out, lse, rest, q_offsets, k_offsets, *masks = ctx.saved_tensors
        dout = dout.contiguous()
        if dout.data_ptr() % 16:                                # (part of a larger gradient, as torch.cat hands them back)
            dout = dout.clone()
        # (rows that no sequence has get no gradient)
        grads = [torch.zeros(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v)]
        ws = ps.alloc_workspace(ps.ps_attention_workspace_bytes(*ctx.shape, backward=True), q.device)
        ps.ps_attention_backward(q, k, v, out, lse, dout, q_offsets, k_offsets, *ctx.bounds, *grads, ws, out_rest=rest,
                                 **dict(zip(ctx.masks, masks)), **ctx.how)
        return (*grads, None, None, None, None, None)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, seqs: Sequences, scale: Optional[float] = None, softcap: float = 0.0,
              causal: bool = False, slopes: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of packed q [n_q, heads, size] to k, v [n_k, kv_heads, size]; slopes are constants.  Rows that no sequence has, or a
    faulty one, are zeros, as is their gradient; faulty sequences are told in ``seqs.status``."""
    _constant(slopes, "attention", "slopes")
    return _Attention.apply(q, k, v, seqs, scale, softcap, causal, slopes)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, frequencies, interleaved, magnitude):
        out = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k)]
        ps.ps_rotary(q, positions, frequencies, out[0], k, out[1], interleaved, magnitude)
        ctx.save_for_backward(positions, frequencies)
        ctx.how = interleaved, magnitude
        return tuple(out)

    @staticmethod
    @_first_only
    def backward(ctx, dq, dk):
        positions, frequencies = ctx.saved_tensors
        dq, dk = (t if t.stride(-1) == 1 else t.contiguous() for t in (dq, dk))
        grads = [torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (dq, dk)]
        ps.ps_rotary(dq, positions, frequencies, grads[0], dk, grads[1], *ctx.how, inverse=True)
        return (*grads, None, None, None, None)


def rotary(q: torch.Tensor, k: torch.Tensor, positions: torch.Tensor, frequencies: torch.Tensor, interleaved: bool = False,
           magnitude: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """Queries and keys turned to their positions; frequencies are constants."""
    _constant(frequencies, "rotary", "frequencies")
    return _Rotary.apply(q, k, positions, frequencies, interleaved, magnitude)


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, bias, residual, rng, p):
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        ps.ps_dropout_forward(x, bias, residual, rng, p, out)
        ctx.save_for_backward(rng)
        ctx.p, ctx.bias = p, None if bias is None else bias.dtype
        return out

    @staticmethod
    @_first_only
    def backward(ctx, dout):
        (rng,) = ctx.saved_tensors
        dout = dout.contiguous()
        dx = torch.empty(dout.shape, dtype=dout.dtype, device=dout.device)
        dbias = ws = None
        if ctx.bias is not None and ctx.needs_input_grad[1]:
            dbias = torch.empty(dout.shape[1], device=dout.device)
            ws = ps.alloc_workspace(ps.ps_dropout_workspace_bytes(*dout.shape), dout.device)
        ps.ps_dropout_backward(dout, rng, ctx.p, dx, dbias, ws)
        return dx, None if dbias is None else dbias.to(ctx.bias), dout if ctx.needs_input_grad[2] else None, None, None


def dropout_add(x: torch.Tensor, bias: Optional[torch.Tensor], residual: Optional[torch.Tensor], rng: torch.Tensor, p: float,
                move_on: bool = True) -> torch.Tensor:
    """residual + dropout(x + bias) of [rows, cols]; rng: two int64 on the GPU, seed and number of the call, which moves on by one.

    With ``move_on=False`` rng stays as it is, and has to until the gradients are taken.  A pass that is made again for its gradients
    (activation checkpointing) needs that, since it has to draw what it drew the first time: calls in it get tensors of their own
    (``rng + rng.new_tensor([0, n])``), and the caller goes on to others.  A call that would move on in such a pass is refused."""
    if not move_on:
        return _Dropout.apply(x, bias, residual, rng, p)
    if torch._C._current_graph_task_id() != -1:                 # (gradients are being taken)
        raise RuntimeError("dropout_add: a pass that is made again for its gradients would draw another mask; call it with move_on=False")
    drawn = rng.clone()                                         # what this call draws from
    rng[1:].add_(1)
    return _Dropout.apply(x, bias, residual, drawn, p)
