"""Forgetting Attention as a PyTorch autograd function.

Glue only: the forward runs fox_gate_prefix and fox_attn_fwd, the backward the
staged backward (recomputing, or keeping dS when asked and the dtype is bf16)
and fox_dlogit_from_dc, which returns the gradient of the gate logits through
log f = logsigmoid(logit) and c = cumsum(log f) (Sec. 3).  GateProjection
gives the logits themselves from the layer input, w_f^T x_t + b_f per head,
with fox_gate_projection and fox_gate_projection_bwd.  Every step runs in the
library's kernels.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import _lib as fox
from . import _packed


class ForgettingAttention(torch.autograd.Function):
    """o = FoX attention of q, k, v [B,H,L,d] with gate logits [B,H,L] (fp32)."""

    @staticmethod
    def forward(ctx, q, k, v, gate_logit, scale, keep_ds):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        gate_logit = gate_logit.contiguous()
        c = fox.fox_gate_prefix(gate_logit)
        o, lse = fox.fox_attn_fwd(q, k, v, c, scale)
        ctx.save_for_backward(q, k, v, gate_logit, c, o, lse)
        ctx.scale = scale
        ctx.keep_ds = bool(keep_ds) and q.dtype == torch.bfloat16
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, gate_logit, c, o, lse = ctx.saved_tensors
        d_o = d_o.to(q.dtype).contiguous()
        dq, dk, dv, d_logit = fox._attn_bwd_logit(q, k, v, c, o, lse, gate_logit, d_o, ctx.scale,
                                                  ctx.keep_ds)
        return dq, dk, dv, d_logit, None, None


def forgetting_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                         gate_logit: torch.Tensor, scale: Optional[float] = None,
                         keep_ds: bool = False) -> torch.Tensor:
    """Causal Forgetting Attention with autograd support.

    q, k, v: [B, H, L, d] bf16 or fp32 on the GPU (d = 64 or 128); gate_logit:
    [B, H, L] fp32, the forget gate f = sigmoid(gate_logit).  scale defaults to
    1/sqrt(d).  keep_ds (bf16): the backward keeps dS in a temporary workspace of
    about B*H*L^2 bytes instead of recomputing it for dQ (faster at long L).
    """
    s = fox.default_scale(q.shape[-1]) if scale is None else float(scale)
    return ForgettingAttention.apply(q, k, v, gate_logit, s, keep_ds)


class PackedForgettingAttention(torch.autograd.Function):
    """o [H,N,d] of packed sequences: q [H,N,d], k, v [H_kv,N,d], gate logits [H,N]."""

    @staticmethod
    def forward(ctx, q, k, v, gate_logit, cu_seqlens, plan, max_len, scale):
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        gate_logit = gate_logit.contiguous()
        plan, c, o, o_lo, lse = _packed._step_forward(q, k, v, gate_logit, cu_seqlens, plan,
                                                      max_len, scale)
        ctx.save_for_backward(q, k, v, gate_logit, c, o, o_lo, lse, cu_seqlens, plan)
        ctx.max_len, ctx.scale = max_len, scale
        return o

    @staticmethod
    def backward(ctx, d_o):
        saved = ctx.saved_tensors
        grads = _packed._step_backward(saved, d_o.to(saved[0].dtype).contiguous(), ctx.max_len,
                                       ctx.scale)
        return (*grads, None, None, None, None)


def forgetting_attention_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                gate_logit: torch.Tensor, cu_seqlens: torch.Tensor,
                                max_len: int = 0, scale: Optional[float] = None,
                                plan: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal Forgetting Attention of packed sequences with grouped heads, with autograd
    support.

    q: [H, N, d], k, v: [H_kv, N, d] bf16 or fp32 on the GPU (d = 64 or 128, H a multiple of
    H_kv); gate_logit: [H, N] fp32 or bf16; cu_seqlens: [B + 1] int32, sequence b being rows
    cu_seqlens[b] .. cu_seqlens[b + 1] - 1.  max_len: the longest sequence, if known (it sets
    how the work is split; without it batches of short sequences are slower and take a workspace
    of fp32 partial sums).  plan: fox_packed_plan(cu_seqlens, N), to share it between layers.
    The output and the gradients are zero in rows behind the last sequence.  bf16: a tensor of
    o's size is kept besides o (what rounding took from it) for dq.

    Forward and backward may be captured into a graph, from leaves of which no eager autograd
    graph lives (torch would wait for that graph's stream inside the capture): capture from
    detached ones.
    """
    s = fox.default_scale(q.shape[-1]) if scale is None else float(scale)
    return PackedForgettingAttention.apply(q, k, v, gate_logit, cu_seqlens, plan, max_len, s)


class GateProjection(torch.autograd.Function):
    """gate_logit[b, h, t] = w_f[h] . x[b, t] + b_f[h] (Sec. 3, gate definition)."""

    @staticmethod
    def forward(ctx, x, w_f, b_f):
        x, w_f = x.contiguous(), w_f.contiguous()
        b = None if b_f is None else b_f.contiguous()
        logit = fox.fox_gate_projection(x, w_f, b)
        ctx.save_for_backward(x, w_f)
        ctx.has_bias = b_f is not None
        return logit

    @staticmethod
    def backward(ctx, d_logit):
        x, w_f = ctx.saved_tensors
        dx, dw, db = fox.fox_gate_projection_bwd(x, w_f, d_logit.contiguous(),
                                                 want_dx=ctx.needs_input_grad[0],
                                                 want_db=ctx.has_bias)
        return dx, dw, db


def forget_gate_logits(x: torch.Tensor, w_f: torch.Tensor,
                       b_f: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The forget-gate logits [B, H, L] fp32 from the layer input x [B, L, M]
    (bf16 or fp32, M % 8 == 0), w_f [H, M] and b_f [H] fp32 (H <= 64), with
    autograd support; feed them to forgetting_attention."""
    return GateProjection.apply(x, w_f, b_f)
