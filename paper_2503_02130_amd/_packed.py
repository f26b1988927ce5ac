"""ctypes binding of the attention over packed sequences: argument marshalling only, as in
_lib.py."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch

from ._lib import (_DT, _call, _check, _check_int, _need, _ptr, _raise, _workspace,
                   _workspace_bytes, default_scale, load)


class _RowsStruct(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("heads", ctypes.c_int), ("row_bytes", ctypes.c_int)]


def _check_cu(cu: torch.Tensor, device):
    """The number of sequences."""
    B = cu.shape[0] - 1
    if cu.dim() != 1 or B < 1:
        raise ValueError(f"cu_seqlens must have shape (B + 1,) with B >= 1 (got {tuple(cu.shape)})")
    _check(cu, "cu_seqlens", (B + 1,), torch.int32, device)
    return B


def _plan_places(B: int, N: int) -> int:
    """Places of fox_packed_plan_bytes(), 16 bytes each."""
    return N // 128 + min(B, N)


def _check_plan(plan: torch.Tensor, B: int, N: int, device):
    _need(plan, "plan", (_plan_places(B, N) * 4,), torch.int32, device)


def _check_qkv(q, k, v):
    """H, H_kv, N, d of packed q [H,N,d] and k, v [H_kv,N,d]."""
    H, N, d = q.shape
    dt, dev = q.dtype, q.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    Hkv = k.shape[0]
    _check(q, "q", (H, N, d), dt, None)
    _need(k, "k", (Hkv, N, d), dt, dev)
    _need(v, "v", (Hkv, N, d), dt, dev)
    return H, Hkv, N, d


def fox_packed_plan(cu_seqlens: torch.Tensor, N: int) -> torch.Tensor:
    """The work list of a batch of packed sequences (cu_seqlens [B+1] int32, N rows), for
    fox_attn_fwd_packed and fox_attn_bwd_packed of every layer."""
    _check_int(N, "N")
    B, dev = _check_cu(cu_seqlens, None), cu_seqlens.device
    lib = load()
    places = _plan_places(B, N)
    plan = torch.empty((places * 4,), device=dev, dtype=torch.int32)
    st = _call(lib.fox_packed_plan, dev, _ptr(cu_seqlens), B, N, _ptr(plan), 16 * places, None, 0)
    _raise(st, "fox_packed_plan")
    return plan


def fox_gate_prefix_packed(gate_logit: torch.Tensor, cu_seqlens: torch.Tensor,
                           c: Optional[torch.Tensor] = None) -> torch.Tensor:
    """c [H,N] fp32, the running sum of log sigmoid(gate_logit) within each sequence;
    gate_logit [H,N] fp32 or bf16."""
    H, N = gate_logit.shape
    _check_int(N, "N")
    dt, dev = gate_logit.dtype, gate_logit.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    _check(gate_logit, "gate_logit", (H, N), dt, None)
    B = _check_cu(cu_seqlens, dev)
    if c is None:
        c = torch.empty((H, N), device=dev, dtype=torch.float32)
    else:
        _need(c, "c", (H, N), torch.float32, dev)
    st = _call(load().fox_gate_prefix_packed, dev, _DT[dt], _ptr(gate_logit), _ptr(cu_seqlens),
               _ptr(c), B, H, N)
    _raise(st, "fox_gate_prefix_packed")
    return c


def fox_packed_start(gate_logit: torch.Tensor, cu_seqlens: torch.Tensor
                     ) -> Tuple[torch.Tensor, torch.Tensor]:
    """(plan, c): fox_packed_plan and fox_gate_prefix_packed in one launch."""
    H, N = gate_logit.shape
    _check_int(N, "N")
    dt, dev = gate_logit.dtype, gate_logit.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    _check(gate_logit, "gate_logit", (H, N), dt, None)
    B = _check_cu(cu_seqlens, dev)
    places = _plan_places(B, N)
    plan = torch.empty((places * 4,), device=dev, dtype=torch.int32)
    c = torch.empty((H, N), device=dev, dtype=torch.float32)
    st = _call(load().fox_packed_start, dev, _DT[dt], _ptr(gate_logit), _ptr(cu_seqlens), _ptr(c), B,
               H, N, _ptr(plan), 16 * places, None, 0)
    _raise(st, "fox_packed_start")
    return plan, c


def fox_attn_fwd_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, c: torch.Tensor,
                        cu_seqlens: torch.Tensor, plan: Optional[torch.Tensor] = None,
                        max_len: int = 0, scale: Optional[float] = None,
                        o: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                        o_lo: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """O [H,N,d] (q's dtype) and LSE [H,N] fp32 of packed sequences: q [H,N,d], k, v
    [H_kv,N,d] bf16 or fp32, c from fox_gate_prefix_packed, plan from fox_packed_plan.
    max_len: the longest sequence, if known.  o_lo (bf16), if given, is filled with what rounding
    took from O, for the backward.  Rows behind the last sequence are not written."""
    H, Hkv, N, d = _check_qkv(q, k, v)
    dev = q.device
    _need(c, "c", (H, N), torch.float32, dev)
    B = _check_cu(cu_seqlens, dev)
    if plan is None:
        plan = fox_packed_plan(cu_seqlens, N)
    else:
        _check_plan(plan, B, N, dev)
    if o is None:
        o = torch.empty_like(q)
    else:
        _need(o, "o", (H, N, d), q.dtype, dev)
    if lse is None:
        lse = torch.empty((H, N), device=dev, dtype=torch.float32)
    else:
        _need(lse, "lse", (H, N), torch.float32, dev)
    if o_lo is not None:
        _need(o_lo, "o_lo", (H, N, d), torch.bfloat16, dev)
    s = default_scale(d) if scale is None else float(scale)
    st = _call(load().fox_attn_fwd_packed, dev, _DT[q.dtype], _ptr(q), _ptr(k), _ptr(v), _ptr(c),
               _ptr(plan), _ptr(o), _ptr(o_lo), _ptr(lse), B, H, Hkv, N, d, max_len, s)
    _raise(st, "fox_attn_fwd_packed")
    return o, lse


def fox_attn_bwd_packed_workspace_bytes(dtype: torch.dtype, H: int, H_kv: int, N: int, d: int,
                                        max_len: int = 0) -> int:
    return int(load().fox_attn_bwd_packed_workspace_bytes(_DT[dtype], H, H_kv, N, d, max_len))


def fox_attn_bwd_packed(q, k, v, c, o, lse, d_o, gate_logit: torch.Tensor,
                        cu_seqlens: torch.Tensor, plan: Optional[torch.Tensor] = None,
                        max_len: int = 0, scale: Optional[float] = None, dq=None, dk=None,
                        dv=None, d_logit=None, d_log_f=None, workspace=None, o_lo=None):
    """dq [H,N,d], dk, dv [H_kv,N,d] and d_logit [H,N] (the gate logits' dtype, fp32 or bf16)
    of sum(o * d_o); d_log_f [H,N] fp32 is filled if given; o_lo as the forward left it.  Rows behind the last sequence are
    not written."""
    H, Hkv, N, d = _check_qkv(q, k, v)
    dt, dev = q.dtype, q.device
    for name, t in (("o", o), ("d_o", d_o)):
        _need(t, name, (H, N, d), dt, dev)
    if o_lo is not None:
        _need(o_lo, "o_lo", (H, N, d), torch.bfloat16, dev)
    for name, t in (("c", c), ("lse", lse)):
        _need(t, name, (H, N), torch.float32, dev)
    gdt = gate_logit.dtype
    if gdt not in _DT:
        raise ValueError(f"unsupported dtype {gdt}")
    _need(gate_logit, "gate_logit", (H, N), gdt, dev)
    B = _check_cu(cu_seqlens, dev)
    if plan is None:
        plan = fox_packed_plan(cu_seqlens, N)
    else:
        _check_plan(plan, B, N, dev)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    d_logit = torch.empty_like(gate_logit) if d_logit is None else d_logit
    _need(dq, "dq", (H, N, d), dt, dev)
    _need(dk, "dk", (Hkv, N, d), dt, dev)
    _need(dv, "dv", (Hkv, N, d), dt, dev)
    _need(d_logit, "d_logit", (H, N), gdt, dev)
    if d_log_f is not None:
        _need(d_log_f, "d_log_f", (H, N), torch.float32, dev)
    lib = load()
    if workspace is None:
        nbytes = lib.fox_attn_bwd_packed_workspace_bytes(_DT[dt], H, Hkv, N, d, max_len)
        workspace = _workspace(nbytes, dev)
    else:
        nbytes = _workspace_bytes(workspace, dev)
    s = default_scale(d) if scale is None else float(scale)
    st = _call(lib.fox_attn_bwd_packed, dev, _DT[dt], _ptr(q), _ptr(k), _ptr(v), _ptr(c), _ptr(o),
               _ptr(o_lo), _ptr(lse), _ptr(d_o), _DT[gdt], _ptr(gate_logit), _ptr(cu_seqlens),
               _ptr(plan), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(d_logit), _ptr(d_log_f), 0, _ptr(workspace),
               nbytes, B, H, Hkv, N, d, max_len, s)
    _raise(st, "fox_attn_bwd_packed")
    return dq, dk, dv, d_logit


def fox_packed_zero_behind(tensors: Sequence[torch.Tensor], cu_seqlens: torch.Tensor) -> None:
    """Zeros in the rows behind the last sequence of up to 8 packed tensors [heads, N, ...]."""
    if not 1 <= len(tensors) <= 8:
        raise ValueError(f"1 to 8 tensors (got {len(tensors)})")
    N = tensors[0].shape[1]
    _check_int(N, "N")
    B, dev = _check_cu(cu_seqlens, None), cu_seqlens.device
    rows = (_RowsStruct * len(tensors))()
    for i, t in enumerate(tensors):
        _need(t, f"tensors[{i}]", (t.shape[0], N, *t.shape[2:]), None, dev)
        rows[i].x, rows[i].heads = _ptr(t), t.shape[0]
        rows[i].row_bytes = t[0, 0].numel() * t.element_size()
    st = _call(load().fox_packed_zero_behind, dev, ctypes.addressof(rows), len(tensors),
               _ptr(cu_seqlens), B, N)
    _raise(st, "fox_packed_zero_behind")


# ---------------------------------------------------------------------------
# The two halves of an autograd step, each with one pass of checks.
def _step_forward(q, k, v, gate_logit, cu_seqlens, plan, max_len, scale):
    """(plan, c, o, o_lo, lse), o zero behind the last sequence; o_lo None for fp32."""
    H, Hkv, N, d = _check_qkv(q, k, v)
    dt, dev = _DT[q.dtype], q.device
    gdt = gate_logit.dtype
    if gdt not in _DT:
        raise ValueError(f"unsupported dtype {gdt}")
    _need(gate_logit, "gate_logit", (H, N), gdt, dev)
    B = _check_cu(cu_seqlens, dev)
    lib, cu = load(), _ptr(cu_seqlens)
    c, lse = (torch.empty((H, N), device=dev, dtype=torch.float32) for _ in range(2))
    o = torch.empty_like(q)
    o_lo = torch.empty_like(q) if q.dtype == torch.bfloat16 else None
    row = _RowsStruct(_ptr(o), H, d * o.element_size())
    if plan is None:
        places = _plan_places(B, N)
        plan = torch.empty((places * 4,), device=dev, dtype=torch.int32)
        _raise(_call(lib.fox_packed_start, dev, _DT[gdt], _ptr(gate_logit), cu, _ptr(c), B, H, N,
                     _ptr(plan), 16 * places, ctypes.addressof(row), 1), "fox_packed_start")
    else:
        _check_plan(plan, B, N, dev)
        _raise(_call(lib.fox_packed_zero_behind, dev, ctypes.addressof(row), 1, cu, B, N),
               "fox_packed_zero_behind")
        _raise(_call(lib.fox_gate_prefix_packed, dev, _DT[gdt], _ptr(gate_logit), cu, _ptr(c), B, H,
                     N), "fox_gate_prefix_packed")
    _raise(_call(lib.fox_attn_fwd_packed, dev, dt, _ptr(q), _ptr(k), _ptr(v), _ptr(c), _ptr(plan),
                 _ptr(o), _ptr(o_lo), _ptr(lse), B, H, Hkv, N, d, max_len, scale),
           "fox_attn_fwd_packed")
    return plan, c, o, o_lo, lse


def _step_backward(saved, d_o, max_len, scale):
    """dq, dk, dv, d_logit, zero behind the last sequence, from what the forward checked."""
    q, k, v, gate_logit, c, o, o_lo, lse, cu_seqlens, plan = saved
    (H, N, d), Hkv, B = q.shape, k.shape[0], cu_seqlens.shape[0] - 1
    dt, gdt, dev = q.dtype, gate_logit.dtype, q.device
    _need(d_o, "d_o", (H, N, d), dt, dev)
    lib, cu = load(), _ptr(cu_seqlens)
    grads = (torch.empty_like(q), torch.empty_like(k), torch.empty_like(v),
             torch.empty_like(gate_logit))
    nbytes = lib.fox_attn_bwd_packed_workspace_bytes(_DT[dt], H, Hkv, N, d, max_len)
    ws = _workspace(nbytes, dev)
    _raise(_call(lib.fox_attn_bwd_packed, dev, _DT[dt], _ptr(q), _ptr(k), _ptr(v), _ptr(c),
                 _ptr(o), _ptr(o_lo), _ptr(lse), _ptr(d_o), _DT[gdt], _ptr(gate_logit), cu,
                 _ptr(plan), *map(_ptr, grads), None, 1, _ptr(ws), nbytes, B, H, Hkv, N, d, max_len, scale),
           "fox_attn_bwd_packed")
    return grads
