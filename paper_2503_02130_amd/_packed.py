"""ctypes binding of the attention over packed sequences: argument marshalling only, as in
_lib.py."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple

import torch

from ._lib import (_DT, _check, _on_device, _ptr, _raise, _raw_stream, _workspace, default_scale,
                   load)


class _RowsStruct(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("heads", ctypes.c_int), ("row_bytes", ctypes.c_int)]


def _check_cu(cu: torch.Tensor, device):
    """The number of sequences."""
    B = cu.shape[0] - 1
    if cu.dim() != 1 or B < 1:
        raise ValueError(f"cu_seqlens must have shape (B + 1,) with B >= 1 (got {tuple(cu.shape)})")
    _check(cu, "cu_seqlens", (B + 1,), torch.int32, device)
    return B


def _check_plan(plan: torch.Tensor, B: int, N: int, device):
    _check(plan, "plan", (load().fox_packed_plan_bytes(B, N) // 4,), torch.int32, device)


def _check_qkv(q, k, v):
    """H, H_kv, N, d of packed q [H,N,d] and k, v [H_kv,N,d]."""
    H, N, d = q.shape
    dt, dev = q.dtype, q.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    Hkv = k.shape[0]
    _check(q, "q", (H, N, d), dt, None)
    _check(k, "k", (Hkv, N, d), dt, dev)
    _check(v, "v", (Hkv, N, d), dt, dev)
    return H, Hkv, N, d


def fox_packed_plan(cu_seqlens: torch.Tensor, N: int) -> torch.Tensor:
    """The work list of a batch of packed sequences (cu_seqlens [B+1] int32, N rows), for
    fox_attn_fwd_packed and fox_attn_bwd_packed of every layer."""
    B, dev = _check_cu(cu_seqlens, None), cu_seqlens.device
    lib = load()
    nbytes = lib.fox_packed_plan_bytes(B, N)
    plan = torch.empty(max(nbytes // 4, 4), device=dev, dtype=torch.int32)
    with _on_device(dev):
        st = lib.fox_packed_plan(_ptr(cu_seqlens), B, N, _ptr(plan), nbytes,
                                 _raw_stream(dev.index))
    _raise(st, "fox_packed_plan")
    return plan


def fox_gate_prefix_packed(gate_logit: torch.Tensor, cu_seqlens: torch.Tensor,
                           c: Optional[torch.Tensor] = None) -> torch.Tensor:
    """c [H,N] fp32, the running sum of log sigmoid(gate_logit) within each sequence;
    gate_logit [H,N] fp32 or bf16."""
    H, N = gate_logit.shape
    dt, dev = gate_logit.dtype, gate_logit.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    _check(gate_logit, "gate_logit", (H, N), dt, None)
    B = _check_cu(cu_seqlens, dev)
    if c is None:
        c = torch.empty((H, N), device=dev, dtype=torch.float32)
    else:
        _check(c, "c", (H, N), torch.float32, dev)
    with _on_device(dev):
        st = load().fox_gate_prefix_packed(_DT[dt], _ptr(gate_logit), _ptr(cu_seqlens), _ptr(c),
                                           B, H, N, _raw_stream(dev.index))
    _raise(st, "fox_gate_prefix_packed")
    return c


def fox_attn_fwd_packed(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, c: torch.Tensor,
                        cu_seqlens: torch.Tensor, plan: Optional[torch.Tensor] = None,
                        max_len: int = 0, scale: Optional[float] = None,
                        o: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None
                        ) -> Tuple[torch.Tensor, torch.Tensor]:
    """O [H,N,d] (q's dtype) and LSE [H,N] fp32 of packed sequences: q [H,N,d], k, v
    [H_kv,N,d] bf16 or fp32, c from fox_gate_prefix_packed, plan from fox_packed_plan.
    max_len: the longest sequence, if known.  Rows behind the last sequence are not written."""
    H, Hkv, N, d = _check_qkv(q, k, v)
    dev = q.device
    _check(c, "c", (H, N), torch.float32, dev)
    B = _check_cu(cu_seqlens, dev)
    if plan is None:
        plan = fox_packed_plan(cu_seqlens, N)
    else:
        _check_plan(plan, B, N, dev)
    if o is None:
        o = torch.empty_like(q)
    else:
        _check(o, "o", (H, N, d), q.dtype, dev)
    if lse is None:
        lse = torch.empty((H, N), device=dev, dtype=torch.float32)
    else:
        _check(lse, "lse", (H, N), torch.float32, dev)
    s = default_scale(d) if scale is None else float(scale)
    with _on_device(dev):
        st = load().fox_attn_fwd_packed(_DT[q.dtype], _ptr(q), _ptr(k), _ptr(v), _ptr(c),
                                        _ptr(plan), _ptr(o), _ptr(lse), B, H, Hkv, N, d, max_len,
                                        s, _raw_stream(dev.index))
    _raise(st, "fox_attn_fwd_packed")
    return o, lse


def fox_attn_bwd_packed_workspace_bytes(H: int, N: int) -> int:
    return int(load().fox_attn_bwd_packed_workspace_bytes(H, N))


def fox_attn_bwd_packed(q, k, v, c, o, lse, d_o, gate_logit: torch.Tensor,
                        cu_seqlens: torch.Tensor, plan: Optional[torch.Tensor] = None,
                        max_len: int = 0, scale: Optional[float] = None, dq=None, dk=None,
                        dv=None, d_logit=None, d_log_f=None, workspace=None):
    """dq [H,N,d], dk, dv [H_kv,N,d] and d_logit [H,N] (the gate logits' dtype, fp32 or bf16)
    of sum(o * d_o); d_log_f [H,N] fp32 is filled if given.  Rows behind the last sequence are
    not written."""
    H, Hkv, N, d = _check_qkv(q, k, v)
    dt, dev = q.dtype, q.device
    for name, t in (("o", o), ("d_o", d_o)):
        _check(t, name, (H, N, d), dt, dev)
    for name, t in (("c", c), ("lse", lse)):
        _check(t, name, (H, N), torch.float32, dev)
    gdt = gate_logit.dtype
    if gdt not in _DT:
        raise ValueError(f"unsupported dtype {gdt}")
    _check(gate_logit, "gate_logit", (H, N), gdt, dev)
    B = _check_cu(cu_seqlens, dev)
    if plan is None:
        plan = fox_packed_plan(cu_seqlens, N)
    else:
        _check_plan(plan, B, N, dev)
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    d_logit = torch.empty_like(gate_logit) if d_logit is None else d_logit
    _check(dq, "dq", (H, N, d), dt, dev)
    _check(dk, "dk", (Hkv, N, d), dt, dev)
    _check(dv, "dv", (Hkv, N, d), dt, dev)
    _check(d_logit, "d_logit", (H, N), gdt, dev)
    if d_log_f is not None:
        _check(d_log_f, "d_log_f", (H, N), torch.float32, dev)
    lib = load()
    if workspace is None:
        workspace = _workspace(lib.fox_attn_bwd_packed_workspace_bytes(H, N), dev)
    s = default_scale(d) if scale is None else float(scale)
    with _on_device(dev):
        st = lib.fox_attn_bwd_packed(
            _DT[dt], _ptr(q), _ptr(k), _ptr(v), _ptr(c), _ptr(o), _ptr(lse), _ptr(d_o), _DT[gdt],
            _ptr(gate_logit), _ptr(cu_seqlens), _ptr(plan), _ptr(dq), _ptr(dk), _ptr(dv),
            _ptr(d_logit), _ptr(d_log_f), _ptr(workspace),
            workspace.numel() * workspace.element_size(), B, H, Hkv, N, d, max_len, s,
            _raw_stream(dev.index))
    _raise(st, "fox_attn_bwd_packed")
    return dq, dk, dv, d_logit


def fox_packed_zero_behind(tensors: Sequence[torch.Tensor], cu_seqlens: torch.Tensor) -> None:
    """Zeros in the rows behind the last sequence of up to 8 packed tensors [heads, N, ...]."""
    B, dev = _check_cu(cu_seqlens, None), cu_seqlens.device
    N = tensors[0].shape[1]
    rows = (_RowsStruct * len(tensors))()
    for i, t in enumerate(tensors):
        _check(t, f"tensors[{i}]", (t.shape[0], N, *t.shape[2:]), None, dev)
        rows[i].x, rows[i].heads = _ptr(t), t.shape[0]
        rows[i].row_bytes = t[0, 0].numel() * t.element_size()
    with _on_device(dev):
        st = load().fox_packed_zero_behind(ctypes.addressof(rows), len(tensors),
                                           _ptr(cu_seqlens), B, N, _raw_stream(dev.index))
    _raise(st, "fox_packed_zero_behind")
