"""ctypes binding of the paged key/value cache and the attention over it: argument
marshalling only, as in _lib.py."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from ._lib import (_DT, _call, _check, _check_int, _need, _ptr, _raise, _workspace,
                   _workspace_bytes, default_scale, load)

FOX_CACHE_BF16 = 0
FOX_CACHE_E4M3 = 1
_FORMATS = {torch.bfloat16: FOX_CACHE_BF16, torch.float8_e4m3fn: FOX_CACHE_E4M3}


class _CacheStruct(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int), ("n_pages", ctypes.c_int), ("page", ctypes.c_int),
                ("max_pages", ctypes.c_int), ("B", ctypes.c_int), ("H", ctypes.c_int),
                ("H_kv", ctypes.c_int), ("d", ctypes.c_int), ("k", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("c", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class PagedCache:
    """A paged key/value cache over the caller's tensors (fox_cache_t).

    k, v: [n_pages, H_kv, page, d], torch.float8_e4m3fn (quantised) or torch.bfloat16;
    k_exp, v_exp: [n_pages, H_kv, page] uint8, the scales 2^(exp - 127) of quantised rows;
    c: [n_pages, H, page] fp32, the running sum of log f; page_table: [B, max_pages] int32.
    page is 16, 32, 64, 128 or 256.  The tensors are kept and checked once, here; what they
    hold, the page table too, may change between calls.  Other tensors (a larger page table)
    need another PagedCache: the attributes are read-only, and the tensors must not be resized."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, c: torch.Tensor,
                 page_table: torch.Tensor, k_exp: Optional[torch.Tensor] = None,
                 v_exp: Optional[torch.Tensor] = None):
        if k.dtype not in _FORMATS:
            raise ValueError(f"unsupported cache dtype {k.dtype}")
        n_pages, Hkv, page, d = k.shape
        H, (B, max_pages) = c.shape[1], page_table.shape
        dev = k.device
        _check_int(max(n_pages, B, max_pages), "n_pages, B and max_pages")
        _check(k, "k", (n_pages, Hkv, page, d), k.dtype, None)
        _check(v, "v", (n_pages, Hkv, page, d), k.dtype, dev)
        _check(c, "c", (n_pages, H, page), torch.float32, dev)
        _check(page_table, "page_table", (B, max_pages), torch.int32, dev)
        f8 = k.dtype == torch.float8_e4m3fn
        for name, t in (("k_exp", k_exp), ("v_exp", v_exp)):
            if f8:
                _check(t, name, (n_pages, Hkv, page), torch.uint8, dev)
            elif t is not None:
                raise ValueError(f"{name} belongs to a float8_e4m3fn cache")
        struct = _CacheStruct(_FORMATS[k.dtype], n_pages, page, max_pages, B, H, Hkv, d, _ptr(k),
                              _ptr(v), _ptr(k_exp), _ptr(v_exp), _ptr(c), _ptr(page_table))
        self.__dict__.update(
            k=k, v=v, c=c, page_table=page_table, k_exp=k_exp, v_exp=v_exp, dtype=k.dtype,
            device=dev, n_pages=n_pages, page=page, max_pages=max_pages, B=B, H=H, H_kv=Hkv, d=d,
            _struct=struct, _ref=ctypes.addressof(struct))

    # the calls go by the struct's addresses, so what they stand for stays with them
    def __setattr__(self, name, value):
        raise AttributeError(f"PagedCache.{name} is read-only: make another PagedCache")

    def __delattr__(self, name):
        raise AttributeError(f"PagedCache.{name} is read-only")

    @classmethod
    def empty(cls, page_table: torch.Tensor, n_pages: int, heads: int, kv_heads: int, d: int,
              page: int = 64, dtype: torch.dtype = torch.float8_e4m3fn) -> "PagedCache":
        """A cache of n_pages pages on page_table's device, its slots uninitialised."""
        dev = page_table.device
        shape = (n_pages, kv_heads, page, d)
        exps = ([torch.empty(shape[:3], device=dev, dtype=torch.uint8) for _ in range(2)]
                if dtype == torch.float8_e4m3fn else (None, None))
        return cls(torch.empty(shape, device=dev, dtype=dtype),
                   torch.empty(shape, device=dev, dtype=dtype),
                   torch.empty((n_pages, heads, page), device=dev, dtype=torch.float32),
                   page_table, *exps)


def _check_lens(t: Optional[torch.Tensor], name: str, B: int, device):
    if t is not None:
        _need(t, name, (B,), torch.int32, device)


def fox_cache_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor,
                     gate_logit: torch.Tensor, seq_len: torch.Tensor,
                     parent: Optional[torch.Tensor] = None,
                     n_new: Optional[torch.Tensor] = None) -> None:
    """Writes n <= 64 new tokens of each sequence, a chain or (parent [B,n] int32) a tree,
    behind its seq_len [B] int32 cached ones.  k, v [B,H_kv,n,d] bf16 or fp32, gate_logit
    [B,H,n] fp32; n_new [B] int32: how many of the n a sequence has."""
    n, dt, dev = k.shape[2], k.dtype, cache.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    _need(k, "k", (cache.B, cache.H_kv, n, cache.d), dt, dev)
    _need(v, "v", (cache.B, cache.H_kv, n, cache.d), dt, dev)
    _need(gate_logit, "gate_logit", (cache.B, cache.H, n), torch.float32, dev)
    _need(seq_len, "seq_len", (cache.B,), torch.int32, dev)
    if parent is not None:
        _need(parent, "parent", (cache.B, n), torch.int32, dev)
    _check_lens(n_new, "n_new", cache.B, dev)
    st = _call(load().fox_cache_append, dev, cache._ref, _DT[dt], _ptr(k), _ptr(v),
               _ptr(gate_logit), _ptr(seq_len), _ptr(parent), _ptr(n_new), n)
    _raise(st, "fox_cache_append")


def fox_cache_append_packed(cache: PagedCache, k: torch.Tensor, v: torch.Tensor,
                            c: torch.Tensor, cu_seqlens: torch.Tensor,
                            seq_len: Optional[torch.Tensor] = None) -> None:
    """Writes whole prompts, packed (k, v [H_kv,N,d] bf16 or fp32, c [H,N] fp32 from
    fox_gate_prefix_packed, cu_seqlens [B+1] int32), behind the seq_len [B] int32 cached
    tokens of each sequence (None: none)."""
    N, dt, dev = k.shape[1], k.dtype, cache.device
    if dt not in _DT:
        raise ValueError(f"unsupported dtype {dt}")
    _need(k, "k", (cache.H_kv, N, cache.d), dt, dev)
    _need(v, "v", (cache.H_kv, N, cache.d), dt, dev)
    _need(c, "c", (cache.H, N), torch.float32, dev)
    _need(cu_seqlens, "cu_seqlens", (cache.B + 1,), torch.int32, dev)
    _check_lens(seq_len, "seq_len", cache.B, dev)
    st = _call(load().fox_cache_append_packed, dev, cache._ref, _DT[dt], _ptr(k), _ptr(v),
               _ptr(c), _ptr(cu_seqlens), _ptr(seq_len), N)
    _raise(st, "fox_cache_append_packed")


def fox_cache_keep(cache: PagedCache, seq_len: torch.Tensor, index: torch.Tensor,
                   n_keep: torch.Tensor) -> None:
    """Moves new token index[b, j] to place j behind seq_len[b], for j < n_keep[b]: the
    accepted path of a tree of drafts.  index [B,n] (n <= 64), n_keep [B] int32.  seq_len is
    left to the caller, who adds n_keep to it."""
    n, dev = index.shape[1], cache.device
    _check_int(n, "n")
    _need(seq_len, "seq_len", (cache.B,), torch.int32, dev)
    _need(index, "index", (cache.B, n), torch.int32, dev)
    _need(n_keep, "n_keep", (cache.B,), torch.int32, dev)
    st = _call(load().fox_cache_keep, dev, cache._ref, _ptr(seq_len), _ptr(index), _ptr(n_keep),
               n)
    _raise(st, "fox_cache_keep")


def fox_cache_read(cache: PagedCache, seq_len: torch.Tensor, T: int,
                   start: Optional[torch.Tensor] = None, dtype: torch.dtype = torch.bfloat16,
                   k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                   c: Optional[torch.Tensor] = None
                   ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Positions start[b] + t, t < T, below seq_len[b], as (k, v [B,H_kv,T,d], c [B,H,T]
    fp32).  Given k, v and c are filled; their rows without a token are left as they were.
    Otherwise such rows are zero."""
    dev = cache.device
    if k is not None:
        dtype = k.dtype
    if dtype not in _DT:
        raise ValueError(f"unsupported dtype {dtype}")
    shape = (cache.B, cache.H_kv, T, cache.d)
    given = [x is not None for x in (k, v, c)]
    if any(given) and not all(given):
        raise ValueError("k, v and c are given together or not at all")
    if k is None:
        k = torch.empty(shape, device=dev, dtype=dtype)
        v = torch.empty(shape, device=dev, dtype=dtype)
        c = torch.empty((cache.B, cache.H, T), device=dev, dtype=torch.float32)
    else:
        _need(k, "k", shape, dtype, dev)
        _need(v, "v", shape, dtype, dev)
        _need(c, "c", (cache.B, cache.H, T), torch.float32, dev)
    _need(seq_len, "seq_len", (cache.B,), torch.int32, dev)
    _check_lens(start, "start", cache.B, dev)
    st = _call(load().fox_cache_read, dev, cache._ref, _DT[dtype], _ptr(start), _ptr(seq_len),
               _ptr(k), _ptr(v), _ptr(c), T, not given[0])
    _raise(st, "fox_cache_read")
    return k, v, c


def fox_attn_cache_workspace_bytes(cache: PagedCache, n: int, max_len: int = 0) -> int:
    return int(load().fox_attn_cache_workspace_bytes(cache._ref, n, max_len))


def fox_attn_cache(q: torch.Tensor, cache: PagedCache, seq_len: torch.Tensor,
                   parent: Optional[torch.Tensor] = None, n_new: Optional[torch.Tensor] = None,
                   max_len: int = 0, scale: Optional[float] = None,
                   o: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None
                   ) -> Tuple[torch.Tensor, torch.Tensor]:
    """O [B,H,n,d] bf16 and LSE [B,H,n] fp32 of the n <= 64 newest tokens of each sequence
    (at places seq_len[b] .., written by fox_cache_append with the same parent and n_new)
    over the cache.  n = 1 is a decode step.  max_len: the most tokens a sequence has, new
    ones included (0: what the page table holds); it bounds the parts that the keys are split
    into, and the workspace."""
    B, H, n, d = q.shape
    dev = cache.device
    _need(q, "q", (cache.B, cache.H, n, cache.d), torch.bfloat16, dev)
    _need(seq_len, "seq_len", (cache.B,), torch.int32, dev)
    if parent is not None:
        _need(parent, "parent", (B, n), torch.int32, dev)
    _check_lens(n_new, "n_new", B, dev)
    if n_new is not None and (o is None or lse is None):
        # rows that a sequence does not have are not written
        o = torch.zeros_like(q) if o is None else o
        lse = torch.zeros((B, H, n), device=dev) if lse is None else lse
    if o is None:
        o = torch.empty_like(q)
    else:
        _need(o, "o", (B, H, n, d), torch.bfloat16, dev)
    if lse is None:
        lse = torch.empty((B, H, n), device=dev, dtype=torch.float32)
    else:
        _need(lse, "lse", (B, H, n), torch.float32, dev)
    lib = load()
    if workspace is None:
        nbytes = lib.fox_attn_cache_workspace_bytes(cache._ref, n, max_len)
        if nbytes:
            workspace = _workspace(nbytes, dev)
    else:
        nbytes = _workspace_bytes(workspace, dev)
    s = default_scale(d) if scale is None else float(scale)
    st = _call(lib.fox_attn_cache, dev, cache._ref, _ptr(q), _ptr(seq_len), _ptr(parent),
               _ptr(n_new), _ptr(o), _ptr(lse), _ptr(workspace), nbytes, n, max_len, s)
    _raise(st, "fox_attn_cache")
    return o, lse
