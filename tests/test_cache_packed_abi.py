"""Refusals of the cache's and the packed calls on the host: nothing is launched, no device is
needed (the pointers are never followed)."""
import ctypes
import os

import pytest
import torch

import paper_2503_02130_amd as fox
from paper_2503_02130_amd._cache import _CacheStruct
from paper_2503_02130_amd._packed import _RowsStruct

P16 = 0x10000
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(fox.LIB_PATH):
        from paper_2503_02130_amd import build
        build.build()
    return fox.load()


def _cache(**changes):
    f = dict(format=1, n_pages=8, page=64, max_pages=4, B=2, H=4, H_kv=2, d=128, k=P16, v=P16,
             k_exp=P16, v_exp=P16, c=P16, page_table=P16)
    f.update(changes)
    return _CacheStruct(**f)


def _append(lib, cache, dtype=1, ptrs=(P16,) * 4, parent=None, n_new=None, n=4):
    return lib.fox_cache_append(ctypes.addressof(cache) if cache else None, dtype, *ptrs, parent,
                                n_new, n, None)


BAD_CACHES = [
    (dict(n_pages=0), SHAPE), (dict(page=48), SHAPE), (dict(page=8), SHAPE), (dict(page=512), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 25), SHAPE), (dict(B=0), SHAPE),
    (dict(H=5), SHAPE), (dict(H_kv=0), SHAPE), (dict(B=1 << 12, H=1 << 12), SHAPE),
    (dict(B=(1 << 16) + 1, H=1, H_kv=1), SHAPE),
    (dict(d=96), UNSUPPORTED), (dict(format=7), UNSUPPORTED), (dict(k=None), NULL),
    (dict(v=None), NULL), (dict(c=None), NULL), (dict(page_table=None), NULL),
    (dict(k_exp=None), NULL), (dict(v_exp=None), NULL), (dict(c=P16 + 4), ALIGN),
    (dict(k_exp=P16 + 8), ALIGN),
]


@pytest.mark.parametrize("changes,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(lib, changes, status):
    c = _cache(**changes)
    ref, p = ctypes.addressof(c), P16
    assert _append(lib, c) == status
    assert lib.fox_cache_append_packed(ref, 1, p, p, p, p, None, 100, None) == status
    assert lib.fox_cache_keep(ref, p, p, p, 4, None) == status
    assert lib.fox_cache_read(ref, 1, None, p, p, p, p, 10, 0, None) == status
    assert lib.fox_attn_cache(ref, p, p, None, None, p, p, p, 1 << 40, 1, 0, 0.1, None) == status
    assert lib.fox_attn_cache_workspace_bytes(ref, 1, 0) == 0


def test_a_bf16_cache_needs_no_scales(lib):
    c = _cache(format=0, k_exp=None, v_exp=None)
    assert lib.fox_attn_cache_workspace_bytes(ctypes.addressof(c), 1, 0) >= 0
    assert lib.fox_cache_keep(ctypes.addressof(c), None, P16, P16, 4, None) == NULL


def test_append_arguments(lib):
    c, p = _cache(), P16
    assert _append(lib, None) == NULL
    for i in range(4):
        assert _append(lib, c, ptrs=tuple(None if j == i else p for j in range(4))) == NULL
        assert _append(lib, c, ptrs=tuple(p + 2 if j == i else p for j in range(4))) == ALIGN
    assert _append(lib, c, n=0) == SHAPE and _append(lib, c, n=65) == SHAPE
    assert _append(lib, c, dtype=2) == UNSUPPORTED
    assert _append(lib, c, parent=p + 4) == ALIGN and _append(lib, c, n_new=p + 4) == ALIGN
    ref = ctypes.addressof(c)
    packed = lib.fox_cache_append_packed
    assert packed(ref, 1, p, p, None, p, None, 100, None) == NULL
    assert packed(ref, 1, p, p, p, p, None, 0, None) == SHAPE
    assert packed(ref, 1, p, p, p, p, None, 1 << 30, None) == SHAPE
    assert packed(ref, 9, p, p, p, p, None, 100, None) == UNSUPPORTED
    assert packed(ref, 1, p, p, p, p, p + 4, 100, None) == ALIGN


def test_keep_read_and_attention_arguments(lib):
    c, p = _cache(), P16
    ref = ctypes.addressof(c)
    assert lib.fox_cache_keep(ref, p, None, p, 4, None) == NULL
    assert lib.fox_cache_keep(ref, p, p, p, 65, None) == SHAPE
    assert lib.fox_cache_keep(ref, p, p + 4, p, 4, None) == ALIGN
    read = lib.fox_cache_read
    assert read(ref, 1, None, None, p, p, p, 4, 0, None) == NULL
    assert read(ref, 1, None, p, p, p, p, 0, 0, None) == SHAPE
    assert read(ref, 1, None, p, p, p, p, 1 << 30, 0, None) == SHAPE
    assert read(ref, 4, None, p, p, p, p, 4, 0, None) == UNSUPPORTED
    assert read(ref, 1, p + 4, p, p, p, p, 4, 0, None) == ALIGN
    attn = lib.fox_attn_cache
    ok = (ref, p, p, None, None, p, p, p, 1 << 40)
    for i in (1, 2, 5, 6):
        args = list(ok)
        args[i] = None
        assert attn(*args, 1, 0, 0.1, None) == NULL
        args[i] = p + 4
        assert attn(*args, 1, 0, 0.1, None) == ALIGN
    big = _cache(B=1 << 16, H=64, H_kv=8)  # 2^23 rows with two new tokens
    bref = ctypes.addressof(big)
    assert attn(bref, *ok[1:], 2, 0, 0.1, None) == SHAPE and _append(lib, big, n=2) == SHAPE
    assert lib.fox_attn_cache_workspace_bytes(bref, 2, 0) == 0
    assert read(bref, 1, None, p, p, p, p, 400, 0, None) == SHAPE  # 2^32 threads and more
    assert attn(*ok, 0, 0, 0.1, None) == SHAPE and attn(*ok, 65, 0, 0.1, None) == SHAPE
    # tables of 256 tokens leave nothing to split, and nothing to bring
    assert lib.fox_attn_cache_workspace_bytes(ref, 1, 0) == 0
    c.max_pages = 1 << 10
    need = lib.fox_attn_cache_workspace_bytes(ref, 1, 0)
    assert need > 0 and lib.fox_attn_cache_workspace_bytes(ref, 65, 0) == 0
    assert attn(ref, p, p, None, None, p, p, p, need - 1, 1, 0, 0.1, None) == WORKSPACE
    assert attn(ref, p, p, None, None, p, p, None, need, 1, 0, 0.1, None) == WORKSPACE
    assert lib.fox_attn_cache_workspace_bytes(ref, 1, 200) == 0


def test_packed_arguments(lib):
    p = P16
    assert lib.fox_packed_plan_bytes(0, 10) == 0 and lib.fox_packed_plan_bytes(3, 0) == 0
    assert lib.fox_packed_plan_bytes(3, 1000) == 16 * (7 + 3)
    assert lib.fox_packed_plan_bytes(2 ** 31 - 1, 2 ** 31 - 1) == 0
    plan = lib.fox_packed_plan
    assert plan(None, 1, 10, p, 1 << 20, None, 0, None) == NULL
    assert plan(p, 0, 10, p, 1 << 20, None, 0, None) == SHAPE
    assert plan(p, 1, 10, p + 8, 1 << 20, None, 0, None) == ALIGN
    assert plan(p, 1, 10, p, 15, None, 0, None) == WORKSPACE
    assert plan(p, 1, 10, p, 1 << 20, None, 1, None) == NULL
    assert plan(p, 1, 10, p, 1 << 20, None, 9, None) == SHAPE
    start = lib.fox_packed_start
    ok = (1, p, p, p, 1, 2, 10, p, 1 << 20, None, 0, None)
    for i, bad, status in ((1, None, NULL), (2, None, NULL), (3, None, NULL), (7, None, NULL),
                           (0, 3, UNSUPPORTED), (1, p + 2, ALIGN), (7, p + 8, ALIGN), (8, 15, WORKSPACE),
                           (5, 0, SHAPE), (6, 0, SHAPE), (10, 9, SHAPE), (10, 1, NULL)):
        assert start(*ok[:i], bad, *ok[i + 1:]) == status, i
    prefix = lib.fox_gate_prefix_packed
    assert prefix(1, p, None, p, 1, 1, 10, None) == NULL
    assert prefix(1, p, p, p, 1, 0, 10, None) == SHAPE
    assert prefix(1, p, p, p, 1, 1 << 20, 1 << 20, None) == SHAPE
    assert prefix(3, p, p, p, 1, 1, 10, None) == UNSUPPORTED
    assert prefix(1, p + 2, p, p, 1, 1, 10, None) == ALIGN

    def fwd(dtype=1, ptrs=(P16,) * 8, B=1, H=4, Hkv=2, N=100, d=64):
        return lib.fox_attn_fwd_packed(dtype, *ptrs, B, H, Hkv, N, d, 0, 0.1, None)

    for i in range(8):
        if i != 6:  # o_lo
            assert fwd(ptrs=tuple(None if j == i else p for j in range(8))) == NULL
        assert fwd(ptrs=tuple(p + 4 if j == i else p for j in range(8))) == ALIGN
    assert fwd(dtype=0) == UNSUPPORTED  # o_lo of an fp32 o
    assert fwd(H=3) == SHAPE and fwd(N=0) == SHAPE and fwd(B=-1) == SHAPE
    assert fwd(N=1 << 23) == SHAPE  # a head's rows pass 2^31 bytes
    assert fwd(dtype=2) == UNSUPPORTED and fwd(d=32) == UNSUPPORTED
    need = lib.fox_attn_bwd_packed_workspace_bytes
    assert need(1, 4, 3, 100, 64, 0) == 0 and need(1, 4, 2, 100, 80, 0) == 0
    assert need(1, 4, 4, 100, 64, 0) >= 3 * 4 * 100 * 4

    def bwd(dtype=1, gate=0, skip=None, off=None, ws=1 << 40, ws_ptr=P16, d=64):
        a = [p] * 8
        b = [p] * 7
        if skip is not None:
            (a if skip < 8 else b)[skip % 8] = None
        if off is not None:
            (a if off < 8 else b)[off % 8] = p + 4
        return lib.fox_attn_bwd_packed(dtype, *a, gate, *b, None, 0, ws_ptr, ws, 1, 4, 2, 100, d, 0,
                                       0.1, None)

    for i in range(15):
        assert (i == 5 or bwd(skip=i) == NULL) and bwd(off=i) == ALIGN
    assert bwd(dtype=0) == UNSUPPORTED  # o_lo of an fp32 o
    assert bwd(gate=5) == UNSUPPORTED and bwd(d=256) == UNSUPPORTED
    assert bwd(ws=need(1, 4, 2, 100, 64, 0) - 1) == WORKSPACE and bwd(ws_ptr=None) == WORKSPACE
    rows = (_RowsStruct * 2)((p, 2, 64), (p, 2, 63))
    zero = lib.fox_packed_zero_behind
    assert zero(ctypes.addressof(rows), 2, p, 1, 10, None) == SHAPE  # an odd row
    rows[1].row_bytes, rows[1].x = 64, p + 4
    assert zero(ctypes.addressof(rows), 2, p, 1, 10, None) == ALIGN
    assert zero(ctypes.addressof(rows), 0, p, 1, 10, None) == SHAPE
    assert zero(ctypes.addressof(rows), 1, None, 1, 10, None) == NULL


def test_bindings_refuse_host_tensors_and_wrong_shapes():
    f8 = torch.float8_e4m3fn
    table = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(ValueError):
        fox.PagedCache.empty(table, 8, 4, 2, 128)
    with pytest.raises(ValueError):  # a type that no cache has
        fox.PagedCache.empty(table, 8, 4, 2, 128, dtype=torch.float16)
    k = torch.zeros((8, 2, 64, 128), dtype=f8)
    with pytest.raises((ValueError, TypeError)):  # no scales
        fox.PagedCache(k, k, torch.zeros((8, 4, 64)), table)
    cu = torch.tensor([0, 3], dtype=torch.int32)
    for call in (lambda: fox.fox_packed_plan(cu, 3),
                 lambda: fox.fox_packed_plan(cu[:1], 3),
                 lambda: fox.fox_gate_prefix_packed(torch.zeros((2, 3)), cu),
                 lambda: fox.fox_packed_start(torch.zeros((2, 3)), cu),
                 lambda: fox.fox_gate_prefix_packed(torch.zeros((2, 3), dtype=torch.float16), cu),
                 lambda: fox.fox_attn_fwd_packed(*(torch.zeros((2, 3, 64)),) * 3,
                                                 torch.zeros((2, 3)), cu),
                 lambda: fox.forgetting_attention_packed(*(torch.zeros((2, 3, 64)),) * 3,
                                                         torch.zeros((2, 3)), cu)):
        with pytest.raises(ValueError):
            call()
