"""The bindings of the cache and the packed calls, on the host: what they hold on to and what
they refuse before any call."""
import pytest
import torch

import paper_2503_02130_amd as fox

ATTRIBUTES = ("k", "v", "c", "page_table", "k_exp", "v_exp", "dtype", "device", "n_pages", "page",
              "max_pages", "B", "H", "H_kv", "d")


@pytest.mark.parametrize("name", ATTRIBUTES)
def test_a_cache_is_set_once(name):
    """Its addresses and sizes are taken when it is made: another tensor behind the same name
    would leave the calls with memory that nobody holds."""
    cache = object.__new__(fox.PagedCache)
    with pytest.raises(AttributeError):
        setattr(cache, name, None)
    cache.__dict__[name] = 1
    with pytest.raises(AttributeError):
        setattr(cache, name, 2)
    with pytest.raises(AttributeError):
        delattr(cache, name)
    assert getattr(cache, name) == 1


WIDE = (1 << 32) + 128  # 128 as a 32-bit number


def test_sizes_beyond_32_bits_are_refused():
    """The C calls take ints, which ctypes cuts to 32 bits: such a call would do a part of the
    work, or go by other strides, and report success."""
    logit = torch.empty((1, WIDE), device="meta")
    cu = torch.zeros((2,), dtype=torch.int32)
    rows = torch.empty((1, WIDE, 2), device="meta")
    for call in (lambda: fox.fox_packed_plan(cu, WIDE), lambda: fox.fox_gate_prefix_packed(logit, cu),
                 lambda: fox.fox_packed_start(logit, cu),
                 lambda: fox.fox_packed_zero_behind([rows], cu)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
    k = torch.empty((8, 2, 64, 128), device="meta", dtype=torch.bfloat16)
    c, table = (torch.empty(s, device="meta", dtype=t) for s, t in (
        ((8, 4, 64), torch.float32), ((1, WIDE), torch.int32)))
    with pytest.raises(ValueError, match="2\\^31"):
        fox.PagedCache(k, k, c, table)
    cache = object.__new__(fox.PagedCache)
    cache.__dict__.update(B=1, device=torch.device("cuda", 0))
    with pytest.raises(ValueError, match="2\\^31"):
        fox.fox_cache_keep(cache, cu, torch.empty((1, WIDE), device="meta", dtype=torch.int32), cu)


@pytest.mark.parametrize("scale,good", [(0.0, False), (-0.0, False), (2.0 ** -65, False),
                                        (float("inf"), False), (float("nan"), False),
                                        (2.0 ** -64, True), (-0.125, True)])
def test_bf16_packed_attention_needs_a_scale_to_divide_by(scale, good):
    """Its kernels hold (c_i - c_j) / scale; fp32's do not.  A missing workspace or o_lo of an fp32
    o is refused after the scale, so nothing is launched."""
    p, lib = 0x10000, fox.load()
    value, unsupported, workspace, align = 7, 3, 5, 4

    def fwd(dtype, o=p, o_lo=None):
        return lib.fox_attn_fwd_packed(dtype, p, p, p, p, p, o, o_lo, p, 1, 4, 2, 100, 64, 0, scale,
                                       None)

    def bwd(dtype, o_lo=None):
        return lib.fox_attn_bwd_packed(dtype, *(p,) * 5, o_lo, p, p, 0, *(p,) * 7, None, 0, None, 0,
                                       1, 4, 2, 100, 64, 0, scale, None)

    assert fwd(1, o=p + 4) == (align if good else value)
    assert bwd(1) == (workspace if good else value)
    assert fwd(0, o_lo=p) == unsupported and bwd(0, o_lo=p) == unsupported
    assert fwd(0, o=p + 4) == align and bwd(0) == workspace
