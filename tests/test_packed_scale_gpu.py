"""Packed attention with a negative scale: that of the negated queries, within the bounds of
packed_reference."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV, check, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[100, 1, 70], [1111], [64, 128]])
def test_negative_scale(dtype, d, lens):
    H, Hkv, N = 4, 2, sum(lens)
    g = torch.Generator(device=DEV)
    g.manual_seed(71)
    q, k, v, do = (torch.randn((n, N, d), generator=g, device=DEV).to(dtype) for n in (H, Hkv, Hkv, H))
    logit = 2.0 + torch.randn((H, N), generator=g, device=DEV)
    cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
    dcu, s = torch.tensor(cu, device=DEV, dtype=torch.int32), fox.default_scale(d)
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, scale=-s)
    dq, dk, dv, dx = fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, scale=-s)
    ref = reference(-q, k, v, logit, c, cu, s, do)
    for name, x in dict(o=o, lse=lse, dq=-dq, dk=dk, dv=dv, d_logit=dx).items():
        check(name, x, ref[name], N)
