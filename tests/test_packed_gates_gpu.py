"""The gates of packed sequences: logits of any size between others."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV

pytestmark = pytest.mark.gpu


def _cu(lens):
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    return cu, torch.tensor(cu, device=DEV, dtype=torch.int32)


def _randn(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


@pytest.mark.parametrize("value", [-1e10, -1e20, -3e38])
def test_a_large_logit_leaves_the_rows_before_it_alone(value):
    """A gate that forgets everything, at different places of the scan: c of the rows before it
    is as exact as without it."""
    L = 17000
    places = [1, 7, 8, 15, 511, 512, 519, 8191, 8192, 8199, 16383, 16390, 16999]
    logit = 2.0 + _randn(41, len(places), L)
    logit[torch.arange(len(places)), torch.tensor(places)] = value
    packed = logit.view(1, -1).contiguous()
    _, dcu = _cu([L] * len(places))
    c = fox.fox_gate_prefix_packed(packed, dcu).view(len(places), L).double()
    x = logit.double()
    lf = -torch.logaddexp(torch.zeros_like(x), -x)
    want = torch.cumsum(lf, -1)
    # the log sigmoids' own few units and the sum's one rounding
    tol = 2.0 ** -24 * (want.abs() + 6 * torch.cumsum(lf.abs(), -1))
    for i, p in enumerate(places):
        err = (c[i] - want[i]).abs()
        assert (err <= tol[i]).all(), (p, int((err > tol[i]).nonzero()[0]))
