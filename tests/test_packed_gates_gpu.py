"""The gates of packed sequences: logits that are not finite, logits of any size between others."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _cu(lens):
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    return cu, torch.tensor(cu, device=DEV, dtype=torch.int32)


def _randn(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


@pytest.mark.parametrize("gate", [BF, F32])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("at", [0, 133, 299])
def test_a_logit_that_is_not_a_number_is_seen(dtype, gate, at):
    """From its row on, c and o of its sequence and head are NaN, and so is its gradient; what
    does not see it keeps its bits."""
    H, Hkv, d, lens = 2, 1, 64, [140, 300, 77]
    cu, dcu = _cu(lens)
    N = cu[-1]
    q, k, v, do = (_randn(31 + i, n, N, d).to(dtype) for i, n in enumerate((H, Hkv, Hkv, H)))
    clean = (2.0 + _randn(36, H, N)).to(gate)
    bad = clean.clone()
    row = cu[1] + at
    bad[1, row] = float("nan")
    for both in (lambda x: fox.fox_packed_start(x, dcu)[1],
                 lambda x: fox.fox_gate_prefix_packed(x, dcu)):
        want, c = both(clean), both(bad)
        hit = torch.zeros_like(c, dtype=torch.bool)
        hit[1, row:cu[2]] = True
        assert torch.equal(torch.isnan(c), hit)
        assert torch.equal(c[~hit], want[~hit])

    def step(logit):
        leaves = [x.clone().requires_grad_() for x in (q, k, v, logit)]
        o = fox.forgetting_attention_packed(*leaves, dcu, max_len=max(lens))
        return (o.detach(), *torch.autograd.grad(o, leaves, do))

    want, got = step(clean), step(bad)
    assert torch.equal(torch.isnan(got[0]).all(-1), hit) and torch.equal(torch.isnan(got[0]).any(-1), hit)
    assert torch.equal(got[0][~hit], want[0][~hit])
    assert torch.isnan(got[4][1, row])
    others = torch.ones(N, dtype=torch.bool, device=DEV)
    others[cu[1]:cu[2]] = False
    for a, b in zip(want, got):
        assert torch.equal(a[:, others], b[:, others])


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
