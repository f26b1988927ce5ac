"""The gates of packed sequences: logits that are not finite, logits of any size between others,
and the gradient's reverse sums over rows of several segments."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV, U

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


def _gate_gradient(q, k, v, do, c, scale):
    """d(log f) of one sequence and head in 64 bits and the bound of its error in fp32, as in
    packed_reference.reference (the sum over the queries from l on and the keys before l, here
    from the difference of neighbouring l); then each row's own part of it, and its bound."""
    Q, K, V, dO, c = (x.double() for x in (q, k, v, do, c))
    L, d = Q.shape
    future = torch.ones((L, L), dtype=torch.bool, device=DEV).triu(1)
    S = (Q @ K.T).mul_(scale).add_(c[:, None] - c[None, :])
    S.masked_fill_(future, -torch.inf)
    lse = torch.logsumexp(S, -1)
    P = torch.exp(S - lse[:, None])
    dots = (Q.abs() @ K.abs().T).mul_(scale)
    mag = dots.mul_(d + 8).add_(S.abs().mul_(8)).add_((c[:, None] - c[None, :]).abs())
    mag = torch.where(P > U, mag, 0.0).amax(-1)
    del dots, S
    es = U * (mag + 64 + lse.abs())[:, None]
    sums = U * (L + 64)
    ep = 2 * es + sums
    o = P @ V
    bo = ep * (P @ V.abs()) + U * o.abs()
    e2 = ep + 2 * es
    dP = dO @ V.T
    bdP = (dO.abs() @ V.abs().T).mul_(U * (d + 8))
    delta = (dO * o).sum(-1, keepdim=True)
    bdelta = (dO.abs() * bo).sum(-1, keepdim=True) + U * (d + 8) * (dO * o).abs().sum(-1, keepdim=True)
    dS = dP.sub_(delta).mul_(P)
    bS = bdP.add_(bdelta).mul_(P).mul_(1 + e2).add_(e2 * dS.abs())
    suffix = lambda x: torch.flip(torch.cumsum(torch.flip(x, (0,)), 0), (0,))  # noqa: E731
    dlf = suffix(dS.sum(1) - dS.sum(0))
    low = bS.tril(-1)
    step = low.sum(0) - low.sum(1)  # leaving l: its keys' column enters, its queries' row goes
    cross = torch.cumsum(step, 0) - step
    blf = cross.clamp_min(0) + suffix(sums * (dS.abs().sum(1) + dS.abs().sum(0)))
    # one row's own part, dc_l = d(log f)_l - d(log f)_(l+1)
    dc = dS.sum(1) - dS.sum(0)
    bdc = bS.sum(1) + bS.sum(0) + sums * (dS.abs().sum(1) + dS.abs().sum(0))
    return dlf, blf, dc, bdc


@pytest.mark.parametrize("gate", [BF, F32])
@pytest.mark.parametrize("L", [8193, 17000])
def test_gradient_of_rows_of_several_segments(L, gate):
    """The reverse sums run over segments of 8192 rows from the sequence's end: row by row
    against 64 bits, and from row to row, where a sum that is lost at a border shows whole."""
    d, lens = 64, [5, L]
    cu, dcu = _cu(lens)
    N, scale = cu[-1], fox.default_scale(d)
    q, k, v, do = (_randn(51 + i, 1, N, d) for i in range(4))
    logit = (4.0 + _randn(56, 1, N)).to(gate)
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu)
    dlf = torch.empty_like(c)
    d_logit = fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, d_log_f=dlf)[3]
    r = slice(cu[1], cu[2])
    want, bound, dc, bdc = _gate_gradient(q[0, r], k[0, r], v[0, r], do[0, r], c[0, r], scale)
    got = dlf[0, r].double()
    assert ((got - want).abs() <= bound + 1e-30).all()
    # both sums are rounded once
    tol = bdc[:-1] + U * (got[:-1].abs() + got[1:].abs())
    assert ((got[:-1] - got[1:] - dc[:-1]).abs() <= tol).all()
    # (a sum lost behind a segment's first row moves the step there by itself: beyond the
    # tolerance, whatever the kernel's own error, if it is more than twice that)
    for row in range(L - 8192, 0, -8192):
        assert float(want[row].abs()) > 2 * float(tol[row - 1])
    # d(logit) is its product with sigmoid(-logit), rounded
    wx = got * torch.sigmoid(-logit[0, r].double())
    hx = 2.0 ** -8 if gate == BF else 8 * U
    assert ((d_logit[0, r].double() - wx).abs() <= hx * wx.abs() + 1e-30).all()
