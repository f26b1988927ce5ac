"""Attention over the cache: values that are not numbers."""
import pytest
import torch

import paper_2503_02130_amd as fox
from cache_reference import DEV, Cache, ancestors, attend, ints

pytestmark = pytest.mark.gpu


def _check(cache, lens, n_new, q, o, lse, scale, tiny=0.0):
    """Each row within cache_reference's bounds, tiny of the values' size more."""
    for b, L in enumerate(lens):
        m = n_new[b]
        if m == 0:
            continue
        seen = [list(range(L)) + [L + j for j in path] for path in ancestors(None, m)]
        ro, rl, to, tl = attend(q[b][:, :m], cache.k[b], cache.v[b], cache.c[b], L, seen, scale)
        err = (o[b][:, :m].double() - ro).abs()
        top = cache.v[b].abs().amax()
        assert (err <= to + tiny * top).all(), (b, float((err / (to + tiny * top)).max()))
        assert ((lse[b][:, :m].double() - rl).abs() <= tl).all(), b


@pytest.mark.parametrize("fmt,H,n,T", [("e4m3", 4, 1, 60), ("e4m3", 4, 2, 3000), ("bf16", 8, 5, 60),
                                       ("bf16", 8, 5, 3000)])
def test_what_is_not_a_number_is_seen(fmt, H, n, T):
    """A NaN in q or in c, in one piece and in several joined: o and lse of the rows that see it
    are NaN, the others' within their bounds."""
    lens, d = [T, 45], 64
    cache = Cache(2, H, 2, d, 64, (T + n + 63) // 64, fmt, 121)
    cache.fill([x + n for x in lens])
    q = torch.randn((2, H, n, d), device=DEV, generator=cache.g).to(torch.bfloat16)
    clean = fox.fox_attn_cache(q, cache.dev, ints(lens))
    bad = q.clone()
    bad[0, 1, n - 1, 3] = float("nan")
    hit = torch.zeros((2, H, n), dtype=torch.bool, device=DEV)
    hit[0, 1, n - 1] = True
    o, lse = fox.fox_attn_cache(bad, cache.dev, ints(lens))
    assert torch.equal(torch.isnan(o).all(-1), hit) and torch.equal(torch.isnan(lse), hit)
    o[hit], lse[hit] = clean[0][hit], clean[1][hit]
    _check(cache, lens, [n, n], q, o, lse, fox.default_scale(d))
    # the last cached token's c of head 2 of sequence 0: every new token attends to it
    p, s = cache.at(0, T - 1)
    cache.dev.c[p, 2, s] = float("nan")
    hit[:] = False
    hit[0, 2] = True
    o, lse = fox.fox_attn_cache(q, cache.dev, ints(lens))
    assert torch.equal(torch.isnan(o).all(-1), hit) and torch.equal(torch.isnan(lse), hit)
    o[hit], lse[hit] = clean[0][hit], clean[1][hit]
    _check(cache, lens, [n, n], q, o, lse, fox.default_scale(d))
