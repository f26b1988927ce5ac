"""Attention over the cache: batches of more sequences than a wave has lanes, and values of any
size."""
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


@pytest.mark.parametrize("fmt,H,Hkv,n", [("e4m3", 4, 2, 2), ("bf16", 8, 2, 5)])
@pytest.mark.parametrize("B", [64, 65, 130])
def test_many_sequences(B, fmt, H, Hkv, n):
    """Both kernels, lengths of zero and long ones that are split and joined on both sides of
    every 64th sequence, some without new tokens there."""
    print(B, fmt, H, Hkv, n, flush=True)
    d, page = 64, 16
    lens = [(i * 37) % 71 for i in range(B)]
    n_new = [n - (i % 3 == 1) for i in range(B)]
    for b, L in ((0, 2100), (3, 0), (62, 1500), (63, 3000), (64, 2500), (65, 0), (66, 700),
                 (127, 1300), (128, 2000), (129, 2777)):
        if b < B:
            lens[b] = L
    for b in (5, 61, 65, 67, 126, 128):
        if b < B:
            n_new[b] = 0
    cache = Cache(B, H, Hkv, d, page, (3000 + n + page - 1) // page, fmt, 101)
    cache.fill([a + b for a, b in zip(lens, n_new)])
    q = torch.randn((B, H, n, d), device=DEV, generator=cache.g).to(torch.bfloat16)
    assert fox.fox_attn_cache_workspace_bytes(cache.dev, n) > 0  # some are split
    o, lse = torch.full_like(q, 7.0), torch.full((B, H, n), 7.0, device=DEV)
    fox.fox_attn_cache(q, cache.dev, ints(lens), n_new=ints(n_new), o=o, lse=lse)
    _check(cache, lens, n_new, q, o, lse, fox.default_scale(d))
    for b in range(B):  # rows that a sequence does not have
        assert (o[b][:, n_new[b]:] == 7).all() and (lse[b][:, n_new[b]:] == 7).all()
    # lengths in another order, so that the long ones lie elsewhere
    order = torch.randperm(B, generator=torch.Generator().manual_seed(3)).tolist()
    moved = fox.PagedCache(cache.dev.k, cache.dev.v, cache.dev.c, cache.table[order].contiguous(),
                           cache.dev.k_exp, cache.dev.v_exp)
    for name in ("k", "v", "c"):
        setattr(cache, name, [getattr(cache, name)[i] for i in order])
    lens, n_new = [lens[i] for i in order], [n_new[i] for i in order]
    o, lse = fox.fox_attn_cache(q[order].contiguous(), moved, ints(lens), n_new=ints(n_new))
    _check(cache, lens, n_new, q[order], o, lse, fox.default_scale(d))


@pytest.mark.parametrize("d,H,n", [(64, 4, 1), (128, 4, 1), (128, 32, 3)])
def test_values_of_every_size(d, H, n):
    """e4m3 rows of V between 2^-90 and 2^100: the scale multiplies a weight, which is rounded to
    bf16 then, where those below 2^-126 may vanish: 2^-29 of the largest at 2^-90."""
    sizes = [-90, -60, -17, 0, 40, 97]
    lens = [700] * len(sizes)
    cache = Cache(len(sizes), H, 1, d, 64, 12, "e4m3", 111)
    cache.fill([x + n for x in lens])
    for b, e in enumerate(sizes):
        pages = cache.table[b].long()
        cache.dev.v_exp[pages] = (cache.dev.v_exp[pages].int() + e).clamp(1, 254).to(torch.uint8)
        cache.v[b] = cache.v[b] * 2.0 ** e
    q = torch.randn((len(sizes), H, n, d), device=DEV, generator=cache.g).to(torch.bfloat16)
    o, lse = fox.fox_attn_cache(q, cache.dev, ints(lens))
    # at most 703 weights of them
    _check(cache, lens, [n] * len(sizes), q, o, lse, fox.default_scale(d), 703 * 2.0 ** -29)


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
