"""The packed and the cache calls as a server uses them together: prompts of different lengths
through the packed attention and into a quantised cache, decode steps, a tree of drafts and its
accepted path, more decode steps; every output against 64 bits over what the cache stands for."""
import pytest
import torch

import paper_2503_02130_amd as fox
from cache_reference import DEV, F8, ancestors, attend, ints, quantise
from packed_reference import check, reference

pytestmark = pytest.mark.gpu


class Server:
    def __init__(self, fmt, H, Hkv, d, page, max_pages, prompts, seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.g, self.H, self.Hkv, self.d, self.B = g, H, Hkv, d, len(prompts)
        n_pages = self.B * max_pages
        table = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32).view(self.B, -1)
        self.f8 = fmt == "e4m3"
        self.cache = fox.PagedCache.empty(table.contiguous(), n_pages, H, Hkv, d, page,
                                          F8 if self.f8 else torch.bfloat16)
        self.seq = ints([0] * self.B)
        self.lens = [0] * self.B
        self.k, self.v, self.c = ([None] * self.B for _ in range(3))

    def randn(self, *s):
        return torch.randn(s, generator=self.g, device=DEV)

    def means(self, x):
        """What the cache stands for after rows x are written."""
        return quantise(x)[0] if self.f8 else x.double()

    def prefill(self, prompts):
        cu = [0]
        for x in prompts:
            cu.append(cu[-1] + x)
        N, dcu = cu[-1], ints(cu)
        q, k, v = (self.randn(n, N, self.d).bfloat16() for n in (self.H, self.Hkv, self.Hkv))
        logit = 3 + self.randn(self.H, N)
        plan = fox.fox_packed_plan(dcu, N)
        c = fox.fox_gate_prefix_packed(logit, dcu)
        o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, plan)
        fox.fox_cache_append_packed(self.cache, k, v, c, dcu, self.seq)
        self.seq += dcu[1:] - dcu[:-1]
        ref = reference(q, k, v, logit, c, cu, fox.default_scale(self.d))
        check("o", o, ref["o"], N)
        check("lse", lse, ref["lse"], N)
        ek, ev = self.means(k), self.means(v)
        for b in range(self.B):
            r = slice(cu[b], cu[b + 1])
            self.k[b], self.v[b], self.c[b] = ek[:, r], ev[:, r], c[:, r].double()
            self.lens[b] = prompts[b]

    def step(self, n, parents=None, accept=None):
        """n new tokens of each sequence; keeps accept[b] of them (all without)."""
        B = self.B
        q, k, v = (self.randn(B, h, n, self.d).bfloat16() for h in (self.H, self.Hkv, self.Hkv))
        logit = 3 + self.randn(B, self.H, n)
        par = None if parents is None else ints(parents)
        fox.fox_cache_append(self.cache, k, v, logit, self.seq, par)
        o, lse = fox.fox_attn_cache(q, self.cache, self.seq, par)
        end = self.seq + n
        # c as the cache has it (its own sums are tested elsewhere)
        c = fox.fox_cache_read(self.cache, end, n, start=self.seq)[2].double()
        if accept is not None:
            idx = ints([a + [0] * (n - len(a)) for a in accept])
            kept = ints([len(a) for a in accept])
            fox.fox_cache_keep(self.cache, self.seq, idx, kept)
            self.seq += kept
        else:
            self.seq += n
        ek, ev = self.means(k), self.means(v)
        for b in range(B):
            L = self.lens[b]
            kk, vv = torch.cat([self.k[b], ek[b]], 1), torch.cat([self.v[b], ev[b]], 1)
            cc = torch.cat([self.c[b], c[b]], 1)
            paths = ancestors(None if parents is None else parents[b], n)
            seen = [list(range(L)) + sorted(L + j for j in p) for p in paths]
            ro, rl, to, tl = attend(q[b], kk, vv, cc, L, seen, fox.default_scale(self.d))
            assert ((o[b].double() - ro).abs() <= to).all()
            assert ((lse[b].double() - rl).abs() <= tl).all()
            take = list(range(L)) + [L + j for j in (range(n) if accept is None else accept[b])]
            self.k[b], self.v[b], self.c[b] = kk[:, take], vv[:, take], cc[:, take]
            self.lens[b] = len(take)


@pytest.mark.parametrize("fmt,H,Hkv,d,page", [("e4m3", 8, 2, 128, 32), ("bf16", 6, 3, 64, 16)])
def test_serving(fmt, H, Hkv, d, page):
    prompts = [1, 150, 333]
    s = Server(fmt, H, Hkv, d, page, (333 + 64 + page - 1) // page, prompts, 7)
    s.prefill(prompts)
    for _ in range(3):
        s.step(1)
    tree = [[-1, 0, 0, 1, 2, 2, 5, 6], [-1, -1, 1, 1, 3, 0, 5, 4], [-1, 0, 1, 2, 3, 4, 5, 6]]
    s.step(8, tree, accept=[[0, 2, 5, 6], [1], [0, 1, 2, 3, 4, 5, 6, 7]])
    s.step(1)
    s.step(8, tree, accept=[[0], [1, 3, 4, 7], []])
    s.step(5)  # a chain
    # what is left in the cache
    T = max(s.lens)
    k, v, c = fox.fox_cache_read(s.cache, s.seq, T, dtype=torch.float32)
    for b in range(3):
        L = s.lens[b]
        assert int(s.seq[b]) == L
        assert torch.equal(k[b, :, :L].double(), s.k[b]) and torch.equal(v[b, :, :L].double(), s.v[b])
        assert torch.equal(c[b, :, :L].double(), s.c[b]) and not k[b, :, L:].any()


def test_a_prompt_in_parts():
    """A prompt written in two parts, and read back for the packed attention over all of it: the
    second part's rows come out as a whole prompt's do."""
    H, Hkv, d, parts = 4, 2, 64, (100, 61)
    s = Server("bf16", H, Hkv, d, 16, 11, [sum(parts)], 8)
    N = sum(parts)
    q, k, v = (s.randn(n, N, d).bfloat16() for n in (H, Hkv, Hkv))
    logit = 3 + s.randn(H, N)
    whole = ints([0, N])
    c = fox.fox_gate_prefix_packed(logit, whole)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, whole)
    at = 0
    for n in parts:
        cu, r = ints([0, n]), slice(at, at + n)
        cp = fox.fox_gate_prefix_packed(logit[:, r].contiguous(), cu)
        fox.fox_cache_append_packed(s.cache, k[:, r].contiguous(), v[:, r].contiguous(), cp, cu, s.seq)
        s.seq += n
        at += n
    rk, rv, rc = fox.fox_cache_read(s.cache, s.seq, N)
    assert torch.equal(rk[0], k) and torch.equal(rv[0], v)
    # the second part's c: one more fp32 addition
    assert ((rc[0] - c).abs() <= 2.0 ** -23 * c.abs()).all()
    o2, lse2 = fox.fox_attn_fwd_packed(q, rk[0], rv[0], rc[0].contiguous(), whole)
    assert torch.equal(o2[:, :parts[0]], o[:, :parts[0]])
    assert torch.equal(lse2[:, :parts[0]], lse[:, :parts[0]])
