"""A paged cache in plain 64-bit torch, for the tests of fox_cache_* and fox_attn_cache."""
import math

import torch

import paper_2503_02130_amd as fox

DEV = "cuda:0"
F8 = torch.float8_e4m3fn


def quantise(x):
    """Nearest e4m3 multiples of each row's scale, and the biased exponents, by the header's
    words: the least power of two from 2^-126 that brings the largest magnitude to 448."""
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, -126.0)
    for _ in range(260):
        e = torch.where(amax > 448.0 * torch.exp2(e), e + 1, e)
    y = x * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e), (e + 127).to(torch.uint8)[..., 0]


def log_f(x):
    x = x.double()
    return -torch.logaddexp(torch.zeros_like(x), -x)


class Cache:
    """Random pages, every slot filled with what must not be used, and the logical contents."""

    def __init__(self, B, H, Hkv, d, page, max_pages, fmt, seed, extra_pages=3):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.g, self.B, self.H, self.Hkv, self.d, self.page = g, B, H, Hkv, d, page
        n_pages = B * max_pages + extra_pages
        table = torch.randperm(n_pages, generator=g, device=DEV)[:B * max_pages]
        self.table = table.to(torch.int32).view(B, max_pages).contiguous()
        self.dev = fox.PagedCache.empty(self.table, n_pages, H, Hkv, d, page,
                                        F8 if fmt == "e4m3" else torch.bfloat16)
        for t in (self.dev.k, self.dev.v):
            if fmt == "e4m3":
                t.view(torch.uint8).fill_(0x7f)  # NaN
            else:
                t.fill_(float("nan"))
        self.dev.c.fill_(float("nan"))
        if fmt == "e4m3":
            self.dev.k_exp.fill_(255)
            self.dev.v_exp.fill_(255)
        self.f8 = fmt == "e4m3"

    def at(self, b, t):
        return int(self.table[b, t // self.page]), t % self.page

    def fill(self, lens, mean=3.0, std=1.0):
        """lens[b] tokens of random k, v and gates, written by plain indexing; keeps k, v
        [Hkv, T, d] and c [H, T] of each sequence in 64 bits."""
        self.k, self.v, self.c = [], [], []
        for b, T in enumerate(lens):
            raw = [torch.randn((self.Hkv, T, self.d), generator=self.g, device=DEV).bfloat16()
                   for _ in range(2)]
            gates = mean + std * torch.randn((self.H, T), generator=self.g, device=DEV)
            c = torch.cumsum(log_f(gates), -1).float()
            vals = []
            pages = self.table[b].long()[torch.arange(T, device=DEV) // self.page]
            slots = torch.arange(T, device=DEV) % self.page
            for name, x in (("k", raw[0]), ("v", raw[1])):
                if self.f8:
                    val, e = quantise(x)
                    code = (val * torch.exp2(127 - e.double())[..., None]).float().to(F8)
                    getattr(self.dev, name).view(torch.uint8)[pages, :, slots] = code.view(
                        torch.uint8).transpose(0, 1)
                    getattr(self.dev, name + "_exp")[pages, :, slots] = e.transpose(0, 1)
                else:
                    val = x.double()
                    getattr(self.dev, name)[pages, :, slots] = x.transpose(0, 1)
                vals.append(val)
            self.dev.c[pages, :, slots] = c.transpose(0, 1)
            self.k.append(vals[0])
            self.v.append(vals[1])
            self.c.append(c.double())

    def snapshot(self):
        t = [self.dev.k, self.dev.v, self.dev.c] + ([self.dev.k_exp, self.dev.v_exp] if self.f8 else [])
        return [x.view(torch.uint8).clone() for x in t]


def ints(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def ancestors(parent, n):
    """Lists of each token's ancestors and itself, from its parents (None: a chain)."""
    out = []
    for i in range(n):
        up = i - 1 if parent is None else int(parent[i])
        out.append([i] + (out[up] if 0 <= up < i else []))
    return out


def attend(q, k, v, c, base, seen, scale):
    """o [H,n,d], lse [H,n] in 64 bits, the bound of each o by the roundings (see below), and
    the bound of lse: k, v [Hkv,T,d], c [H,T], seen[i] the positions that token i attends to,
    base + i its own."""
    H, n, d = q.shape
    G = H // k.shape[0]
    T = k.shape[1]
    o = torch.zeros((H, n, d), device=DEV, dtype=torch.float64)
    lse = torch.full((H, n), -math.inf, device=DEV, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(o), torch.zeros_like(lse)
    for i in range(n):
        ix = torch.tensor(seen[i], device=DEV, dtype=torch.long)
        if not len(ix):
            continue
        for h in range(H):
            kk, vv = k[h // G][ix], v[h // G][ix]
            s = kk @ q[h, i].double() * scale + c[h, base + i] - c[h, ix]
            lse[h, i] = torch.logsumexp(s, 0)
            w = torch.softmax(s, 0)
            o[h, i] = w @ vv
            # A weight is rounded to bf16 once (2^-8 of itself) and so is o.  A score's fp32
            # error: d products summed, and a few roundings of the terms it is made of, all
            # relative to their magnitudes (2^-24 each); it enters a weight as a factor and
            # lse as itself, and the far keys' weights vanish, so magnitudes near the maximum
            # count.
            near = w > 2.0 ** -24
            dots = (kk[near].abs() @ q[h, i].double().abs()) * scale
            mag = dots.max() * d + 8 * (dots.max() + (c[h, base + i] - c[h, ix][near]).abs().max())
            es = 2.0 ** -24 * (mag + 64)
            A = w @ vv.abs()
            tol_o[h, i] = (2.0 ** -8 + 2 * es) * A + 2.0 ** -8 * o[h, i].abs() + 1e-30
            tol_l[h, i] = es + 2.0 ** -22 * lse[h, i].abs()
    return o, lse, tol_o, tol_l
