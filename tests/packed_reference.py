"""Causal attention with grouped heads of packed sequences in plain 64-bit torch, and bounds of
the kernels' errors from their roundings."""
import math

import torch

DEV = "cuda:0"
U = 2.0 ** -24  # fp32


def reference(q, k, v, logit, c32, cu, scale, d_o=None):
    """64-bit results and, beside each, the bound of the kernels' error:
    {name: (value, bound)} for o, lse and, with d_o, dq, dk, dv, d_log_f, d_logit.

    c32 is the prefix sum that the kernels were given.  With e_p the relative error of a weight
    (its rounding, if any, and the fp32 error of its exponent), a sum of w_j x_j is off
    by at most sum |w_j x_j| (e_p + its fp32 summation), and a stored value by half a step
    more.  Delta comes from the stored O, so it is off by the products of |dO| and O's bound;
    dS = P (dP - Delta) by e_p of itself and P times Delta's error (and for the products once
    more by its rounding); d(log f)_l = the sum of dS over queries from l on and keys before l,
    both halves of dc being sums of one matrix."""
    H, N, d = q.shape
    G = H // k.shape[0]
    bf = q.dtype == torch.bfloat16
    half = 2.0 ** -8 if bf else U
    names = ("o", "dq") + ("dk", "dv")
    out = {}
    for name in names:
        like = q if name in ("o", "dq") else k
        out[name] = [torch.zeros(like.shape, device=DEV, dtype=torch.float64) for _ in range(2)]
    for name in ("lse", "d_log_f", "d_logit"):
        out[name] = [torch.zeros((H, N), device=DEV, dtype=torch.float64) for _ in range(2)]
    for b in range(len(cu) - 1):
        lo, hi = cu[b], cu[b + 1]
        L = hi - lo
        if L == 0:
            continue
        future = torch.ones((L, L), dtype=torch.bool, device=DEV).triu(1)
        for h in range(H):
            g = h // G
            Q, K, V = q[h, lo:hi].double(), k[g, lo:hi].double(), v[g, lo:hi].double()
            c = c32[h, lo:hi].double()
            S = Q @ K.T * scale + c[:, None] - c[None, :]
            S.masked_fill_(future, -math.inf)
            lse = torch.logsumexp(S, -1)
            P = torch.exp(S - lse[:, None])
            o = P @ V
            # fp32 error of an exponent: d products, and terms as large as the score's parts
            dots = (Q.abs() @ K.abs().T) * scale
            near = P > U
            # The bf16 kernels hold c relative to the first row of a 128-row block (of the query
            # in the forward, of the key in the backward): a score's accumulator starts from
            # such a difference, is rounded at its size in each of the d / 16 steps, and the
            # rest of c_i - c_j enters afterwards.  Where a block forgets much, these parts are
            # far larger than the c_i - c_j of the keys that matter: d / 16 + 8 roundings of them.
            first = torch.arange(L, device=DEV) // 128 * 128
            spread = (c - c[first]).abs() if bf else torch.zeros_like(c)
            parts = spread[:, None] + spread[None, :] + (c[:, None] - c[None, :]).abs()
            mag = torch.where(near, (d / 16 + 8) * parts +
                              dots * (d + 8) + 8 * S.abs(), 0.0)
            es = U * (mag.amax(-1) + 64 + lse.abs())[:, None]  # by row
            sums = U * (L + 64)
            ep = (2.0 ** -8 if bf else 0.0) + 2 * es + sums
            A = P @ V.abs()
            bo = ep * A + half * o.abs()
            out["o"][0][h, lo:hi], out["o"][1][h, lo:hi] = o, bo
            out["lse"][0][h, lo:hi], out["lse"][1][h, lo:hi] = lse, es[:, 0] + sums + 2 * U * lse.abs()
            if d_o is None:
                continue
            dO = d_o[h, lo:hi].double()
            e2 = ep + 2 * es  # P again, from the stored LSE
            dP = dO @ V.T
            bdP = U * (d + 8) * (dO.abs() @ V.abs().T)
            delta = (dO * o).sum(-1, keepdim=True)
            bdelta = (dO.abs() * bo).sum(-1, keepdim=True) + U * (d + 8) * (dO * o).abs().sum(-1, keepdim=True)
            dS = P * (dP - delta)
            bS = e2 * dS.abs() + P * (1 + e2) * (bdP + bdelta)
            bSr = bS + (half if bf else 0.0) * (dS.abs() + bS) + sums * dS.abs()
            dv = P.T @ dO
            out["dv"][0][g, lo:hi] += dv
            out["dv"][1][g, lo:hi] += (e2 * P).T @ dO.abs() + sums * (P.T @ dO.abs())
            out["dq"][0][h, lo:hi] = dS @ K * scale
            out["dq"][1][h, lo:hi] = bSr @ K.abs() * scale + half * (dS @ K * scale).abs()
            out["dk"][0][g, lo:hi] += dS.T @ Q * scale
            out["dk"][1][g, lo:hi] += bSr.T @ Q.abs() * scale
            # queries from l on, keys before l
            suffix = lambda x: torch.flip(torch.cumsum(torch.flip(x, (0,)), 0), (0,))  # noqa: E731
            dlf = suffix(dS.sum(1) - dS.sum(0))
            cross = lambda m: torch.stack([m[l:, :l].sum() for l in range(L)])  # noqa: E731
            # the halves sum the same dS in different orders, each entry an fp32 away
            blf = cross(bS) + suffix(sums * (dS.abs().sum(1) + dS.abs().sum(0)))
            out["d_log_f"][0][h, lo:hi], out["d_log_f"][1][h, lo:hi] = dlf, blf
            sig = torch.sigmoid(-logit[h, lo:hi].double())
            hg = 2.0 ** -8 if logit.dtype == torch.bfloat16 else 8 * U
            out["d_logit"][0][h, lo:hi] = dlf * sig
            out["d_logit"][1][h, lo:hi] = blf * sig * 1.01 + hg * (dlf * sig).abs()
    for name in ("dk", "dv"):
        out[name][1] += half * out[name][0].abs()
    return out


def check(name, got, ref, rows):
    """Every element within its bound, in the first `rows` rows."""
    value, bound = (x[:, :rows] for x in ref)
    err = (got[:, :rows].double() - value).abs()
    worst = float((err / (bound + 1e-30)).max()) if err.numel() else 0.0
    assert torch.isfinite(got[:, :rows].double()).all(), name
    assert worst <= 1.0, f"{name}: {worst:.2f} of the bound"
    return worst
