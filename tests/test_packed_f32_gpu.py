"""fp32 packed attention on batches large enough that a row block gets half the waves (more than
512 row blocks, of the queries, of the keys or of both), against 64 bits."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV, check, reference

pytestmark = pytest.mark.gpu

F32 = torch.float32


def _head_split(H, Hkv, N, d, max_len):
    """The groups that a key head's query heads are split into, from the workspace's size."""
    nbytes = fox.fox_attn_bwd_packed_workspace_bytes(F32, H, Hkv, N, d, max_len)
    return max(1, (nbytes // 4 - 3 * ((H * N + 3) // 4 * 4)) // (2 * Hkv * N * d))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,lens,splits,queries,keys", [
    (8, 8, [1500, 700, 33, 1], 1, True, True),
    (8, 4, [200] * 8 + [65], 1, True, False),   # the keys' blocks keep all the waves
    (8, 4, [100] * 20, 1, True, True),          # two heads, one after the other
    (8, 2, [100] * 20, 2, True, True),          # four, in two groups
    (4, 4, [300, 65], 1, False, False),
])
def test_row_blocks_of_fewer_waves(H, Hkv, d, lens, splits, queries, keys):
    print(H, Hkv, d, lens, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(61 + H + d)
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    N, max_len = cu[-1] + 3, max(lens)
    assert _head_split(H, Hkv, N, d, max_len) == splits
    items = N // 128 + len(lens)
    assert (4 * items * H > 512) == queries and (4 * items * Hkv * splits > 512) == keys
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    q, k, v, do = (r(n, N, d) for n in (H, Hkv, Hkv, H))
    logit = 5.0 * torch.rand((H, 1), generator=g, device=DEV) + r(H, N)
    for x in (q, k, v, do, logit):
        x[:, cu[-1]:] = float("nan")
    dcu = torch.tensor(cu, device=DEV, dtype=torch.int32)
    fill = lambda *s: torch.full(s, 7.0, device=DEV)  # noqa: E731
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, max_len=max_len, o=fill(H, N, d), lse=fill(H, N))
    outs = dict(dq=fill(H, N, d), dk=fill(Hkv, N, d), dv=fill(Hkv, N, d), d_logit=fill(H, N))
    dlf = fill(H, N)
    fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, max_len=max_len, d_log_f=dlf, **outs)
    ref = reference(q, k, v, logit, c, cu, fox.default_scale(d), do)
    for name, x in dict(o=o, lse=lse, d_log_f=dlf, **outs).items():
        check(name, x, ref[name], cu[-1])
        assert (x[:, cu[-1]:] == 7).all(), name  # left as they were
