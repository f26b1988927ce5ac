"""Attention over packed sequences with grouped heads, forward and backward, against 64 bits;
its work list, prefix sums, refusals of nothing it should take, graphs and autograd."""
import pytest
import torch

import paper_2503_02130_amd as fox
from packed_reference import DEV, check, reference

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _ints(x):
    return torch.tensor(x, device=DEV, dtype=torch.int32)


def _inputs(H, Hkv, d, lens, dtype, gate_dtype, seed, behind=0, mean=(0.0, 5.0)):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    N = cu[-1] + behind
    r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    q, k, v, do = (r(n, N, d).to(dtype) for n in (H, Hkv, Hkv, H))
    m = mean[0] + (mean[1] - mean[0]) * torch.rand((H, 1), generator=g, device=DEV)
    logit = (m + r(H, N)).to(gate_dtype)
    for x in (q, k, v, do, logit):  # rows behind the last sequence may hold anything
        x[:, cu[-1]:] = float("nan")
    return q, k, v, do, logit, cu, torch.tensor(cu, device=DEV, dtype=torch.int32)


CASES = [
    # H, Hkv, d, lens, dtype, gate dtype, rows behind
    (2, 2, 64, [1], BF, F32, 0),
    (4, 2, 64, [1, 0, 2, 63, 64, 65], BF, BF, 7),
    (4, 1, 128, [127, 128, 129, 1], BF, F32, 0),
    (3, 3, 128, [300, 31, 33], BF, BF, 1),
    (8, 2, 64, [257, 0, 0, 640, 5], BF, F32, 130),
    (6, 2, 128, [500, 385], BF, BF, 0),
    (6, 1, 64, [32, 32, 96, 191, 70], BF, BF, 3),
    (2, 1, 64, [1, 2, 31, 32, 33, 0, 65], F32, F32, 5),
    (6, 2, 128, [129, 256, 40], F32, F32, 0),
    (4, 4, 64, [400, 1, 77], F32, BF, 66),
    (1, 1, 128, [700], F32, F32, 0),
]


@pytest.mark.parametrize("H,Hkv,d,lens,dtype,gate,behind", CASES)
def test_forward_and_backward(H, Hkv, d, lens, dtype, gate, behind):
    print(H, Hkv, d, lens, dtype, gate, behind, flush=True)
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, dtype, gate, 100 + H + d, behind)
    N, scale = q.shape[1], fox.default_scale(d)
    plan = fox.fox_packed_plan(dcu, N)
    fill = lambda *s, t=F32: torch.full(s, 7.0, device=DEV, dtype=t)  # noqa: E731
    c = fox.fox_gate_prefix_packed(logit, dcu, c=fill(H, N))
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, plan, o=fill(H, N, d, t=dtype),
                                     lse=fill(H, N))
    dlf = fill(H, N)
    outs = dict(dq=fill(H, N, d, t=dtype), dk=fill(Hkv, N, d, t=dtype),
                dv=fill(Hkv, N, d, t=dtype), d_logit=fill(H, N, t=gate))
    fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, plan, d_log_f=dlf, **outs)
    ref = reference(q, k, v, logit, c, cu, scale, do)
    got = dict(o=o, lse=lse, d_log_f=dlf, **outs)
    worst = {n: round(check(n, got[n], ref[n], cu[-1]), 2) for n in got}
    print(worst, flush=True)
    for n, x in dict(c=c, **got).items():
        assert (x[:, cu[-1]:] == 7).all(), n  # left as they were
    fox.fox_packed_zero_behind(list(got.values()), dcu)
    for n, x in got.items():
        assert not x[:, cu[-1]:].any(), n
        assert torch.isfinite(x.float()).all(), n


@pytest.mark.parametrize("lens,max_len", [([3001], 0), ([3001], 1), ([64, 1500, 900, 1], 1500),
                                          ([128] * 20 + [1000], 1000)])
@pytest.mark.parametrize("d", [64, 128])
def test_long_rows(lens, max_len, d):
    """Rows of many tiles, whatever max_len says; gates that forget at once and hardly."""
    H, Hkv = 4, 2
    for mean in ((-4.0, -4.0), (8.0, 8.0)):
        q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, BF, F32, 7 + d, 0, mean)
        c = fox.fox_gate_prefix_packed(logit, dcu)
        o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, max_len=max_len)
        dlf = torch.empty_like(c)
        g = fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, max_len=max_len,
                                    d_log_f=dlf)
        ref = reference(q, k, v, logit, c, cu, fox.default_scale(d), do)
        for n, x in dict(o=o, lse=lse, dq=g[0], dk=g[1], dv=g[2], d_log_f=dlf, d_logit=g[3]).items():
            check(n, x, ref[n], cu[-1])


@pytest.mark.parametrize("H,Hkv,d,lens", [(4, 2, 128, [700, 1, 130]), (3, 3, 64, [333, 0, 90])])
def test_what_rounding_took_from_o(H, Hkv, d, lens):
    """o_lo is o's rounding error: with it o is off by the bound less o's half step, plus o_lo's
    own.  The backward then starts from a Delta without that part, so dq moves towards the
    exact one."""
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, BF, F32, 77, 5)
    N, scale = q.shape[1], fox.default_scale(d)
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o_lo = torch.full_like(q, 7.0)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, o_lo=o_lo)
    alone = fox.fox_attn_fwd_packed(q, k, v, c, dcu)
    n = cu[-1]
    assert torch.equal(alone[0][:, :n], o[:, :n]) and torch.equal(alone[1][:, :n], lse[:, :n])
    assert (o_lo[:, n:] == 7).all()
    assert (o_lo[:, :n].abs() <= 2.0 ** -8 * o[:, :n].abs()).all()
    ref = reference(q, k, v, logit, c, cu, scale, do)
    value, bound = ref["o"]
    # o_lo's own rounding is half a step of a value of at most 2^-8 |o|
    tight = bound - 2.0 ** -8 * value.abs() + 2.0 ** -15 * value.abs()
    check("o + o_lo", o.double() + o_lo.double(), (value, tight), n)
    dq = {}
    for lo in (None, o_lo):
        got = fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, o_lo=lo)
        for name, x in zip(("dq", "dk", "dv", "d_logit"), got):
            check(name, x, ref[name], n)
        dq[lo is not None] = float((got[0][:, :n].double() - ref["dq"][0][:, :n]).norm())
    assert dq[True] < dq[False]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_prefix_sums(dtype):
    """Rounded once from 64 bits: at most half a step of the sum and the log sigmoids' own."""
    lens = [1, 0, 8191, 8192, 8193, 20000, 3]
    _, _, _, _, logit, cu, dcu = _inputs(3, 1, 64, lens, BF, dtype, 5, 4)
    c = fox.fox_gate_prefix_packed(logit, dcu)
    for b in range(len(lens)):
        x = logit[:, cu[b]:cu[b + 1]].double()
        lf = -torch.logaddexp(torch.zeros_like(x), -x)
        want = torch.cumsum(lf, -1)
        tol = 2.0 ** -24 * (want.abs() + 6 * torch.cumsum(lf.abs(), -1))
        assert ((c[:, cu[b]:cu[b + 1]].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens", [[1], [0, 0, 5], [3] * 300 + [5000], list(range(0, 700, 7))])
def test_both_in_one_launch(lens, dtype):
    """fox_packed_start's list and prefix sums are bit for bit those of the two calls."""
    _, _, _, _, logit, cu, dcu = _inputs(3, 1, 64, lens, BF, dtype, 6, 4)
    N = logit.shape[1]
    plan, c = fox.fox_packed_start(logit, dcu)
    assert torch.equal(plan, fox.fox_packed_plan(dcu, N))
    assert torch.equal(c[:, :cu[-1]], fox.fox_gate_prefix_packed(logit, dcu)[:, :cu[-1]])


def test_gates_of_every_size():
    """log sigmoid of the smallest to the largest finite logits, each a sequence of its own."""
    x = torch.tensor([0.0, 1e-30, -1e-30, 0.5, -0.5, 17.0, -17.0, 88.0, -88.0, 104.0, -104.0, 1e4, -1e4,
                      1e30, -1e30, 3.4e38, -3.4e38], device=DEV)
    logit = x.view(1, -1).contiguous()
    cu = torch.arange(x.numel() + 1, device=DEV, dtype=torch.int32)
    c = fox.fox_gate_prefix_packed(logit, cu)[0].double()
    want = -torch.logaddexp(torch.zeros_like(x.double()), -x.double())
    # the function is good to a few units of its last place (and exp flushes below 2^-126)
    assert ((c - want).abs() <= 6 * 2.0 ** -24 * want.abs() + 2.0 ** -126).all()


def _plan_reference(lens, N):
    items, cu = [], [0]
    for x in lens:
        cu.append(cu[-1] + x)
    top = max((x + 127) // 128 for x in lens)
    for m in range(top - 1, -1, -1):
        items += [(cu[s], x, m, s) for s, x in enumerate(lens) if (x + 127) // 128 > m]
    return items


@pytest.mark.parametrize("lens", [[1], [0, 0, 5], [128, 129, 0, 127, 1000], [3] * 300 + [5000],
                                  list(range(0, 700, 7))])
def test_plan(lens):
    N = sum(lens) + 10
    cu = [0]
    for x in lens:
        cu.append(cu[-1] + x)
    plan = fox.fox_packed_plan(torch.tensor(cu, device=DEV, dtype=torch.int32), N)
    got = [tuple(x) for x in plan.view(-1, 4).tolist()]
    want = _plan_reference(lens, N)
    assert got[:len(want)] == want
    assert all(x == (0, 0, 0, -1) for x in got[len(want):])


@pytest.mark.parametrize("cu", [[0, 300, 100, 350], [-5, 50, 10 ** 9, 7], [0, 400, 0, 400, 0, 400]])
def test_lengths_out_of_range_stay_inside(cu):
    """Nothing outside [0, N) enters the work list, whose places are enough."""
    N = 400
    plan = fox.fox_packed_plan(torch.tensor(cu, device=DEV, dtype=torch.int32), N)
    for start, length, block, seq in plan.view(-1, 4).tolist():
        assert 0 <= start and 0 <= length and start + length <= N
        assert length == 0 or (128 * block < length and 0 <= seq < len(cu) - 1)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_plan_of_another_batch_stays_inside(dtype):
    """A list of as many places made for more rows: its blocks lie outside and are skipped."""
    H, d, N = 2, 64, 130
    plan = fox.fox_packed_plan(_ints([0, 200, 255]), 255)
    q, k, v, o = (torch.full((H, N, d), 7.0, device=DEV, dtype=dtype) for _ in range(4))
    x = torch.full((H, N), 7.0, device=DEV)
    cu = _ints([0, 100, 130])
    lse = x.clone()
    fox.fox_attn_fwd_packed(q, k, v, x, cu, plan, o=o, lse=lse)
    assert (o == 7).all() and (lse == 7).all()
    grads = [torch.full_like(q, 7.0) for _ in range(3)]
    fox.fox_attn_bwd_packed(q, k, v, x, o, lse, q, x, cu, plan, dq=grads[0], dk=grads[1],
                            dv=grads[2])
    assert all((g == 7).all() for g in grads)


@pytest.mark.parametrize("d", [64, 128])
def test_one_sequence_agrees_with_the_dense_calls(d):
    """H = H_kv, one sequence: fox_attn_fwd's and fox_attn_bwd's results to their roundings."""
    H, L = 3, 777
    q, k, v, do, logit, cu, dcu = _inputs(H, H, d, [L], BF, F32, 9)
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu)
    g = fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu)
    one = lambda x: x[None].contiguous()  # noqa: E731
    c2 = fox.fox_gate_prefix(one(logit))
    o2, lse2 = fox.fox_attn_fwd(one(q), one(k), one(v), c2)
    g2 = fox.fox_attn_bwd(one(q), one(k), one(v), c2, o2, lse2, one(do))
    for a, b in zip((o, *g[:3]), (o2, *g2[:3])):
        # two roundings of each side's factors and one of its result
        assert (a.double() - b[0].double()).norm() <= 6 * 2.0 ** -8 * b.double().norm()
    assert (lse - lse2[0]).abs().max() <= 2.0 ** -7  # the dense sums add bf16 P


def test_same_bits_again_and_in_another_batch():
    lens = [200, 513, 64]
    q, k, v, do, logit, cu, dcu = _inputs(4, 2, 64, lens, BF, BF, 11)

    def run(q, k, v, do, logit, dcu):
        c = fox.fox_gate_prefix_packed(logit, dcu)
        o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, max_len=513)
        return (o, lse, *fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, max_len=513))

    a, b = (run(q, k, v, do, logit, dcu) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    # the second sequence first
    order = torch.cat([torch.arange(cu[i], cu[i + 1]) for i in (1, 0, 2)]).to(DEV)
    moved = [x[:, order].contiguous() for x in (q, k, v, do, logit)]
    e = run(*moved, torch.tensor([0, 513, 713, 777], device=DEV, dtype=torch.int32))
    assert all(torch.equal(x[:, order], y) for x, y in zip(a, e))


def test_autograd_and_differences():
    """Through autograd: the same gradients as the calls give, zeros behind; fp32 gradients
    against central differences of the 64-bit loss."""
    H, Hkv, d, lens = 4, 2, 64, [5, 0, 12]
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, F32, F32, 13, 3)
    for x in (q, k, v, do, logit):
        x[:, cu[-1]:] = 1.0
    leaves = [x.clone().requires_grad_() for x in (q, k, v, logit)]
    o = fox.forgetting_attention_packed(*leaves, dcu)
    assert not o[:, cu[-1]:].any()
    grads = torch.autograd.grad(o, leaves, do)
    for x in grads:
        assert not x[:, cu[-1]:].any()
    c = fox.fox_gate_prefix_packed(logit, dcu)
    o2, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu)
    direct = fox.fox_attn_bwd_packed(q, k, v, c, o2, lse, do, logit, dcu)
    for x, y in zip(grads, direct):
        assert torch.equal(x[:, :cu[-1]], y[:, :cu[-1]])

    def loss(t):
        q, k, v, logit = t
        total = 0.0
        for b in range(len(lens)):
            r = slice(cu[b], cu[b + 1])
            x = logit[:, r]
            cc = torch.cumsum(-torch.logaddexp(torch.zeros_like(x), -x), -1)
            kk, vv = (y[:, r].repeat_interleave(H // Hkv, 0) for y in (k, v))
            S = q[:, r] @ kk.transpose(1, 2) * fox.default_scale(d) + cc[:, :, None] - cc[:, None]
            S = S.masked_fill(torch.ones_like(S, dtype=torch.bool).triu(1), -float("inf"))
            total = total + (torch.softmax(S, -1) @ vv * do[:, r].double()).sum()
        return float(total)

    base = [x.double() for x in (q, k, v, logit)]
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    for i, x in enumerate(grads):
        direction = torch.randn(x.shape, generator=g, device=DEV, dtype=torch.float64)
        direction[:, cu[-1]:] = 0
        e = 1e-4
        up, down = ([y + s * e * direction if j == i else y for j, y in enumerate(base)]
                    for s in (1, -1))
        want = (loss(up) - loss(down)) / (2 * e)
        got = float((x.double() * direction).sum())
        # e^2 of the third derivative, and fp32 gradients
        assert abs(got - want) <= 1e-4 * float((x.double().abs() * direction.abs()).sum())


def test_layers_share_a_plan_and_gate_types():
    """bf16 gate logits through autograd, a shared plan, rows that are views of a larger
    tensor (made contiguous)."""
    H, Hkv, d, lens = 4, 2, 64, [100, 30]
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, BF, BF, 17)
    plan = fox.fox_packed_plan(dcu, 130)
    wide = torch.stack([q, q], 1)
    leaf = wide.requires_grad_()
    a = fox.forgetting_attention_packed(leaf[:, 0], k, v, logit, dcu, plan=plan, max_len=100)
    b = fox.forgetting_attention_packed(q, k, v, logit, dcu)
    assert torch.equal(a, b)
    g = torch.autograd.grad(a, leaf, do)[0]
    assert not g[:, 1].any() and g[:, 0].any()


def test_step_in_a_graph():
    """Forward and backward captured, replayed with new inputs, against the eager step."""
    H, Hkv, d, lens = 4, 2, 64, [200, 1, 400]
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, BF, BF, 19)
    N = cu[-1]

    def step(outs, ws):
        plan = fox.fox_packed_plan(dcu, N)
        c = fox.fox_gate_prefix_packed(logit, dcu)
        o, lse = fox.fox_attn_fwd_packed(q, k, v, c, dcu, plan, o=outs["o"], lse=outs["lse"])
        fox.fox_attn_bwd_packed(q, k, v, c, o, lse, do, logit, dcu, plan, dq=outs["dq"],
                                dk=outs["dk"], dv=outs["dv"], d_logit=outs["d_logit"], workspace=ws)
        fox.fox_packed_zero_behind(list(outs.values()), dcu)

    def buffers():
        e = torch.empty_like
        return (dict(o=e(q), lse=torch.empty((H, N), device=DEV), dq=e(q), dk=e(k), dv=e(v),
                     d_logit=e(logit)),
                torch.empty(fox.fox_attn_bwd_packed_workspace_bytes(BF, H, Hkv, N, d), device=DEV,
                            dtype=torch.uint8))

    (outs, ws), (want, ws2) = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(outs, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs, ws)
    for i in range(4):
        for x in (q, k, v, do, logit):
            x.copy_(torch.randn(x.shape, device=DEV))
        new = [0, 100 + 50 * i, 300, 601 - i]  # other lengths, rows behind
        dcu.copy_(torch.tensor(new, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        step(want, ws2)
        torch.cuda.synchronize()
        for n in outs:
            rows = new[-1] if n in ("o", "lse") else N
            assert torch.equal(outs[n][:, :rows], want[n][:, :rows]), (i, n)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_autograd_step_in_a_graph(dtype):
    """forgetting_attention_packed and its backward captured and replayed with new inputs, against
    the same step run eagerly between the replays."""
    H, Hkv, d, lens = 4, 2, 64, [150, 70]
    q, k, v, do, logit, cu, dcu = _inputs(H, Hkv, d, lens, dtype, F32, 23)
    static = [q, k, v, logit]

    def step():
        leaves = [x.detach().requires_grad_() for x in static]
        o = fox.forgetting_attention_packed(*leaves, dcu, max_len=150)
        return (o.detach(), *torch.autograd.grad(o, leaves, do))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        for x in (*static, do):
            x.copy_(torch.randn(x.shape, device=DEV))
        dcu.copy_(torch.tensor([0, 150 - 40 * i, 220 - i], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        for n, (a, b) in enumerate(zip(outs, want)):
            assert torch.equal(a, b), (i, n)
            assert not a[:, 220 - i:].any()
