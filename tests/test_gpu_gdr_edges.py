"""Calls of the delta layer and the head norm at the far ends: offsets beyond 32 bits, more sequences than a wide block ranks, two streams and two
graphs at once, one fully rotated head per row.  Each is compared with the same work done in a plainer call, bit for bit, except where
test_gpu_gdr.py and test_gpu_qk_norm.py have a bound against the fp64 statement.
"""

import numpy as np
import pytest
import torch

from oracle import gdr
from test_gpu_gdr import Problem, check_states, i32, is_chunked
from test_gpu_qk_norm import DT, LAYOUT, check

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md


def same(a, b):
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


@pytest.mark.parametrize("hv,longest", [(2, 70000), (40, 70000), (2, 32)])
def test_rows_whose_offsets_pass_32_bits(hv, longest):
    """Rows of 32768 values: the last start 2.3e9 values in.  Narrow chain, wide chain, token by token."""
    T, ld, d = 70000, 32768, 128
    big = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    unit = lambda: torch.nn.functional.normalize(torch.randn((T, d), generator=g, device="cuda"), dim=-1).bfloat16()
    src = [unit(), unit(), torch.randn((T, hv * d), generator=g, device="cuda").bfloat16(), torch.randn((T, hv * d), generator=g, device="cuda").bfloat16(),
           torch.randn((T, hv), generator=g, device="cuda").bfloat16(), torch.randn((T, hv), generator=g, device="cuda").bfloat16()]
    far, at = [], ld
    for t in src:
        at -= -(-t.shape[1] // 8) * 8
        far.append(big[:, at:at + t.shape[1]])
        far[-1].copy_(t)
    layer = md.GdrLayer(-torch.linspace(0.5, 16, hv, device="cuda"), torch.full((hv,), -4.58, device="cuda"), torch.ones(d, device="cuda"), 1)
    n = -(-T // longest)
    cu = i32(np.minimum(np.arange(n + 1) * longest, T))
    outs, states = [], []
    for dev, out in ((src, torch.empty((T, hv * d), dtype=torch.bfloat16, device="cuda")), (far, big[:, :hv * d])):
        cache = md.StateCache(1, n, hv * d, d_state=d)
        need = md.mdraft_gdr_prefill_workspace_bytes(layer, T, n, longest)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        md.mdraft_gdr_prefill(layer, cache, 0, *dev, out, cu, longest, None, i32(np.arange(n)), ws)
        torch.cuda.synchronize()
        outs.append(out)
        states.append(cache.ssm)
    assert same(*outs) and torch.equal(*states)
    assert bool(outs[0].isfinite().all())


def test_slots_whose_offsets_pass_32_bits():
    hk, hv, slots = 1, 2, 70000   # of 32768 values each
    big = md.StateCache(1, slots, hv * 128, d_state=128, zero=False, conv_channels=8)
    for rows, heads in ((8, hv), (70, hv)):
        p = Problem(rows, hk, heads, seed=5 + rows)
        h0 = torch.from_numpy(p.states(1)[0]).cuda()
        small = p.cache(2)
        got = []
        for cache, a, b in ((small, 0, 1), (big, slots - 1, slots - 2)):
            cache.ssm[0, a] = h0
            out = p.out()
            md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, rows, i32([a]), i32([b]), p.workspace(1, rows))
            got.append((out, cache.ssm[0, b].clone()))
        assert same(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    p = Problem(2, hk, hv, seed=9)
    small = p.cache(3)
    got = []
    for cache, at in ((small, [0, 1, 2]), (big, [slots - 1, slots - 2, slots - 3])):
        cache.ssm[0, at[0]] = h0
        out = p.out()
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, out, i32(at[:2]), i32(at[1:]), [0, 1, 2])
        if cache is big:
            md.mdraft_state_commit(big, i32([at[2]]), i32([0]))
            assert torch.equal(big.ssm[0, 0], big.ssm[0, at[2]])
        got.append((out, cache.ssm[0, at[2]].clone()))
    assert same(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_wide_slots_in_the_wide_chain():
    """40 heads: the pool's last slot starts 2.6e9 values in."""
    p = Problem(100, 2, 40, seed=8)
    slots = 4000
    big = md.StateCache(1, slots, 40 * 128, d_state=128, zero=False, conv_channels=8)
    h0 = torch.from_numpy(p.states(1)[0]).cuda()
    small = p.cache(2)
    got = []
    for cache, a, b in ((small, 0, 1), (big, slots - 1, slots - 2)):
        cache.ssm[0, a] = h0
        out = p.out()
        md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, 100, i32([a]), i32([b]), p.workspace(1, 100))
        got.append((out, cache.ssm[0, b].clone()))
    assert same(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


def test_more_sequences_than_are_taken_by_length():
    """600 sequences of 1 to 70 tokens; the statement for a few of them, and the rest against calls of 100 sequences."""
    g = np.random.default_rng(4)
    lens = g.integers(1, 71, 600)
    p = Problem(int(lens.sum()), 1, 1, 64, 64, seed=6)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cache, out, status = p.cache(600), p.out(), torch.zeros(1, dtype=torch.int32, device="cuda")
    assert is_chunked(p, list(lens))
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32(cu), 70, None, i32(np.arange(600)), p.workspace(600, 70), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    parts, c2 = p.out(), p.cache(600)
    for a in range(0, 600, 100):
        rows = slice(int(cu[a]), int(cu[a + 100]))
        dev = [None if t is None else t[rows] for t in p.dev]
        ws = torch.empty(md.mdraft_gdr_prefill_workspace_bytes(p.layer, rows.stop - rows.start, 100, 70), dtype=torch.uint8, device="cuda")
        md.mdraft_gdr_prefill(p.layer, c2, 0, *dev, parts[rows], i32(cu[a:a + 101] - cu[a]), 70, None, i32(np.arange(a, a + 100)), ws)
    torch.cuda.synchronize()
    assert same(out, parts) and torch.equal(cache.ssm, c2.ssm)
    for s in (0, 17, 599):
        args = p.args()
        for key in ("q", "k", "v", "z", "dt", "beta"):
            args[key] = args[key][cu[s]:cu[s + 1]]
        want = gdr.encode(**args, cu=np.array([0, lens[s]]))[1]
        check_states(cache.ssm[0, s], np.asarray(want).reshape(-1, 64))


def test_two_streams_at_once():
    ps = [Problem(n, 2, hv, seed=n) for n, hv in ((900, 4), (700, 40), (20, 4))]
    alone, calls = [], []
    for p in ps:
        cache, out = p.cache(1), p.out()
        md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, p.rows, None, i32([0]), p.workspace(1, p.rows))
        alone.append((out, cache.ssm))
        calls.append((p, p.cache(1), p.out(), i32([0]), p.workspace(1, p.rows), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for p, cache, out, final, ws, s in calls:
            md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, p.rows, None, final, ws, stream=s)
    torch.cuda.synchronize()
    for (o, h), (p, cache, out, *_) in zip(alone, calls):
        assert same(o, out) and torch.equal(h, cache.ssm)


def test_two_graphs_that_share_a_workspace():
    ps = [Problem(n, 2, hv, seed=n) for n, hv in ((300, 4), (200, 40))]
    ws = torch.empty(max(md.mdraft_gdr_prefill_workspace_bytes(p.layer, p.rows, 1, p.rows) for p in ps), dtype=torch.uint8, device="cuda")
    runs = []
    for p in ps:
        cache, out, final = p.cache(1), p.out(), i32([0])
        f = lambda p=p, cache=cache, out=out, final=final: md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, p.rows, None, final, ws)
        f()
        torch.cuda.synchronize()
        want = (out.clone(), cache.ssm.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f()
        out.fill_(0)
        runs.append((graph, out, cache, want))
    for _ in range(4):
        for graph, *_ in runs:
            graph.replay()
    torch.cuda.synchronize()
    for _, out, cache, (o, h) in runs:
        assert same(out, o) and torch.equal(cache.ssm, h)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("heads,d", [(1, 64), (1, 128), (1, 256), (2, 32)])
def test_wholly_rotated_heads_in_many_rows(act, layout, heads, d):
    """One or two heads to a row and all of their values turn: a pass's turns take as much shared memory as they ever do."""
    t = DT[act]
    x = torch.randn((40000, heads * d), device="cuda").to(t)
    freqs = torch.linspace(1, 0.001, d // 2, device="cuda")
    pos = torch.arange(40000, dtype=torch.int32, device="cuda") * 7
    spec = md.QkNorm(d, heads, 0, t, md.MDRAFT_NORM_RMS, rot_dim=d, rot_layout=LAYOUT[layout], freqs=freqs)
    o = torch.empty_like(x)
    md.mdraft_qk_norm(spec, x, None, o, None, pos)
    want = gdr.head_norm(x.double().cpu().numpy(), d, "rms", None, 1e-6, pos.cpu().numpy(), freqs.double().cpu().numpy(), layout)
    check(o, want, d, d, layout, act)
    spec = md.QkNorm(d, 0, heads, t, md.MDRAFT_NORM_RMS, rot_dim=d, rot_layout=LAYOUT[layout], freqs=freqs)
    for a in range(0, 40000, 1000):
        part = torch.empty_like(x[:1000])
        md.mdraft_qk_norm(spec, None, x[a:a + 1000], None, part, pos[a:a + 1000])
        assert torch.equal(part, o[a:a + 1000])


def test_norm_rows_whose_offsets_pass_32_bits():
    T, ld = 70000, 32768
    big = torch.empty((T, ld), dtype=torch.bfloat16, device="cuda")
    x = torch.randn((T, 384), device="cuda").bfloat16()
    big[:, -384:] = x
    freqs = torch.linspace(1, 0.001, 32, device="cuda")
    spec = md.QkNorm(64, 4, 2, rot_dim=64, freqs=freqs)
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    o = torch.empty_like(x)
    md.mdraft_qk_norm(spec, x[:, :256], x[:, 256:], o[:, :256], o[:, 256:], pos)
    md.mdraft_qk_norm(spec, big[:, -384:-128], big[:, -128:], big[:, -384:-128], big[:, -128:], pos)
    torch.cuda.synchronize()
    assert same(o, big[:, -384:])


@pytest.mark.parametrize("hv", [2, 40])
def test_a_nan_reaches_nothing_ahead_of_its_64_tokens(hv):
    """What the encode says of a NaN among a sequence's own values: it stays with the sequence and behind the start of its 64 tokens."""
    p = Problem(400, 2, hv, seed=70)
    cu, final = i32([0, 200, 400]), i32([0, 1])
    res = []
    for poison in (False, True):
        if poison:
            p.dev[2][100].fill_(float("nan"))
        out, cache = p.out(), p.cache(2)
        md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, cu, 200, None, final, p.workspace(2, 200))
        torch.cuda.synchronize()
        res.append((out, cache.ssm[0].clone()))
    (a, sa), (b, sb) = res
    assert same(a[:64], b[:64]) and same(a[200:], b[200:]) and torch.equal(sa[1], sb[1])
    assert bool(b[100:200].isnan().all()) and bool(sb[0].isnan().any())


@pytest.mark.parametrize("hq,hk,apart", [(40, 1, "k"), (1, 40, "q"), (33, 0, "q"), (0, 33, "k")])
def test_norm_of_queries_and_keys_with_strides_far_apart(hq, hk, apart):
    """More heads than a block takes, so that its last groups have none: they keep to one operand's rows and strides (read with the other's, the rows of the
    narrow one would end long before)."""
    rows, d = 5, 128
    wide = lambda x: torch.zeros((rows, 1 << 20), dtype=torch.bfloat16, device="cuda").index_copy_(1, torch.arange(x.shape[1], device="cuda"), x)[:, :x.shape[1]]
    q, k = (torch.randn((rows, h * d), device="cuda").bfloat16() if h else None for h in (hq, hk))
    spec = md.QkNorm(d, hq, hk)
    new = lambda x: None if x is None else torch.empty_like(x)
    want = [new(q), new(k)]
    md.mdraft_qk_norm(spec, q, k, *want)
    far = [wide(q) if apart == "q" else q, wide(k) if apart == "k" else k]
    got = [new(q), new(k)]
    md.mdraft_qk_norm(spec, *far, *got)
    torch.cuda.synchronize()
    for a, b, x, h in zip(want, got, (q, k), (hq, hk)):
        if h:
            assert torch.equal(a, b)
            check(a, gdr.head_norm(x.double().cpu().numpy(), d, "l2"), d, 0, "half", "bf16")


@pytest.mark.parametrize("huge", [1e4, 1e12, 3e38, float("inf")])
@pytest.mark.parametrize("n,hv", [(24, 2), (200, 2), (200, 40)])
def test_one_token_that_forgets_everything_leaves_the_decays_behind_it_exact(n, hv, huge):
    """A step size that takes the decay to zero, however large: what the tokens behind it write decays as ever."""
    p = Problem(n, 1, hv, seed=71)
    p.np["dt"][[5, n // 2, n // 2 + 1, n - 10]] = torch.tensor(huge).bfloat16().float().item()
    p.upload()
    cache, out, status = p.cache(2), p.out(), torch.zeros(1, dtype=torch.int32, device="cuda")
    h0 = p.states(1)
    cache.ssm[0, 0] = torch.from_numpy(h0[0]).cuda()
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, n, i32([0]), i32([1]), p.workspace(1, n), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    with np.errstate(over="ignore"):
        w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=[0, n], S0=h0, sizes=True)
    check_states(cache.ssm[0, 1], np.asarray(w_states)[0])
    p.check_out(out, w_out, o, size, size64 if is_chunked(p, [n]) else None)


@pytest.mark.parametrize("act,n,hv", [("bf16", 24, 2), ("f32", 100, 2), ("bf16", 200, 2), ("bf16", 200, 40)])
@pytest.mark.parametrize("which", ["k", "v", "dt", "beta"])
def test_a_nan_reaches_every_token_behind_it(act, n, hv, which):
    """As in the recurrence: no clamp, comparison or mask on the way of a decay, a strength or an operand takes it for a number."""
    t = n // 2
    p = Problem(n, 1, hv, act=act, gate=False, norm=False, seed=72)
    p.np[which][t] = np.nan
    p.upload()
    cache, out = p.cache(1), p.out()
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, n, None, i32([0]), p.workspace(1, n))
    torch.cuda.synchronize()
    assert bool(out[t:].isnan().all()) and bool(cache.ssm.isnan().all())
    assert bool(out[:t // 64 * 64].isfinite().all())


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("which", ["k", "v", "dt", "beta"])
def test_a_nan_reaches_the_nodes_below_it(act, which):
    p = Problem(4, 1, 2, act=act, gate=False, norm=False, seed=73)
    p.np[which][1] = np.nan
    p.upload()
    cache, out = p.cache(5), p.out()
    cache.ssm[0, 0] = torch.from_numpy(p.states(1)[0]).cuda()
    md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, out, i32([0, 0, 1, 2]), i32([1, 2, 3, 4]), [0, 2, 4])   # nodes 0 and 1 below the root, 2 below 0, 3 below 1
    torch.cuda.synchronize()
    for node, bad in enumerate((False, True, False, True)):
        assert bool(out[node].isnan().all() if bad else out[node].isfinite().all())
        assert bool(cache.ssm[0, 1 + node].isnan().all() if bad else cache.ssm[0, 1 + node].isfinite().all())
