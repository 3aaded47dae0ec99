"""The delta layer (context encode, tree step, commit) against the fp64 statement of oracle/gdr.py.

Tolerances.  States are fp32.  A token's dot products of d_k <= 128 values, taken in a few partial sums, are off by at most
(16 + 3 + 2) 2^-24 of the sum of the products' sizes, the update by 3 * 2^-24 of the entry; with random signs over the some hundred tokens that
these tests run (errors decay with the state) the state is off by no more than 1e-5 of max(|entry|, rms): STATE.  The chunked encode's
products take operands split into three bf16 values (24 bits) and stay inside the same bound.
Outputs before norm and gate are sums of d_k products scale S q: each is off by the state's error and (16 + 3 + 2) 2^-24, together
no more than STATE of its size, so the sum is off by STATE times the sum of the products' sizes (which can be far more than
the output where a query hardly meets the state).  The chunked encode rounds one operand of each of its two output products to bf16 (the
incoming state; the masked products of queries and keys): 2^-8 of every product's size more, over the incoming state's products
and the chunk's.  An error e of a row goes through the norm as e / sqrt(mean o^2 + eps) and, by the row's mean square, as the output
times rms(e) / sqrt(mean o^2 + eps); then times weight and gate.  Last comes half a step of the result's type (2^-8; fp32: 2^-22 for
the roundings of norm and gate).
"""

import numpy as np
import pytest
import torch

import gen
from oracle import gdr

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md
from paper_2506_01206_b200.device_inputs import i32

STATE = 1e-5
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Problem:
    """A delta layer with inputs: numpy in the activation type's values for the statement, strided tensors on the device for the library."""

    def __init__(self, rows, hk=2, hv=4, dk=128, dv=128, act="bf16", gate=True, norm=True, seed=0, unit=True, raw=False, pad=16):
        g = np.random.default_rng(seed)
        rnd = lambda a: gen.round_to_act(np.asarray(a, dtype=np.float32), act)
        self.hk, self.hv, self.dk, self.dv, self.act, self.rows = hk, hv, dk, dv, act, rows
        k = g.normal(size=(rows, hk, dk))
        if unit:
            k /= np.linalg.norm(k, axis=-1, keepdims=True)
        q = g.normal(size=(rows, hk, dk))
        q /= np.linalg.norm(q, axis=-1, keepdims=True)
        self.flags = 0 if raw else md.MDRAFT_DT_SOFTPLUS | md.MDRAFT_BETA_SIGMOID
        self.np = {"q": rnd(q.reshape(rows, hk * dk)), "k": rnd(k.reshape(rows, hk * dk)), "v": rnd(g.normal(size=(rows, hv * dv))),
                   "z": rnd(g.normal(size=(rows, hv * dv))) if gate else None,
                   "dt": rnd(np.abs(g.normal(size=(rows, hv))) * 0.05 if raw else 0.5 * g.normal(size=(rows, hv))),
                   "beta": rnd(g.uniform(0, 1, size=(rows, hv)) if raw else g.normal(size=(rows, hv)))}
        self.A = -g.uniform(0.5, 16, size=hv).astype(np.float32)
        self.dt_bias = None if raw else np.full(hv, -4.579712, dtype=np.float32)
        self.norm_w = (1 + 0.2 * g.normal(size=dv)).astype(np.float32) if norm else None
        self.pad = pad
        self.g = g
        self.upload()

    def upload(self):
        t = DT[self.act]
        n = self.np
        qkv = np.concatenate([n["q"], n["k"], n["v"]], axis=1)
        u = torch.full((self.rows + 3, qkv.shape[1] + self.pad), float("nan"), dtype=t, device="cuda")   # NaN beside and behind the rows
        u[:self.rows, :qkv.shape[1]] = torch.from_numpy(qkv).to(t)
        a, b = self.hk * self.dk, self.hv * self.dv
        u = u[:self.rows]
        gates = torch.full((self.rows + 3, 2 * self.hv + 1), float("nan"), dtype=t, device="cuda")
        gates[:self.rows, :self.hv], gates[:self.rows, self.hv:2 * self.hv] = torch.from_numpy(n["dt"]).to(t), torch.from_numpy(n["beta"]).to(t)
        self.dev = [u[:, :a], u[:, a:2 * a], u[:, 2 * a:2 * a + b], None if n["z"] is None else torch.from_numpy(n["z"]).to(t).cuda(),
                    gates[:self.rows, :self.hv], gates[:self.rows, self.hv:2 * self.hv]]
        f = lambda x: None if x is None else torch.from_numpy(x).cuda()
        self.layer = md.GdrLayer(f(self.A), f(self.dt_bias), f(self.norm_w), self.hk, self.dk, self.dv, t, self.flags)

    def states(self, n):
        return (0.3 * self.g.normal(size=(n, self.hv * self.dv, self.dk))).astype(np.float32)

    def cache(self, slots, n_layers=1):
        c = md.StateCache(n_layers, slots, self.hv * self.dv, d_state=self.dk, act=DT[self.act])
        c.ssm.fill_(float("nan"))
        return c

    def args(self):
        soft = bool(self.flags & md.MDRAFT_DT_SOFTPLUS)
        return dict(**self.np, A=self.A, dt_bias=self.dt_bias, norm_w=self.norm_w, n_k_heads=self.hk, d_k=self.dk, d_v=self.dv, softplus=soft, sigmoid=soft)

    def out(self, rows=None):
        return torch.full((self.rows if rows is None else rows, self.hv * self.dv), float("nan"), dtype=DT[self.act], device="cuda")

    def workspace(self, n_seq, longest):
        n = md.mdraft_gdr_prefill_workspace_bytes(self.layer, self.rows, n_seq, longest)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None   # NaN in every word

    def check_out(self, got, want, o, size, size64=None):
        got, w = got.double().cpu().numpy(), np.asarray(want)
        e = STATE * size + (0.0 if size64 is None else 2.0 ** -8 * size64)
        gate = np.ones_like(w) if self.np["z"] is None else np.abs(gdr.silu(self.np["z"].astype(np.float64)))
        if self.norm_w is not None:
            f = 1.0 / np.sqrt(np.mean(o * o, axis=-1, keepdims=True) + 1e-5)
            e = f * np.abs(self.norm_w) * (e + np.abs(o) * f * np.sqrt(np.mean(e * e, axis=-1, keepdims=True)))
        over = np.abs(got - w) - e.reshape(w.shape) * gate - (2.0 ** -8 if self.act == "bf16" else 2.0 ** -22) * np.abs(w)
        assert np.all(np.isfinite(got)) and np.all(over <= 1e-30), float(over.max())


def check_states(got, want):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    assert np.all(np.isfinite(got))
    floor = np.sqrt(np.mean(want * want)) if want.size else 1.0
    assert np.max(np.abs(got - want) / np.maximum(np.abs(want), floor), initial=0.0) <= STATE


def run_encode(p, lens, init=False, offsets=True, in_place=False):
    S = len(lens)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cache, status, out = p.cache(2 * S), torch.zeros(1, dtype=torch.int32, device="cuda"), p.out()
    h0 = p.states(S) if init else None
    if init:
        cache.ssm[0, :S] = torch.from_numpy(h0).cuda()
    final = np.arange(S) if in_place else np.arange(S, 2 * S)
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32(cu) if offsets else None, max(lens), i32(np.arange(S)) if init else None, i32(final),
                          p.workspace(S, max(lens)), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return cu, h0, out, cache.ssm[0, torch.from_numpy(final).cuda()]


def is_chunked(p, lens):
    return md.mdraft_gdr_prefill_workspace_bytes(p.layer, sum(lens), len(lens), max(lens)) > 0


SIZES = [(2, 4, 128, 128), (1, 1, 64, 64), (3, 3, 128, 64), (1, 3, 64, 128)]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("hk,hv,dk,dv", SIZES)
@pytest.mark.parametrize("lens,init", [([1], True), ([40], False), ([64], True), ([200], False), ([1, 2, 0, 63, 64, 65, 130, 16, 17], True)])
def test_encode_matches_the_statement(act, hk, hv, dk, dv, lens, init):
    p = Problem(sum(lens), hk, hv, dk, dv, act, gate=init, norm=dk == dv, seed=sum(lens))
    cu, h0, out, states = run_encode(p, lens, init)
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    check_states(states, w_states)
    p.check_out(out, w_out, o, size, size64 if is_chunked(p, lens) else None)


# As many heads as make the library take a whole head per block, in single sequences too (plan_gdr in csrc/api.cu).
MANY = [(38, 38, 128, 128), (13, 39, 64, 128), (5, 80, 128, 64), (76, 76, 64, 64)]


@pytest.mark.parametrize("hk,hv,dk,dv", MANY)
@pytest.mark.parametrize("lens,init", [([40], False), ([64], True), ([200], True), ([1, 2, 0, 63, 64, 65, 130], True)])
def test_encode_of_many_heads_matches_the_statement(hk, hv, dk, dv, lens, init):
    p = Problem(sum(lens), hk, hv, dk, dv, gate=init, norm=dk == dv, seed=sum(lens) + hv)
    cu, h0, out, states = run_encode(p, lens, init, offsets=len(lens) > 1)
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    check_states(states, w_states)
    p.check_out(out, w_out, o, size, size64)


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("n,hv", [(9, 2), (150, 2), (150, 38)])
def test_encode_with_and_without_norm_and_gate(gate, norm, n, hv):
    p = Problem(n, 1, hv, gate=gate, norm=norm, seed=4)
    cu, h0, out, states = run_encode(p, [n], True, offsets=False)
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    check_states(states, w_states)
    p.check_out(out, w_out, o, size, size64 if is_chunked(p, [n]) else None)


@pytest.mark.parametrize("lens,hv", [([5, 9, 3], 4), ([100, 1, 70], 4), ([100, 1, 0, 70, 200], 8)])
def test_encode_in_place_equals_slot_to_slot(lens, hv):
    a = run_encode(Problem(sum(lens), hv=hv, seed=5), lens, True)
    b = run_encode(Problem(sum(lens), hv=hv, seed=5), lens, True, in_place=True)
    assert torch.equal(a[2].view(torch.int16), b[2].view(torch.int16)) and torch.equal(a[3], b[3])


@pytest.mark.parametrize("hv", [2, 38])
def test_encode_with_raw_gates_and_keys_of_other_sizes(hv):
    """Step sizes and strengths as given, zero among them; keys twice and a hundredth of unit length with strengths that fit."""
    for scale, cap in ((2.0, 0.4), (0.01, 1.0)):
        p = Problem(140, 2, hv, raw=True, seed=6)
        p.np["k"] = gen.round_to_act((p.np["k"] * scale).astype(np.float32), "bf16")
        p.np["beta"] = gen.round_to_act((p.np["beta"] * cap).astype(np.float32), "bf16")
        p.np["dt"][::3] = 0
        p.np["beta"][::5] = 0
        p.upload()
        cu, h0, out, states = run_encode(p, [140], True)
        w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
        check_states(states, w_states)
        p.check_out(out, w_out, o, size, size64)


@pytest.mark.parametrize("n,hv", [(10, 2), (130, 2), (130, 38)])
def test_nothing_written_and_nothing_decayed_leaves_the_state_as_it_was(n, hv):
    p = Problem(n, 1, hv, raw=True, seed=7)
    p.np["dt"][:] = 0
    p.np["beta"][:] = 0
    p.upload()
    cu, h0, out, states = run_encode(p, [n], True)
    assert torch.equal(states, torch.from_numpy(h0).cuda())


@pytest.mark.parametrize("n,hv", [(20, 1), (150, 1), (150, 38)])
def test_the_same_key_again_and_again(n, hv):
    """Identical keys at full strength: the state holds the last value only; the triangle of a chunk is as full as it gets."""
    p = Problem(n, 1, hv, raw=True, seed=8, gate=False, norm=False)
    p.np["k"][:] = 0
    p.np["k"][:, 3] = 1
    p.np["beta"][:] = 1
    p.upload()
    cu, h0, out, states = run_encode(p, [n], True)
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    check_states(states, w_states)
    p.check_out(out, w_out, o, size, size64 if is_chunked(p, [n]) else None)


@pytest.mark.parametrize("n,times", [(24, 1), (200, 1), (200, 10)])
def test_steep_and_absent_decay(n, times):
    """Heads that forget everything at once (their log decays sum to -10^4 in a chunk), heads that forget nothing."""
    p = Problem(n, 2, 4 * times, seed=9)
    p.A[:] = [-3000.0, 0.0, -300.0, -1e-3] * times
    p.np["dt"][:] = gen.round_to_act(np.random.default_rng(1).uniform(-3, 8, size=p.np["dt"].shape).astype(np.float32), "bf16")
    p.upload()
    cu, h0, out, states = run_encode(p, [n], True)
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    got, want = (np.asarray(x).reshape(-1, 128, 128) for x in (states[0].double().cpu().numpy(), w_states[0]))
    for j in range(4 * times):   # per head: their sizes differ
        check_states(torch.from_numpy(got[j]), want[j])
    p.check_out(out, w_out, o, size, size64 if is_chunked(p, [n]) else None)


@pytest.mark.parametrize("lens,hv", [([3, 4, 5], 4), ([70, 80, 90], 4), ([70, 80, 90], 14)])
def test_values_of_other_sequences_and_of_rows_behind_them_do_not_matter(lens, hv):
    """NaN in one sequence's rows and in the rows that belong to none leave the other sequences as they are; those rows' outputs stay unwritten."""
    T = sum(lens) + 7
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    res = []
    for spoil in (False, True):
        p = Problem(T, hv=hv, seed=10)
        if spoil:
            for n in ("q", "k", "v", "z", "dt", "beta"):
                p.np[n][cu[1]:cu[2]] = np.nan
                p.np[n][cu[3]:] = np.inf
            p.upload()
        cache, status, out = p.cache(3), torch.zeros(1, dtype=torch.int32, device="cuda"), p.out()
        md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32(cu), max(lens), None, i32([0, 1, 2]), p.workspace(3, max(lens)), status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0 and bool(out[cu[3]:].isnan().all())
        res.append((out, cache.ssm[0]))
    for s in (0, 2):
        assert torch.equal(res[0][0][cu[s]:cu[s + 1]], res[1][0][cu[s]:cu[s + 1]]) and torch.equal(res[0][1][s], res[1][1][s])


@pytest.mark.parametrize("lens,hv", [([3, 4], 4), ([70, 80], 4), ([70, 80], 20)])
def test_bad_slots_and_offsets_are_flagged_not_followed(lens, hv):
    p = Problem(sum(lens), hv=hv, seed=12)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ws = p.workspace(2, max(lens))
    for final, offsets, init, bit, good in (([0, 9], cu, None, md.MDRAFT_DEV_BAD_SLOT, 0), ([0, 1], cu, [5, -1], md.MDRAFT_DEV_BAD_SLOT, 1),
                                            ([0, 1], [0, lens[0], 1], None, md.MDRAFT_DEV_BAD_SEQLENS, 0),
                                            ([0, 1], [0, lens[0], 10 ** 6], None, md.MDRAFT_DEV_BAD_SEQLENS, 0)):
        cache, status, out = p.cache(3), torch.zeros(1, dtype=torch.int32, device="cuda"), p.out()
        cache.ssm.fill_(5.0)
        md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32(offsets), max(lens), None if init is None else i32(init), i32(final), ws, status)
        torch.cuda.synchronize()
        assert int(status.item()) == bit
        rows = [out[:lens[0]], out[lens[0]:]]
        assert bool(rows[good].isfinite().all()) and bool(rows[1 - good].isnan().all())
        assert not bool((cache.ssm[0, good] == 5.0).all()) and bool((cache.ssm[0, 1 - good] == 5.0).all()) and bool((cache.ssm[0, 2] == 5.0).all())


@pytest.mark.parametrize("hv", [4, 20])
def test_overlapping_sequences_stay_inside_the_workspace(hv):
    T = 300
    p = Problem(T, hv=hv, seed=13)
    need = md.mdraft_gdr_prefill_workspace_bytes(p.layer, T, 3, T)
    ws = torch.full((2 * need + 256,), 77, dtype=torch.uint8, device="cuda")
    cache, status, out = p.cache(3), torch.zeros(1, dtype=torch.int32, device="cuda"), p.out()
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32([0, T, 0, T]), T, None, i32([0, 1, 2]), ws[:need] if need else None, status)
    torch.cuda.synchronize()
    assert int(status.item()) & md.MDRAFT_DEV_BAD_SEQLENS and bool((ws[need:] == 77).all())
    _, w_states = gdr.encode(**p.args(), cu=[0, T])
    check_states(cache.ssm[0, :1], w_states)


def test_a_bound_on_the_length_that_is_too_low_changes_rounding_only():
    p = Problem(150, 1, 2, seed=14)
    out, cache = p.out(), p.cache(1)
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, 1, None, i32([0]), p.workspace(1, 150))
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=[0, 150], sizes=True)
    check_states(cache.ssm[0], w_states)
    p.check_out(out, w_out, o, size, size64)


def test_empty_batches():
    p = Problem(0, 1, 1)
    cache = p.cache(4)
    h = torch.randn((2, 128, 128), device="cuda")
    cache.ssm[0, :2] = h
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, p.out(), i32([0, 0, 0]), 0, i32([0, 1]), i32([2, 3]), p.workspace(2, 0))
    assert torch.equal(cache.ssm[0, 2:], h)
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, p.out(), i32([0, 0, 0]), 0, None, i32([2, 3]), p.workspace(2, 0))
    assert not bool(cache.ssm[0, 2:].any())


# ---------------------------------------------------------------- tree step
TREES = {"one": gen.chain_tree(1), "chain": gen.chain_tree(6), "full": gen.full_tree([2, 2, 2]), "paper": gen.paper_tree((3, 3, 2, 1))}


def tree_call(p, tree, cache, one_call=True, committed=True, stream=None):
    M = tree.n_nodes
    parent = i32(np.where(tree.parents < 0, 0 if committed else -1, tree.parents + 1))
    node, out, status = i32(np.arange(M) + 1), p.out(), torch.zeros(1, dtype=torch.int32, device="cuda")
    lv = [int(v) for v in tree.level_offsets]
    if one_call:
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, out, parent, node, lv, status, stream)
    else:
        cut = lambda t, a, b: None if t is None else t[a:b]
        for a, b in zip(lv[:-1], lv[1:]):
            md.mdraft_gdr_tree_step(p.layer, cache, 0, *[cut(t, a, b) for t in p.dev], out[a:b], parent[a:b], node[a:b], None, status, stream)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("hk,hv,dk,dv", SIZES)
@pytest.mark.parametrize("shape", TREES)
def test_tree_matches_the_statement(act, hk, hv, dk, dv, shape):
    tree = TREES[shape]
    p = Problem(tree.n_nodes, hk, hv, dk, dv, act, gate=shape != "full", norm=dk == dv, seed=20)
    committed = shape != "chain"
    h0 = p.states(1)[0] if committed else None
    outs = []
    for one_call in (True, False):
        cache = p.cache(1 + tree.n_nodes)
        if committed:
            cache.ssm[0, 0] = torch.from_numpy(h0).cuda()
        outs.append((tree_call(p, tree, cache, one_call, committed), cache.ssm[0, 1:]))
    w_out, w_states, o, size = gdr.tree(tree.parents, **p.args(), S0=h0, sizes=True)
    check_states(outs[0][1], w_states)
    p.check_out(outs[0][0], w_out, o, size)
    assert torch.equal(outs[0][0].view(torch.uint8), outs[1][0].view(torch.uint8)) and torch.equal(outs[0][1], outs[1][1]), "level by level: the same bits"


def test_tree_bad_slots_are_flagged_not_followed():
    p = Problem(4, seed=21)
    cache, status, out = p.cache(5), torch.zeros(1, dtype=torch.int32, device="cuda"), p.out()
    cache.ssm.fill_(5.0)
    md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, out, i32([0, 5, -2, 0]), i32([1, 2, 3, -1]), None, status)
    torch.cuda.synchronize()
    assert int(status.item()) == md.MDRAFT_DEV_BAD_SLOT
    assert bool(out[0].isfinite().all()) and bool(out[1:].isnan().all()) and bool((cache.ssm[0, 2:] == 5.0).all()) and not bool((cache.ssm[0, 1] == 5.0).all())


def test_second_layer_of_a_pool_and_strided_slots():
    """Layer 1 of a pool whose slots lie apart: only the named layer's named slots change."""
    p = Problem(3, 1, 2, 64, 64, seed=22)
    big = torch.full((2, 5, 2 * 128, 64), 7.0, device="cuda")
    cache = p.cache(4, n_layers=2)
    cache.ssm = big[:, :4, :128]
    h0 = p.states(1)[0]
    cache.ssm[1, 0] = torch.from_numpy(h0).cuda()
    out = p.out()
    md.mdraft_gdr_tree_step(p.layer, cache, 1, *p.dev, out, i32([0, 0, 0]), i32([1, 2, 3]))
    w_out, w_states = gdr.tree([-1, -1, -1], **p.args(), S0=h0)
    check_states(cache.ssm[1, 1:], w_states)
    assert bool((big[0] == 7.0).all()) and bool((big[:, :, 128:] == 7.0).all()) and bool((big[:, 4] == 7.0).all())


# ---------------------------------------------------------------- as they are used together
def test_conv_norm_encode_draft_commit():
    """A layer from its projection rows to a committed node: conv over q | k | v (window in the same pool), norm of q and k, encode; then a
    tree round of the same three calls below the encoded state, the commit of a node, and one more token from there.  Against the whole
    path encoded at once."""
    hk, hv, dk, dv = 2, 4, 128, 128
    ch = 2 * hk * dk + hv * dv
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")
    conv = md.Layer(-torch.ones((ch, 16), device="cuda"), None, rand(ch, 4) * 0.5, None, None, torch.bfloat16, md.MDRAFT_CONV_ONLY)
    rule = md.GdrLayer(-torch.rand(hv, device="cuda", generator=g) * 8, torch.full((hv,), -4.5, device="cuda"), torch.ones(dv, device="cuda"), hk, dk, dv)
    norm = md.QkNorm(dk, hk, hk)
    ctx, tree = 150, gen.full_tree([2, 2])
    path = [0, 2, 5]   # root, its second child, that one's first
    assert list(tree.parents) == [-1, 0, 0, 1, 1, 2, 2]
    x = rand(ctx + tree.n_nodes + 1, ch).bfloat16()
    z, dt, b = rand(x.shape[0], hv * dv).bfloat16(), rand(x.shape[0], hv).bfloat16(), rand(x.shape[0], hv).bfloat16()
    ws = torch.empty(max(256, md.mdraft_prefill_workspace_bytes(conv, 200, 1, 200), md.mdraft_gdr_prefill_workspace_bytes(rule, 200, 1, 200)), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    pool = lambda n: md.StateCache(1, n, hv * dv, d_state=dk, conv_channels=ch)
    split = lambda u: (u[:, :hk * dk], u[:, hk * dk:2 * hk * dk], u[:, 2 * hk * dk:])

    def behind_conv(u):
        q, k, v = split(u)
        md.mdraft_qk_norm(norm, q, k, q, k)
        return q, k, v

    def encode(cache, rows, final):
        u, out = torch.empty((len(rows), ch), dtype=torch.bfloat16, device="cuda"), torch.empty((len(rows), hv * dv), dtype=torch.bfloat16, device="cuda")
        md.mdraft_conv_scan_prefill(conv, cache, 0, x[rows], None, None, None, None, u, None, len(rows), None, i32([final]), ws, 0, status)
        md.mdraft_gdr_prefill(rule, cache, 0, *behind_conv(u), z[rows], dt[rows], b[rows], out, None, len(rows), None, i32([final]), ws, status)
        return out

    def step(cache, rows, parent, node, levels):
        u, out = torch.empty((len(rows), ch), dtype=torch.bfloat16, device="cuda"), torch.empty((len(rows), hv * dv), dtype=torch.bfloat16, device="cuda")
        md.mdraft_tree_step(conv, cache, 0, x[rows], None, None, None, None, u, i32(parent), i32(node), levels, status)
        md.mdraft_gdr_tree_step(rule, cache, 0, *behind_conv(u), z[rows], dt[rows], b[rows], out, i32(parent), i32(node), levels, status)
        return out

    M = tree.n_nodes
    cache = pool(1 + M)
    encode(cache, list(range(ctx)), 0)
    nodes = step(cache, list(range(ctx, ctx + M)), [0] + [1 + int(p) for p in tree.parents[1:]], list(range(1, M + 1)), [int(v) for v in tree.level_offsets])
    md.mdraft_state_commit(cache, i32([1 + path[-1]]), i32([0]), status)
    assert torch.equal(cache.ssm[0, 0], cache.ssm[0, 1 + path[-1]]) and torch.equal(cache.conv[0, 0], cache.conv[0, 1 + path[-1]])
    last = step(cache, [ctx + M], [0], [0], None)
    whole = pool(1)
    rows = list(range(ctx)) + [ctx + v for v in path] + [ctx + M]
    want = encode(whole, rows, 0)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    assert torch.equal(cache.conv[0, 0], whole.conv[0, 0])
    # both sides round to bf16 at the same places (conv, norm); what differs is fp32 summation, and operand roundings of the chunked outputs
    scale = float(whole.ssm.square().mean().sqrt())
    assert float((cache.ssm[0, 0] - whole.ssm[0, 0]).abs().max()) <= 2 * STATE * max(scale, float(whole.ssm.abs().max()))
    got = torch.cat([nodes[path], last]).float()
    ref = want[ctx:].float()
    assert float((got - ref).abs().max()) <= (2.0 ** -7 + 8 * 2.0 ** -9) * float(ref.abs().max())


def test_on_another_stream_and_replayed_from_a_graph():
    tree = TREES["paper"]
    p = Problem(tree.n_nodes, seed=30)
    h0 = torch.from_numpy(p.states(1)[0]).cuda()

    def fresh():
        c = p.cache(1 + tree.n_nodes)
        c.ssm[0, 0] = h0
        return c
    a = fresh()
    want = tree_call(p, tree, a)
    s = torch.cuda.Stream()
    b = fresh()
    torch.cuda.synchronize()
    got = tree_call(p, tree, b, stream=s)
    assert torch.equal(want, got) and torch.equal(a.ssm, b.ssm)
    # a graph of an encode and a round, replayed after its inputs have changed
    e = Problem(200, seed=31)
    cache, out, o2 = e.cache(2 + tree.n_nodes), e.out(), p.out()
    final, ws = i32([0]), e.workspace(1, 200)
    parent, node, lv = i32(np.where(tree.parents < 0, 0, tree.parents + 1)), i32(np.arange(tree.n_nodes) + 1), [int(v) for v in tree.level_offsets]

    def both():
        md.mdraft_gdr_prefill(e.layer, cache, 0, *e.dev, out, None, 200, None, final, ws)
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, o2, parent, node, lv)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    e.dev[2].mul_(0.5)
    p.dev[0].mul_(2.0)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    r = [t.clone() for t in (out, o2, cache.ssm[0, :1 + tree.n_nodes])]
    both()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(r, (out, o2, cache.ssm[0, :1 + tree.n_nodes])))


def test_calls_in_a_row_on_one_workspace():
    """Encodes of different shapes one behind another without a wait, sharing a workspace, equal the same calls alone."""
    ps = [(Problem(n, hk, hv, dk, dv, seed=40 + n), lens) for n, hk, hv, dk, dv, lens in
          ((300, 2, 4, 128, 128, [300]), (260, 1, 3, 64, 128, [130, 130]), (200, 2, 40, 128, 128, [200]), (70, 3, 39, 64, 64, [33, 37]), (90, 2, 2, 128, 64, [9, 81]), (500, 2, 4, 128, 128, [500]), (24, 1, 1, 128, 128, [8, 16]))]
    alone = [run_encode(p, lens, False)[2:] for p, lens in ps]
    need = max(md.mdraft_gdr_prefill_workspace_bytes(p.layer, p.rows, len(lens), max(lens)) for p, lens in ps)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    calls = []
    for p, lens in ps:
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        calls.append((p, i32(cu), max(lens), p.cache(len(lens)), i32(np.arange(len(lens))), p.out()))
    torch.cuda.synchronize()
    for _ in range(3):
        for p, cu, longest, cache, final, out in calls:
            md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, cu, longest, None, final, ws)
    torch.cuda.synchronize()
    for (o, s), (p, cu, longest, cache, final, out) in zip(alone, calls):
        assert torch.equal(o.view(torch.int16), out.view(torch.int16)) and torch.equal(s, cache.ssm[0])


def test_refusals():
    p = Problem(5, 1, 2, 64, 64)
    cache = p.cache(2)
    call = lambda args, out=None, c=cache, **kw: md.mdraft_gdr_prefill(p.layer, c, 0, *args, p.out() if out is None else out, None, 5, None, i32([0]), None, **kw)
    call(p.dev)
    for i in range(6):
        with pytest.raises(ValueError):
            call([t[:4] if j == i else t for j, t in enumerate(p.dev)])
        with pytest.raises(TypeError):
            call([t.float() if j == i else t for j, t in enumerate(p.dev)])
    with pytest.raises(ValueError):
        call(p.dev, out=p.out(4))
    with pytest.raises(ValueError):
        call(p.dev, c=md.StateCache(1, 2, 128, d_state=128))
    with pytest.raises(TypeError):
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, p.out(), torch.zeros(5, dtype=torch.int64, device="cuda"), i32([0, 1, 0, 1, 0]))
    with pytest.raises(ValueError):
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *p.dev, p.out(), i32([0]), i32([0, 1, 0, 1, 0]))
    with pytest.raises(md.MdraftError):
        md.mdraft_gdr_tree_step(p.layer, cache, 3, *p.dev, p.out(), i32([0] * 5), i32([1] * 5))


def test_a_single_row_may_have_any_row_stride():
    p = Problem(1, 1, 1, 64, 64, seed=3)
    outs = []
    for dev in (p.dev, [t.T.contiguous().T for t in p.dev]):   # strides (1, 1)
        cache, out = p.cache(1), p.out()
        md.mdraft_gdr_tree_step(p.layer, cache, 0, *dev, out, i32([-1]), i32([0]))
        outs.append(out)
    assert torch.equal(outs[0], outs[1])
