"""The outputs of the delta layer's encode in chunks are off by little more than their own rounding, as those of the encode token by token are: a call's results
do not depend on the way it is done beyond that.

Bounds.  Before norm and gate an output of the narrow chain is scale e^G (S q) + M X, with the chunk's incoming state S, X what its tokens wrote and M the
masked products of queries and keys.  S, M and X go into the products as two bf16 values each, whose remainders are off by 2^-8 (half a step) of 2^-8: 2^-16 of every
product for S, as much for M, for X and for the product of the two second parts, which is left out.  With what fp32 sums and the state's own error
make of the products' sizes (STATE, test_gpu_gdr.py) that is STATE of the outputs' size and (3 2^-16 + STATE) of the size of the products of both sums.  What an error becomes on
its way through norm, weight and gate, and the last rounding, are as test_gpu_gdr.py has them.
"""

import numpy as np
import pytest

from oracle import gdr
from test_gpu_gdr import STATE, Problem, is_chunked, run_encode

pytestmark = pytest.mark.gpu

CHUNKED = 3 * 2.0 ** -16 + STATE


def check(p, got, want, o, e):
    """e: what the outputs may be off by before norm and gate."""
    got, w = got.double().cpu().numpy(), np.asarray(want)
    gate = np.ones_like(w) if p.np["z"] is None else np.abs(gdr.silu(p.np["z"].astype(np.float64)))
    if p.norm_w is not None:
        f = 1.0 / np.sqrt(np.mean(o * o, axis=-1, keepdims=True) + 1e-5)
        e = f * np.abs(p.norm_w) * (e + np.abs(o) * f * np.sqrt(np.mean(e * e, axis=-1, keepdims=True)))
    over = np.abs(got - w) - e.reshape(w.shape) * gate - 2.0 ** -8 * np.abs(w)
    assert np.all(np.isfinite(got)) and np.all(over <= 1e-30), float(over.max())


SIZES = [(2, 4, 128, 128), (1, 1, 64, 64), (3, 3, 128, 64), (1, 3, 64, 128)]


@pytest.mark.parametrize("hk,hv,dk,dv", SIZES)
@pytest.mark.parametrize("lens,init,gate,norm", [([300], True, True, True), ([65], False, False, False), ([64, 1, 130], True, False, True)])
def test_narrow_chain(hk, hv, dk, dv, lens, init, gate, norm):
    p = Problem(sum(lens), hk, hv, dk, dv, gate=gate, norm=norm, seed=90 + sum(lens))
    assert is_chunked(p, lens)
    cu, h0, out, states = run_encode(p, lens, init)
    want, _, o, size, size64 = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)
    check(p, out, want, o, STATE * size + CHUNKED * size64)


def test_the_same_tokens_in_chunks_and_token_by_token():
    """64 tokens in a call of their own (token by token) and as the first of 128 (in chunks): both within the bounds of the same statement."""
    p = Problem(64, 1, 2, seed=91)
    long = Problem(128, 1, 2, seed=92)
    for n in p.np:
        if p.np[n] is not None:
            long.np[n][:64] = p.np[n]
    long.A, long.dt_bias, long.norm_w = p.A, p.dt_bias, p.norm_w
    long.upload()
    assert not is_chunked(p, [64]) and is_chunked(long, [128])
    a, b = run_encode(p, [64])[2], run_encode(long, [128])[2][:64]
    want, _, o, size, size64 = gdr.encode(**p.args(), cu=[0, 64], sizes=True)
    check(p, a, want, o, STATE * size)
    check(p, b, want, o, STATE * size + CHUNKED * size64)


# ---------------------------------------------------------------- the wide chain
# Its outputs are scale e^G (S q) + (M T) R with R = V - e^G (K S^T) and T the inverse of the chunk's triangle: other products than M X, though the same sum.  The second
# parts of S and R are truncated, 2^-7 of 2^-8; M T is rounded twice, 2^-16; the product of the second parts of M T and R is left out, 2^-16.
WIDE_S, WIDE_MT = 2.0 ** -15, 2.0 ** -15 + 2 * 2.0 ** -16


def wide_sizes(p, cu, S0):
    """(T, Hv, d_v): sums of the sizes of the products of either sum, in 64 bits, a chunk at a time by the closed form."""
    a = {n: None if v is None else np.asarray(v, np.float64) for n, v in p.args().items() if n in ("q", "k", "v", "dt", "beta", "A", "dt_bias")}
    x = np.logaddexp(0.0, a["dt"] + a["dt_bias"]) * a["A"]
    beta, scale, dk, dv = 1 / (1 + np.exp(-a["beta"])), p.dk ** -0.5, p.dk, p.dv
    of_s, of_mt = np.zeros((p.rows, p.hv, dv)), np.zeros((p.rows, p.hv, dv))
    for s in range(len(cu) - 1):
        for h in range(p.hv):
            S = np.zeros((dv, dk)) if S0 is None else np.asarray(S0, np.float64).reshape(-1, p.hv, dv, dk)[s, h]
            g = slice(h // (p.hv // p.hk) * dk, (h // (p.hv // p.hk) + 1) * dk)
            for t in range(int(cu[s]), int(cu[s + 1]), 64):
                r = slice(t, min(t + 64, int(cu[s + 1])))
                q, k, v, b, G = a["q"][r, g], a["k"][r, g], a["v"][r, h * dv:(h + 1) * dv], beta[r, h], np.cumsum(x[r, h])
                between = np.tril(np.exp(np.minimum(G[:, None] - G, 0)))
                T = np.linalg.inv(np.eye(len(G)) + np.tril(b[:, None] * between * (k @ k.T), -1)) * b
                M, R = scale * between * (q @ k.T), v - np.exp(G)[:, None] * (k @ S.T)
                of_s[r, h], of_mt[r, h] = scale * np.exp(G)[:, None] * (np.abs(q) @ np.abs(S).T), np.abs(M @ T) @ np.abs(R)
                S = np.exp(G[-1]) * S + (np.exp(G[-1] - G)[:, None] * (T @ R)).T @ k
    return of_s, of_mt


MANY = [(38, 38, 128, 128), (13, 39, 64, 128), (5, 80, 128, 64), (76, 76, 64, 64)]   # plan_gdr (csrc/api.cu): a whole head per block


@pytest.mark.parametrize("hk,hv,dk,dv", MANY)
@pytest.mark.parametrize("lens,init,gate,norm", [([200], True, True, True), ([65], False, False, False), ([64, 1, 70], True, False, True)])
def test_wide_chain(hk, hv, dk, dv, lens, init, gate, norm):
    p = Problem(sum(lens), hk, hv, dk, dv, gate=gate, norm=norm, seed=93 + sum(lens))
    assert is_chunked(p, lens)
    cu, h0, out, states = run_encode(p, lens, init)
    want, _, o, size = gdr.encode(**p.args(), cu=cu, S0=h0, sizes=True)[:4]
    of_s, of_mt = wide_sizes(p, cu, h0)
    check(p, out, want, o, STATE * (size + of_s + of_mt) + WIDE_S * of_s + WIDE_MT * of_mt)
