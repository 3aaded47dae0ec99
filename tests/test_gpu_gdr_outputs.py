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
