"""The decays of the delta layer alone: tokens that write nothing (beta = 0 as given), so that a state only shrinks, by exp(sum of softplus(dt) A), which
is compared entry by entry with that power in 64 bits.

Bound, in units of u = 2^-24 relative to the entry.  exp_f32 is off by no more than 2: its argument's rounding errors, together at most 1.5 u of |y| <= 0.347, the
rounding of the last sum (1) and the series' remainder (0.1).  softplus = log1p(exp): 2 from the exp (log1p passes on no more than what its argument is off by) and
2 for log1pf (one unit of the last place); the product with A: 1; a decay of X in all is so off by 5 X.  A token (token by token) or a chunk of 64 tokens (in chunks) then is one
exp, 2, and one multiplication of the state, 1.  Together 5 X + 3 per token or chunk.
"""

import numpy as np
import pytest
import torch

import gen
from test_gpu_gdr import DT, i32

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md

U = 2.0 ** -24


def layer_and_rows(rows, hv, act, A, spread, d):
    """One head for each of hv step sizes: softplus of the values from spread[0] to spread[1], the same in every row."""
    t = DT[act]
    dt = gen.round_to_act(np.linspace(*spread, hv).astype(np.float32), act).astype(np.float64)
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda n: torch.randn((rows, n), generator=g, device="cuda").to(t)
    layer = md.GdrLayer(torch.full((hv,), A, device="cuda"), None, None, 1, d, d, t, md.MDRAFT_DT_SOFTPLUS)
    dev = [rand(d), rand(d), rand(hv * d), None, torch.from_numpy(np.tile(dt, (rows, 1))).to(t).cuda(), torch.zeros((rows, hv), dtype=t, device="cuda")]
    s0 = torch.randn((hv * d, d), generator=g, device="cuda")
    x = np.log1p(np.exp(dt)) * float(np.float32(A))   # log of a token's decay
    return layer, dev, s0, x


def check(got, s0, x, tokens, steps, d):
    got, s0 = (a.double().cpu().numpy().reshape(len(x), d, d) for a in (got, s0))
    want = s0 * np.exp(tokens * x)[:, None, None]
    bound = 5 * tokens * np.abs(x) + 3 * steps
    over = np.abs(got - want) - U * bound[:, None, None] * np.abs(want)
    assert np.all(np.isfinite(got)) and np.all(over <= 0), over.max(axis=(1, 2))


# the branch of softplus where exp(dt) is neither small nor large, and both sides of it
SPREADS = [(-3.46, -2.0), (-2.0, 3.0), (-9.0, -3.47)]


@pytest.mark.parametrize("act,tokens,hv", [("bf16", 24, 16), ("f32", 24, 16), ("f32", 480, 64)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spread", SPREADS)
def test_token_by_token(act, tokens, hv, d, spread):
    A = -3.0 / (24 * np.log1p(np.exp(spread[1])))
    layer, dev, s0, x = layer_and_rows(tokens, hv, act, A, spread, d)
    cache, out = md.StateCache(1, 1, hv * d, d_state=d, act=DT[act]), torch.empty((tokens, hv * d), dtype=DT[act], device="cuda")
    cache.ssm[0, 0] = s0
    assert md.mdraft_gdr_prefill_workspace_bytes(layer, tokens, 1, tokens) == 0
    md.mdraft_gdr_prefill(layer, cache, 0, *dev, out, None, tokens, i32([0]), i32([0]))
    torch.cuda.synchronize()
    check(cache.ssm[0, 0], s0, x, tokens, tokens, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spread", SPREADS)
@pytest.mark.parametrize("tokens,hv", [(1024, 12), (1000, 76)])   # the narrow and the wide chain
def test_in_chunks(d, spread, tokens, hv):
    A = -3.0 / (tokens * np.log1p(np.exp(spread[1])))
    layer, dev, s0, x = layer_and_rows(tokens, hv, "bf16", A, spread, d)
    cache, out, status = md.StateCache(1, 1, hv * d, d_state=d), torch.empty((tokens, hv * d), dtype=torch.bfloat16, device="cuda"), i32([0])
    cache.ssm[0, 0] = s0
    need = md.mdraft_gdr_prefill_workspace_bytes(layer, tokens, 1, tokens)
    assert need > 0
    md.mdraft_gdr_prefill(layer, cache, 0, *dev, out, None, tokens, i32([0]), i32([0]), torch.empty(need, dtype=torch.uint8, device="cuda"), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    check(cache.ssm[0, 0], s0, x, tokens, -(-tokens // 64), d)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("spread", SPREADS)
def test_tree_levels(act, spread):
    d, hv, depth = 128, 16, 12
    A = -3.0 / (depth * np.log1p(np.exp(spread[1])))
    layer, dev, s0, x = layer_and_rows(depth, hv, act, A, spread, d)
    cache, out = md.StateCache(1, 1 + depth, hv * d, d_state=d, act=DT[act]), torch.empty((depth, hv * d), dtype=DT[act], device="cuda")
    cache.ssm[0, 0] = s0
    md.mdraft_gdr_tree_step(layer, cache, 0, *dev, out, i32(np.arange(depth)), i32(np.arange(depth) + 1), list(range(depth + 1)))
    torch.cuda.synchronize()
    for n in range(depth):
        check(cache.ssm[0, 1 + n], s0, x, n + 1, n + 1, d)
