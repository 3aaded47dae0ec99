"""The delta layer's chunked encode with warps held up for 50 microseconds where their being late has to be harmless (``libmdraft_holdtest.so``, the same
sources): far longer than the products and copies that run meanwhile, so a read or an allocation that only timing puts in order gives other results or an
error status.  Both libraries do the same arithmetic in the same order, so results are compared bit for bit."""

import numpy as np
import pytest
import torch

from test_gpu_gdr import Problem, is_chunked
from test_gpu_wait_expiry import using

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md
from paper_2506_01206_b200 import binding
from paper_2506_01206_b200.build import build_library
from paper_2506_01206_b200.device_inputs import i32


@pytest.fixture(scope="module")
def heldlib():
    return binding.load_library(build_library(variant="holdtest"))


def encode(p, lens):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cache, out, status = p.cache(len(lens)), p.out(), torch.zeros(1, dtype=torch.int32, device="cuda")
    md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, i32(cu), max(lens), None, i32(np.arange(len(lens))), p.workspace(len(lens), max(lens)), status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return out, cache.ssm


# heads that make single sequences wide, and few heads, which are narrow
@pytest.mark.parametrize("hk,hv,dk,dv", [(38, 38, 128, 128), (13, 39, 64, 128), (5, 80, 128, 64), (76, 76, 64, 64), (1, 2, 128, 128)])
def test_a_late_warp_of_the_chain_reads_its_own_chunk(heldlib, hk, hv, dk, dv):
    """Eight chunks whose decays differ widely: the state scaled by another chunk's would be off by factors."""
    p = Problem(500, hk, hv, dk, dv, seed=80)
    p.np["dt"][:] = np.repeat(np.tile([-2.0, 2.0], 4), 64)[:500, None]
    p.upload()
    assert is_chunked(p, [500])
    want = encode(p, [500])
    with using(heldlib):
        got = encode(p, [500])
    assert torch.equal(got[1], want[1]) and torch.equal(got[0].view(torch.int16), want[0].view(torch.int16))


@pytest.mark.parametrize("hk,hv,dk,dv", [(1, 2, 64, 64), (1, 1, 128, 64), (1, 1, 128, 128)])
def test_a_block_late_with_its_tensor_memory_is_not_shut_out(heldlib, hk, hv, dk, dv):
    """Many short sequences, so that blocks of the chain are ready long before the last chunk's block of the kernel ahead has looked up what it works on: they
    do not start, and take the SMs' tensor memory, before that one has its own."""
    lens = list(np.random.default_rng(3).integers(1, 71, 1500))
    p = Problem(int(sum(lens)), hk, hv, dk, dv, seed=81)
    assert is_chunked(p, lens)
    want = encode(p, lens)
    with using(heldlib):
        got = encode(p, lens)
    assert torch.equal(got[1], want[1]) and torch.equal(got[0].view(torch.int16), want[0].view(torch.int16))


@pytest.mark.parametrize("n", [2, 19, 512])
def test_sequences_taken_by_length_keep_their_rows_and_slots(n):
    """Lengths in an order unlike their ranks, equal ones among them: every sequence equals the same sequence in a call that does not rank (one of 600)."""
    lens = [int(v) for v in np.random.default_rng(n).choice([1, 40, 64, 70, 129, 130], n)]
    lens[0], lens[-1] = 40, 130
    hv = 152 // n + 1 if n < 38 else 2
    p = Problem(sum(lens), 1, hv, 64, 128, seed=82)
    assert is_chunked(p, lens)
    want = encode(p, lens)
    more = lens + [0] * (600 - n)
    got = encode(p, more)
    assert torch.equal(got[1][:, :n], want[1]) and torch.equal(got[0].view(torch.int16), want[0].view(torch.int16))
