"""The give-up paths of the delta layer's chunked encode, with the library of test_gpu_wait_expiry (short limits, copies that are told to be larger than
they are): the calls return, flag it, write neither outputs nor states and free their tensor memory; the ordinary library is right afterwards."""

import pytest
import torch

from oracle import gdr
from test_gpu_gdr import Problem, check_states
from test_gpu_wait_expiry import using, waitlib  # noqa: F401

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md
from paper_2506_01206_b200.device_inputs import i32


@pytest.mark.parametrize("hv,norm,gate", [(2, False, True), (38, False, True), (38, True, True), (38, True, False)])
def test_encode_wait_runs_out_and_the_call_returns(waitlib, hv, norm, gate):  # noqa: F811
    n = 300
    p = Problem(n, 1, hv, gate=gate, norm=norm, seed=50)
    cache, status, ws = p.cache(1), torch.zeros(1, dtype=torch.int32, device="cuda"), p.workspace(1, n)
    cache.ssm.fill_(3.0)
    out = torch.full((n, hv * 128), 7.0, dtype=torch.bfloat16, device="cuda")
    call = lambda: md.mdraft_gdr_prefill(p.layer, cache, 0, *p.dev, out, None, n, None, i32([0]), ws, status)
    with using(waitlib):
        for _ in range(10):   # more failing blocks than an SM has tensor-memory columns for, if any were leaked
            call()
        torch.cuda.synchronize()
    assert int(status.item()) == md.MDRAFT_DEV_WAIT_EXPIRED
    assert bool((out == 7.0).all()) and bool((cache.ssm == 3.0).all())
    status.zero_()
    call()
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    w_out, w_states, o, size, size64 = gdr.encode(**p.args(), cu=[0, n], sizes=True)
    check_states(cache.ssm[0], w_states)
    p.check_out(out, w_out, o, size, size64)
