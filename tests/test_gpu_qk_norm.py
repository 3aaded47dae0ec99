"""mdraft_qk_norm against the fp64 statement.

Tolerances.  Arithmetic is fp32 and rounded once.  A sum of squares of at most 256 values by fused multiply-adds and shuffles is off by at most
(32 + 5 + 1) 2^-24, its root's reciprocal by half that and 2 ulp of the instruction, the two products by 2^-24 each: 25 * 2^-24.
The rotation adds an absolute error of 4 * 2^-24 (sine and cosine good to 2 ulp of 1, a turn good to 2^-25 of a turn, which is 2 pi
2^-25 < 4 * 2^-24 radians) times the pair's size, and three roundings.  So |error| <= 40 * 2^-24 * (size of the value or its pair) plus, for bf16, half a
step of the result: 2^-8.
"""

import numpy as np
import pytest
import torch

from oracle import gdr

pytestmark = pytest.mark.gpu

import paper_2506_01206_b200 as md

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
NORM = {"none": md.MDRAFT_NORM_NONE, "l2": md.MDRAFT_NORM_L2, "rms": md.MDRAFT_NORM_RMS}
LAYOUT = {"half": md.MDRAFT_ROT_HALF, "pairs": md.MDRAFT_ROT_PAIRS}


def bound(want, d, rot, layout, act):
    """Per value: 40 * 2^-24 of the larger of the value and its pair's size, and half a step of the result's type."""
    y = np.abs(want).reshape(want.shape[0], -1, d)
    size = y.copy()
    if rot:
        a, b = (np.s_[..., :rot // 2], np.s_[..., rot // 2:rot]) if layout == "half" else (np.s_[..., 0:rot:2], np.s_[..., 1:rot:2])
        size[a] = size[b] = np.hypot(y[a], y[b])
    return (40 * 2.0 ** -24 * size + (2.0 ** -8 * y if act == "bf16" else 0.0)).reshape(want.shape)


def check(got, want, d, rot, layout, act):
    e = np.abs(got.double().cpu().numpy() - want) - bound(want, d, rot, layout, act)
    assert np.all(e <= 1e-37), float(e.max())


def run(rows, hq, hk, d, act="bf16", norm="rms", weights=True, rot=0, layout="half", positions=None, eps=1e-6, rot_scale=1.0, x=None, seed=0, in_place=False):
    g = torch.Generator().manual_seed(seed)
    u = (torch.randn((rows, (hq + hk) * d + 24), generator=g) * 3).to(DT[act]) if x is None else x
    u = u.cuda()
    q, k = u[:, :hq * d], u[:, hq * d:(hq + hk) * d]
    w = [torch.rand(d, generator=g) + 0.5 if weights else None for _ in range(2)]
    freqs = torch.from_numpy(10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)).float() if rot else None
    pos = torch.arange(rows) * 3 + 1 if positions is None else torch.as_tensor(positions)
    dev = lambda t: None if t is None else t.cuda()
    spec = md.QkNorm(d, hq, hk, DT[act], NORM[norm], dev(w[0]), dev(w[1]), eps, rot, LAYOUT[layout], dev(freqs), rot_scale)
    want = [gdr.head_norm(t.double().cpu().numpy(), d, norm, None if w_ is None else w_.double().numpy(), eps, pos.numpy(), None if freqs is None else freqs.double().numpy(),
                          layout, rot_scale) for t, w_ in ((q, w[0]), (k, w[1]))]
    if in_place:
        qo, ko = q, k
        rest = u[:, (hq + hk) * d:].clone()
    else:
        o = torch.full((rows + 1, (hq + hk) * d + 8), float("nan"), dtype=DT[act], device="cuda")
        qo, ko = o[:rows, :hq * d], o[:rows, hq * d:(hq + hk) * d]
    md.mdraft_qk_norm(spec, q if hq else None, k if hk else None, qo if hq else None, ko if hk else None, pos.to(torch.int32).cuda())
    torch.cuda.synchronize()
    check(qo, want[0], d, rot, layout, act)
    check(ko, want[1], d, rot, layout, act)
    if in_place:
        assert torch.equal(u[:, (hq + hk) * d:], rest)
    else:
        assert bool(o[rows].isnan().all()) and bool(o[:, (hq + hk) * d:].isnan().all()), "nothing beside the heads is written"


@pytest.mark.parametrize("act", ["f32", "bf16"])
@pytest.mark.parametrize("norm", ["none", "l2", "rms"])
@pytest.mark.parametrize("rows,hq,hk,d,rot,layout", [
    (1, 1, 1, 8, 0, "half"), (1, 12, 12, 128, 128, "half"), (18, 12, 4, 128, 64, "pairs"), (77, 6, 3, 96, 48, "half"), (5, 3, 1, 80, 80, "pairs"),
    (1000, 2, 2, 64, 32, "half"), (3, 40, 20, 256, 256, "half"), (33, 5, 1, 32, 2, "pairs"), (700, 0, 3, 24, 16, "half"), (9, 7, 0, 192, 190, "pairs")])
def test_matches_the_statement(act, norm, rows, hq, hk, d, rot, layout):
    run(rows, hq, hk, d, act, norm, weights=rows % 2 == 1, rot=rot, layout=layout)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_far_and_negative_positions(layout):
    pos = [0, 1, -1, 4095, 1 << 20, 10000019, -(1 << 30), (1 << 31) - 1, -(1 << 31)]
    run(len(pos), 2, 1, 64, "f32", "none", rot=64, layout=layout, positions=pos, rot_scale=1.25)


def test_in_place():
    run(50, 3, 2, 128, "bf16", "l2", rot=128, in_place=True)


def test_rows_of_zeros_tiny_and_huge_values():
    """A row of zeros stays zero under a positive eps; fp32 squares neither lose bf16's tiny values in eps nor overflow at 1e15."""
    x = torch.zeros((4, 2 * 64 + 24), dtype=torch.bfloat16)
    x[1] = 1e-20
    x[2, ::2] = 1e15
    x[3, 5] = -7.0
    run(4, 1, 1, 64, "bf16", "l2", weights=False, x=x, rot=32)


def test_a_row_with_nan_or_infinity_stays_alone():
    x = torch.randn((6, 2 * 64 + 24)).bfloat16()
    x[2, 3], x[4, 70] = float("nan"), float("inf")
    u = x.cuda()
    o = torch.empty_like(u)
    spec = md.QkNorm(64, 1, 1, norm=md.MDRAFT_NORM_RMS)
    md.mdraft_qk_norm(spec, u[:, :64], u[:, 64:128], o[:, :64], o[:, 64:128])
    bad = (~o[:, :128].isfinite()).view(6, 2, 64)
    assert bool(bad[2, 0].all()) and bool(bad[4, 1].any()) and int(bad.any(-1).sum()) == 2


def test_on_another_stream_and_replayed_from_a_graph():
    g = torch.Generator(device="cuda").manual_seed(3)
    u = torch.randn((300, 3 * 128), device="cuda", generator=g).bfloat16()
    f = torch.rand(32, device="cuda")
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    spec = md.QkNorm(128, 2, 1, norm=md.MDRAFT_NORM_RMS, rot_dim=64, freqs=f)
    outs = [torch.zeros_like(u) for _ in range(3)]
    call = lambda o, **kw: md.mdraft_qk_norm(spec, u[:, :256], u[:, 256:], o[:, :256], o[:, 256:], pos, **kw)
    call(outs[0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    call(outs[1], stream=s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[2])
    outs[2].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_refusals():
    x = torch.zeros((4, 128), device="cuda", dtype=torch.bfloat16)
    spec = md.QkNorm(64, 2, 2)
    with pytest.raises(ValueError):
        md.mdraft_qk_norm(spec, x, x[:3], x, x)
    with pytest.raises(ValueError):
        md.mdraft_qk_norm(spec, x[:, :64], x, x, x)
    with pytest.raises(TypeError):
        md.mdraft_qk_norm(spec, x.float(), x, x, x)
    with pytest.raises(md.MdraftError):
        md.mdraft_qk_norm(md.QkNorm(64, 2, 2, rot_dim=24, freqs=torch.zeros(12, device="cuda")), x, x, x, x, torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(md.MdraftError):
        md.mdraft_qk_norm(md.QkNorm(64, 2, 2, rot_dim=32, freqs=torch.zeros(16, device="cuda")), x, x, x, x)   # no positions
    with pytest.raises(TypeError):
        md.mdraft_qk_norm(md.QkNorm(64, 2, 2, rot_dim=32, freqs=torch.zeros(16, device="cuda")), x, x, x, x, torch.zeros(4, dtype=torch.int64, device="cuda"))
