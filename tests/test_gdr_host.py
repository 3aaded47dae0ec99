"""The delta layer's and the head norm's entry points turn bad arguments away before any launch (no GPU needed)."""

import ctypes as C

import pytest
import torch

INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    from paper_2506_01206_b200.build import build_library
    from paper_2506_01206_b200 import binding
    build_library()
    return binding.load_library()


def _layer(**kw):
    from paper_2506_01206_b200 import binding
    base = dict(n_k_heads=2, n_v_heads=4, d_k=128, d_v=128, act=1, flags=1 | 16, scale=0.1, eps=1e-5, A=0x1000, dt_bias=0, norm_w=0)
    base.update(kw)
    return binding._GdrLayer(*[base[n] for n in ("n_k_heads", "n_v_heads", "d_k", "d_v", "act", "flags", "scale", "eps", "A", "dt_bias", "norm_w")])


def _cache(**kw):
    from paper_2506_01206_b200 import binding
    base = dict(ssm=0x10000, ssm_layer_stride=4 * 512 * 128, ssm_slot_stride=512 * 128, conv=0, conv_layer_stride=0, conv_slot_stride=0, n_layers=1, n_slots=4)
    base.update(kw)
    return binding._Cache(*[base[k] for k in ("ssm", "ssm_layer_stride", "ssm_slot_stride", "conv", "conv_layer_stride", "conv_slot_stride", "n_layers", "n_slots")])


IO = dict(q=0x100000, ldq=256, k=0x200000, ldk=256, v=0x300000, ldv=512, z=0x400000, ldz=512, dt=0x500000, lddt=4, b=0x600000, ldb=4, out=0x700000, ldo=512)


def _io(kw):
    a = {**IO, **{n: kw.pop(n) for n in list(kw) if n in IO}}
    return [a[n] for n in ("q", "ldq", "k", "ldk", "v", "ldv", "z", "ldz", "dt", "lddt", "b", "ldb", "out", "ldo")]


def _prefill(lib, layer=None, cache=True, li=0, T=300, S=1, longest=300, cu=None, init=None, final=0x800000, ws=None, ws_bytes=0, **kw):
    layer = layer or _layer()
    c = _cache() if cache is True else cache
    io = _io(kw)
    assert not kw
    return lib.mdraft_gdr_prefill(C.byref(layer), C.byref(c) if c is not None else None, li, *io, T, S, longest, cu, init, final, ws, ws_bytes, None, None)


def _step(lib, layer=None, cache=True, n=3, par=0x900000, nod=0xA00000, n_levels=1, levels=None, **kw):
    layer = layer or _layer()
    c = _cache() if cache is True else cache
    io = _io(kw)
    assert not kw
    return lib.mdraft_gdr_tree_step(C.byref(layer), C.byref(c) if c is not None else None, 0, *io, n, par, nod, n_levels, levels, None, None)


@pytest.mark.parametrize("kw,status", [
    (dict(d_k=96), UNSUPPORTED), (dict(d_v=32), UNSUPPORTED), (dict(act=2), UNSUPPORTED), (dict(n_k_heads=3), UNSUPPORTED), (dict(n_v_heads=0), INVALID),
    (dict(n_k_heads=-1), INVALID), (dict(A=0), INVALID), (dict(flags=2), INVALID), (dict(flags=8), INVALID), (dict(n_v_heads=8192), UNSUPPORTED)])
def test_layers_that_are_refused(lib, kw, status):
    assert _prefill(lib, _layer(**kw)) == status
    assert _step(lib, _layer(**kw)) == status
    assert lib.mdraft_gdr_prefill_workspace_bytes(C.byref(_layer(**kw)), 300, 1, 300) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID), (dict(dt=None), INVALID), (dict(b=None), INVALID),
    (dict(ldq=248), INVALID), (dict(ldv=504), INVALID), (dict(ldz=256), INVALID), (dict(lddt=3), INVALID), (dict(ldb=3), INVALID),
    (dict(k=0x200008), MISALIGNED), (dict(ldk=260), MISALIGNED), (dict(z=0x400002), MISALIGNED), (dict(ldo=513), MISALIGNED)])
def test_activations_that_are_refused(lib, kw, status):
    assert _prefill(lib, **kw) == status
    assert _step(lib, **kw) == status


def test_encode_calls_that_are_refused(lib):
    assert _prefill(lib, T=-1) == INVALID and _prefill(lib, S=-1) == INVALID and _prefill(lib, longest=-1) == INVALID
    assert _prefill(lib, S=2) == INVALID                                  # offsets may be left out for one sequence only
    assert _prefill(lib, cache=None) == INVALID                           # a slot is named but there is no pool
    assert _prefill(lib, li=1) == INVALID
    assert _prefill(lib, cache=_cache(ssm_slot_stride=511 * 128)) == INVALID
    assert _prefill(lib, cache=_cache(ssm_slot_stride=512 * 128 + 2)) == MISALIGNED
    assert _prefill(lib, S=0, T=0) == 0


def test_step_calls_that_are_refused(lib):
    assert _step(lib, cache=None) == INVALID and _step(lib, par=None) == INVALID and _step(lib, nod=None) == INVALID and _step(lib, n=-1) == INVALID
    assert _step(lib, n_levels=2) == INVALID
    assert _step(lib, n_levels=2, levels=(C.c_int32 * 3)(0, 2, 4)) == INVALID
    assert _step(lib, n_levels=2, levels=(C.c_int32 * 3)(0, 4, 3)) == INVALID
    assert _step(lib, n=0) == 0


def test_commit_calls_that_are_refused(lib):
    def commit(cache=None, d=512, n=128, ch=1024, w=4, act=1, m=1, src=0x1000, dst=0x2000):
        c = cache or _cache(conv=0x40000, conv_slot_stride=3 * 1024, conv_layer_stride=12 * 1024)
        return lib.mdraft_gdr_state_commit(C.byref(c), d, n, ch, w, act, m, src, dst, None, None)
    assert commit(n=16) == UNSUPPORTED and commit(w=3) == UNSUPPORTED and commit(ch=1023) == UNSUPPORTED and commit(act=5) == UNSUPPORTED
    assert commit(d=0) == INVALID and commit(ch=-8) == INVALID and commit(ch=1032) == INVALID and commit(m=-1) == INVALID and commit(src=None) == INVALID
    assert commit(cache=_cache(), ch=1024) == INVALID                     # windows are named but the pool has none
    assert commit(m=0) == 0 and commit(cache=_cache(), ch=0, m=0) == 0


def _spec(**kw):
    from paper_2506_01206_b200 import binding
    base = dict(d_head=64, n_q_heads=4, n_k_heads=2, act=1, norm=2, rot_dim=32, rot_layout=0, eps=1e-6, rot_scale=1.0, q_w=0, k_w=0, freqs=0x9000)
    base.update(kw)
    return binding._QkNormSpec(*[base[n] for n in ("d_head", "n_q_heads", "n_k_heads", "act", "norm", "rot_dim", "rot_layout", "eps", "rot_scale", "q_w", "k_w", "freqs")])


def _norm(lib, spec=None, q=0x100000, ldq=256, k=0x200000, ldk=128, qo=0x300000, ldqo=256, ko=0x400000, ldko=128, pos=0x500000, n=5):
    s = spec or _spec()
    return lib.mdraft_qk_norm(C.byref(s), q, ldq, k, ldk, qo, ldqo, ko, ldko, pos, n, None)


@pytest.mark.parametrize("kw,status", [
    (dict(d_head=60), UNSUPPORTED), (dict(d_head=264), UNSUPPORTED), (dict(d_head=0), UNSUPPORTED), (dict(act=3), UNSUPPORTED), (dict(rot_dim=72), UNSUPPORTED),
    (dict(rot_dim=24), UNSUPPORTED), (dict(rot_dim=7, rot_layout=1), UNSUPPORTED), (dict(rot_dim=-2), INVALID), (dict(norm=3), INVALID),
    (dict(rot_layout=2), INVALID), (dict(freqs=0), INVALID), (dict(q_w=0x1008), MISALIGNED), (dict(n_q_heads=-1), INVALID)])
def test_norm_specs_that_are_refused(lib, kw, status):
    assert _norm(lib, _spec(**kw)) == status


def test_norm_calls_that_are_refused(lib):
    assert _norm(lib, q=None) == INVALID and _norm(lib, ko=None) == INVALID and _norm(lib, pos=None) == INVALID and _norm(lib, n=-1) == INVALID
    assert _norm(lib, ldq=248) == INVALID and _norm(lib, ldk=132) == MISALIGNED and _norm(lib, qo=0x300008) == MISALIGNED
    assert _norm(lib, n=0) == 0 and _norm(lib, _spec(n_q_heads=0, n_k_heads=0)) == 0


def test_tensors_that_are_refused(lib):
    """The extension looks at types, shapes and devices; tensors of the host never reach the library."""
    import paper_2506_01206_b200 as md
    e = md.binding._entry()
    spec = type("Spec", (), dict(d_head=64, n_q_heads=1, n_k_heads=1, act=torch.bfloat16, norm=1, rot_dim=0, rot_layout=0, eps=1e-6, rot_scale=1.0,
                                 q_w=None, k_w=None, freqs=None))()
    x = torch.zeros((3, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA tensor"):
        md.binding._host.qk_norm(e, spec, x, x, x, x, None, 0)
    with pytest.raises(TypeError, match="q: must be a tensor"):
        md.binding._host.qk_norm(e, spec, None, x, x, x, None, 0)
    with pytest.raises(ValueError, match="float32 CUDA tensor"):
        md.GdrLayer(torch.zeros(4), None, None, 2)
    with pytest.raises(ValueError, match="float32 CUDA tensor"):
        md.QkNorm(64, 1, 1, rot_dim=32, freqs=torch.zeros(16))


@pytest.mark.parametrize("name,count", [("gdr_prefill", 19), ("gdr_tree_step", 17), ("gdr_commit", 6), ("qk_norm", 8)])
def test_the_extension_checks_how_many_arguments_it_is_given(lib, name, count):
    from paper_2506_01206_b200 import binding
    f = getattr(binding._host, name)
    for n in (0, count - 1, count + 1):
        with pytest.raises(TypeError, match=f"expected {count} arguments, got {n}"):
            f(*[None] * n)


def test_more_rows_than_the_norm_counts_are_refused(lib):
    s = _spec(rot_dim=0)
    assert _norm(lib, s, n=2 ** 31 - 1) == UNSUPPORTED and _norm(lib, s, n=2 ** 31 - 4096) == UNSUPPORTED


def test_a_commit_takes_any_cache_that_has_a_pools_attributes(monkeypatch):
    """mdraft_state_commit reads the attributes of a pool and no more: one without `conv_channels` has windows as wide as its states, and goes the ordinary way."""
    import types

    import paper_2506_01206_b200 as md
    from paper_2506_01206_b200 import binding
    calls = []
    fake = types.SimpleNamespace(commit=lambda *a: calls.append("ordinary") or 0, gdr_commit=lambda *a: calls.append("delta") or 0)
    monkeypatch.setattr(binding, "_host", fake)
    monkeypatch.setattr(binding, "_entry", lambda: None)
    pool = lambda **kw: types.SimpleNamespace(**{**dict(d_inner=512, d_state=16, d_conv=4, act=torch.bfloat16, n_layers=1, n_slots=4), **kw})
    for cache, way in ((pool(), "ordinary"), (pool(d_state=128), "ordinary"), (pool(d_state=64), "ordinary"), (pool(conv_channels=512), "ordinary"),
                       (pool(d_state=128, conv_channels=1024), "delta"), (pool(d_state=64, conv_channels=512), "delta"), (None, "ordinary")):
        calls.clear()
        md.mdraft_state_commit(cache, None, None)
        assert calls == [way]
