"""What pins the fp64 statement of the delta rule and the head norm (oracle/gdr.py): closed forms, other formulations, brute force."""

import numpy as np
import pytest

from oracle import gdr

rng = np.random.default_rng(11)


def layer(T, Hk=1, Hv=2, dk=8, dv=4):
    k = rng.normal(size=(T, Hk, dk))
    k /= np.linalg.norm(k, axis=-1, keepdims=True)
    return dict(q=rng.normal(size=(T, Hk * dk)), k=k.reshape(T, -1), v=rng.normal(size=(T, Hv * dv)), z=None, dt=rng.normal(size=(T, Hv)),
                beta=rng.normal(size=(T, Hv)), A=-rng.uniform(0.1, 2, size=Hv), dt_bias=rng.normal(size=Hv), norm_w=None, n_k_heads=Hk, d_k=dk, d_v=dv)


def test_full_strength_write_is_read_back():
    """beta = 1 and a unit key: right after the write the state maps the key to exactly the value, whatever it held."""
    d = layer(1)
    d.update(beta=np.ones((1, 2)), q=d["k"], dt=np.zeros((1, 2)), dt_bias=None)
    S0 = rng.normal(size=(1, 8, 8))
    out, _ = gdr.encode(**d, cu=[0, 1], S0=S0, scale=1.0, softplus=False, sigmoid=False)
    assert np.allclose(out, d["v"])


def test_orthogonal_keys_make_it_linear_attention():
    """Orthonormal keys, no decay: nothing held is ever replaced, so S = sum beta v k^T."""
    T = 6
    d = layer(T)
    kk = np.linalg.qr(rng.normal(size=(8, 8)))[0][:T]
    b = rng.uniform(0, 1, size=(T, 2))
    d.update(k=kk, beta=b, A=np.zeros(2))
    out, S = gdr.encode(**d, cu=[0, T], scale=1.0, sigmoid=False)
    v = d["v"].reshape(T, 2, 4)
    for j in range(2):
        assert np.allclose(S[0].reshape(2, 4, 8)[j], sum(b[t, j] * np.outer(v[t, j], kk[t]) for t in range(T)))


def test_chunk_form_agrees():
    """S_T and the outputs from one triangular system over the whole sequence."""
    T = 9
    d = layer(T, Hk=2, Hv=4)
    S0 = rng.normal(size=(1, 16, 8))
    out, S = gdr.encode(**d, cu=[0, T], S0=S0)
    alpha, b = gdr._gates(d["dt"], d["beta"], d["A"], d["dt_bias"], True, True)
    for j in range(4):
        q, k = (d[n].reshape(T, 2, 8)[:, j // 2] for n in ("q", "k"))
        v, s0 = d["v"].reshape(T, 4, 4)[:, j], S0[0].reshape(4, 4, 8)[j]
        G = np.cumsum(np.log(alpha[:, j]))
        D = np.tril(np.exp(G[:, None] - G[None]))
        X = np.linalg.solve(np.eye(T) + np.tril(b[:, j, None] * (k @ k.T) * D, -1), b[:, j, None] * (v - np.exp(G)[:, None] * (k @ s0.T)))
        o = 8 ** -0.5 * (np.exp(G)[:, None] * (q @ s0.T) + ((q @ k.T) * D) @ X)
        assert np.allclose(out.reshape(T, 4, 4)[:, j], o)
        assert np.allclose(S[0].reshape(4, 4, 8)[j], np.exp(G[-1]) * s0 + (np.exp(G[-1] - G)[:, None] * X).T @ k)


def test_norm_and_gate_behind_the_rule():
    d = layer(3)
    w, z = rng.normal(size=4), rng.normal(size=(3, 8))
    plain, _ = gdr.encode(**d, cu=[0, 3])
    full, _ = gdr.encode(**{**d, "norm_w": w, "z": z}, cu=[0, 3], eps=0.0)
    before, _ = gdr.encode(**{**d, "norm_w": w}, cu=[0, 3], eps=0.0)
    o = plain.reshape(3, 2, 4)
    want = (o * w / np.sqrt((o ** 2).mean(-1, keepdims=True))).reshape(3, 8)
    assert np.allclose(before, want) and np.allclose(full, want * z / (1 + np.exp(-z)))


def test_packed_sequences_are_apart_and_a_tree_path_is_a_sequence():
    d = layer(7)
    out, S = gdr.encode(**d, cu=[0, 3, 3, 7])
    sub = lambda a, b: {n: (x[a:b] if n in ("q", "k", "v", "dt", "beta") else x) for n, x in d.items()}
    o2, S2 = gdr.encode(**sub(3, 7), cu=[0, 4])
    assert np.array_equal(out[3:], o2) and np.array_equal(S[2], S2[0]) and not S[1].any()
    t_out, t_S = gdr.tree([-1, 0, 0, 2, 1], **sub(0, 5))
    path = [0, 2, 3]
    o3, S3 = gdr.encode(**{n: (x[path] if n in ("q", "k", "v", "dt", "beta") else x) for n, x in d.items()}, cu=[0, 3])
    assert np.allclose(t_out[3], o3[2]) and np.allclose(t_S[3], S3[0])


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_rotation_keeps_sizes_and_depends_on_distance_only(layout):
    f = 10000.0 ** (-np.arange(4) / 4)
    a, b = rng.normal(size=(1, 12)), rng.normal(size=(1, 12))
    turn = lambda x, p: gdr.head_norm(x, 12, positions=[p], freqs=f, layout=layout)
    assert np.allclose(np.linalg.norm(turn(a, 17)), np.linalg.norm(a)) and np.allclose(turn(a, 0), a)
    assert np.allclose(turn(a, 1017) @ turn(b, 1009).T, turn(a, 8) @ turn(b, 0).T)
    assert np.array_equal(turn(a, 5)[:, 8:], a[:, 8:]), "values behind the rotated part stay"


def test_norms():
    x = rng.normal(size=(3, 2 * 8))
    w = rng.normal(size=8)
    l2 = gdr.head_norm(x, 8, "l2", eps=0.0).reshape(3, 2, 8)
    assert np.allclose(np.linalg.norm(l2, axis=-1), 1.0)
    assert np.allclose(gdr.head_norm(x, 8, "rms", w=w, eps=0.0).reshape(3, 2, 8), l2 * np.sqrt(8) * w)


def test_the_sums_of_sizes_bound_the_outputs():
    T = 130
    d = layer(T)
    _, _, o, size, size64 = gdr.encode(**d, cu=[0, T], S0=rng.normal(size=(1, 8, 8)), sizes=True)
    assert np.all(np.abs(o) <= size * (1 + 1e-12)) and np.all(np.abs(o) <= size64 * (1 + 1e-12))
    one = gdr.encode(**{n: (x[:1] if n in ("q", "k", "v", "dt", "beta") else x) for n, x in d.items()}, cu=[0, 1], sizes=True)
    assert np.allclose(one[4], np.abs(one[2])), "a first token writes its value once: nothing to cancel"
