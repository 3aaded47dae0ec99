"""fp64 statement of the gated delta rule layer and of the head norm with rotation (numpy; test infrastructure only).

Written token by token in the order of the definitions (include/mdraft.h), without chunks, tricks or shared code with the
library.  The pins are in tests/test_gdr_oracle.py.
"""

from __future__ import annotations

from typing import Optional

import numpy as np


def _f(a):
    return None if a is None else np.asarray(a, dtype=np.float64)


def silu(v):
    return v / (1.0 + np.exp(-v))


def token(S, q, k, v, alpha, beta, scale):
    """One token of one head: S (d_v, d_k) -> (o (d_v,), new S)."""
    held = S @ k
    S = alpha * S + np.outer(beta * (v - alpha * held), k)
    return scale * (S @ q), S


def _gates(dt, beta, A, dt_bias, softplus, sigmoid):
    v = _f(dt) + (0.0 if dt_bias is None else _f(dt_bias))
    delta = np.where(v > 30, v, np.log1p(np.exp(np.minimum(v, 30)))) if softplus else v
    b = 1.0 / (1.0 + np.exp(-_f(beta))) if sigmoid else _f(beta)
    return np.exp(delta * _f(A)), b


def _behind(o, z, norm_w, eps):
    if norm_w is not None:
        o = o / np.sqrt(np.mean(o * o, axis=-1, keepdims=True) + eps) * _f(norm_w)
    o = o.reshape(o.shape[0], -1)
    return o if z is None else o * silu(_f(z))


def encode(q, k, v, z, dt, beta, A, dt_bias, norm_w, n_k_heads, d_k, d_v, cu, S0=None, scale=None, eps=1e-5, softplus=True, sigmoid=True, sizes=False):
    """Packed sequences.  q, k: (T, Hk d_k); v, z: (T, Hv d_v); dt, beta: (T, Hv); S0: (n_seq, Hv d_v, d_k) or None.
    Returns (out (T, Hv d_v), final states like S0); with `sizes` also, each (T, Hv, d_v), the outputs o before norm and gate, the sums of
    the sizes of the products that make them up, scale sum |S| |q|, and the same where o is taken from the state 64 tokens' boundary ago and
    the tokens since: scale (sum |alpha.. S_boundary| |q| + sum_j |q . k_j| alpha.. |what token j wrote|)."""
    q, k, v = _f(q), _f(k), _f(v)
    T, H = v.shape[0], v.shape[1] // d_v
    scale = d_k ** -0.5 if scale is None else scale
    alpha, b = _gates(dt, beta, A, dt_bias, softplus, sigmoid)
    n = len(cu) - 1
    S = np.zeros((n, H, d_v, d_k)) if S0 is None else _f(S0).reshape(n, H, d_v, d_k).copy()
    o, size, size64 = np.zeros((T, H, d_v)), np.zeros((T, H, d_v)), np.zeros((T, H, d_v))
    for s in range(n):
        for j in range(H):
            g = slice(j // (H // n_k_heads) * d_k, (j // (H // n_k_heads) + 1) * d_k)
            for t in range(int(cu[s]), int(cu[s + 1])):
                vt = v[t, j * d_v:(j + 1) * d_v]
                if (t - int(cu[s])) % 64 == 0:
                    carried, wrote = S[s, j].copy(), []
                wrote = [alpha[t, j] * w for w in wrote] + [b[t, j] * (vt - alpha[t, j] * (S[s, j] @ k[t, g]))]
                carried = carried * alpha[t, j]
                o[t, j], S[s, j] = token(S[s, j], q[t, g], k[t, g], vt, alpha[t, j], b[t, j], scale)
                if sizes:
                    near = np.abs(k[t + 1 - len(wrote):t + 1, g] @ q[t, g])
                    size[t, j] = scale * (np.abs(S[s, j]) @ np.abs(q[t, g]))
                    size64[t, j] = scale * (np.abs(carried) @ np.abs(q[t, g]) + near @ np.abs(np.array(wrote)))
    out = _behind(o, z, norm_w, eps), S.reshape(n, H * d_v, d_k)
    return (*out, o, size, size64) if sizes else out


def tree(parents, q, k, v, z, dt, beta, A, dt_bias, norm_w, n_k_heads, d_k, d_v, S0=None, scale=None, eps=1e-5, softplus=True, sigmoid=True, sizes=False):
    """Every node from its parent's state, the roots from the committed state S0 (Hv d_v, d_k).  Returns (out (M, Hv d_v), states (M, Hv d_v,
    d_k)); with `sizes` also the outputs before norm and gate and the sums of sizes, as encode."""
    q, k, v = _f(q), _f(k), _f(v)
    M, H = v.shape[0], v.shape[1] // d_v
    scale = d_k ** -0.5 if scale is None else scale
    alpha, b = _gates(dt, beta, A, dt_bias, softplus, sigmoid)
    root = np.zeros((H, d_v, d_k)) if S0 is None else _f(S0).reshape(H, d_v, d_k)
    o, size, states = np.zeros((M, H, d_v)), np.zeros((M, H, d_v)), np.zeros((M, H, d_v, d_k))
    for m in range(M):
        before = root if parents[m] < 0 else states[parents[m]]
        for j in range(H):
            g = slice(j // (H // n_k_heads) * d_k, (j // (H // n_k_heads) + 1) * d_k)
            o[m, j], states[m, j] = token(before[j], q[m, g], k[m, g], v[m, j * d_v:(j + 1) * d_v], alpha[m, j], b[m, j], scale)
            size[m, j] = scale * (np.abs(states[m, j]) @ np.abs(q[m, g]))
    out = _behind(o, z, norm_w, eps), states.reshape(M, H * d_v, d_k)
    return (*out, o, size) if sizes else out


def head_norm(x, d_head, norm="none", w=None, eps=1e-6, positions=None, freqs=None, layout="half", rot_scale=1.0):
    """x: (rows, heads * d_head).  Rotation where freqs is given, of the first 2 len(freqs) values of every head."""
    y = _f(x).reshape(x.shape[0], -1, d_head).copy()
    if norm != "none":
        size = np.sum(y * y, axis=-1, keepdims=True) / (d_head if norm == "rms" else 1)
        y = y / np.sqrt(size + eps) * (1.0 if w is None else _f(w))
    if freqs is not None and len(freqs):
        n = len(freqs)
        for i, f in enumerate(_f(freqs)):
            a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
            t = (np.asarray(positions, dtype=np.float64) * f)[:, None]
            ya, yb = y[..., a].copy(), y[..., b].copy()
            y[..., a] = (ya * np.cos(t) - yb * np.sin(t)) * rot_scale
            y[..., b] = (yb * np.cos(t) + ya * np.sin(t)) * rot_scale
    return y.reshape(x.shape)
