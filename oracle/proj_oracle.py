"""Plain CPU oracle (float64 numpy) of the operators between hidden states and attention: rows in
8-bit integers and their products, rotary positions, attention over a shared prefix. TEST INFRASTRUCTURE
ONLY, like the rest of ``oracle``.

Every function follows the operator's definition; nothing is shared with the kernels.
"""
from __future__ import annotations

import numpy as np

from . import cond_oracle as O


def i8_rows(x):
    """x [rows, K] (exact values of the stored type) -> (codes float64 [rows, K], scales float32 [rows])."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(1)
    top = np.abs(np.where(bad[:, None], 0.0, x)).max(1).astype(np.float32)
    s = np.maximum(top * (np.float32(1) / np.float32(127)), np.float32(2.0 ** -126))
    codes = np.rint(np.where(bad[:, None], 0.0, x) / s.astype(np.float64)[:, None])   # ties to even
    return codes, np.where(bad, np.float32(np.nan), s)


def i8_linear(a, s, b, t, bias=None, silu=False):
    """Codes a [m, k], b [n, k] with scales s [m], t [n] -> (y, z before the activation, z without bias)."""
    p = (np.asarray(a, np.float64) @ np.asarray(b, np.float64).T) * np.asarray(s, np.float64)[:, None] * \
        np.asarray(t, np.float64)[None]
    z = p if bias is None else p + np.asarray(bias, np.float64)
    with np.errstate(over="ignore"):
        return (z / (1 + np.exp(-z)) if silu else z), z, p


def rotary(x, positions, freq, interleaved=False, sections=None, factor=1.0, inverse=False):
    """x [T, H, d], positions [T] or [axes, T], freq [pairs] -> [T, H, d]."""
    x = np.array(x, np.float64)
    pairs = len(freq)
    p = np.asarray(positions, np.float64)
    axis = np.zeros(pairs, int) if sections is None else np.repeat(np.arange(len(sections)), sections)
    p = p[None] if p.ndim == 1 else p
    for i in range(pairs):
        a = p[axis[i]] * float(freq[i]) * (-1.0 if inverse else 1.0)
        c, s = np.cos(a)[:, None], np.sin(a)[:, None]
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        x1, x2 = x[..., i1].copy(), x[..., i2].copy()
        x[..., i1], x[..., i2] = factor * (x1 * c - x2 * s), factor * (x2 * c + x1 * s)
    return x


def prefix(q, pk, pv, k, v, q_lens, kv_lens, causal, scale=None):
    """Queries over the shared keys pk, pv and their sequence's own -> as cond_oracle.attend."""
    scale = 1 / np.sqrt(q.shape[2]) if scale is None else scale
    outs, s, t, P = [], 0, 0, pk.shape[0]
    for n, m in zip(q_lens, kv_lens):
        see = np.ones((n, P + m), bool)
        if causal:
            see[:, P:] = np.arange(m)[None] <= (m - n + np.arange(n))[:, None]
        kk, vv = np.concatenate([pk, k[t:t + m]]), np.concatenate([pv, v[t:t + m]])
        if n:
            outs.append(_rows(q[s:s + n], kk, vv, see, scale))
        s, t = s + n, t + m
    if not outs:
        z = np.zeros((0, q.shape[1], q.shape[2]))
        return z, z, z[..., 0]
    return tuple(np.concatenate(x) for x in zip(*outs))


def _rows(q, k, v, see, scale):
    """attend() where rows see different tokens, some of which may hold infinities or NaN: those are read by
    the rows that see them alone."""
    wild = ~(np.isfinite(k).all((1, 2)) & np.isfinite(v).all((1, 2)))
    if not wild.any():
        return O.attend(q, k, v, see, scale)
    parts = []
    for i in range(q.shape[0]):
        on = see[i]
        parts.append(O.attend(q[i:i + 1], k[on], v[on], np.ones((1, on.sum()), bool), scale))
    return tuple(np.concatenate(x) for x in zip(*parts))
