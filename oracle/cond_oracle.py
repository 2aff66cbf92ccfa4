"""Plain CPU oracle (float64 numpy) of the operators that read the conditioning: cross attention,
the 8-bit key/value cache, group norm with an activation. TEST INFRASTRUCTURE ONLY, like
the rest of ``oracle``.

Every function follows the operator's definition row by row; nothing is shared with the
kernels' data layouts but ``V_ORDER``, the documented order of a block's tokens in the value
codes.
"""
from __future__ import annotations

import numpy as np

from . import e4m3 as Q

BLOCK = 32
# place 16 h + 8 t + 4 a + i holds token 16 t + 8 a + 4 h + i
V_ORDER = [16 * t + 8 * a + 4 * h + i for h in range(2) for t in range(2) for a in range(2) for i in range(4)]


def attend(q, k, v, see, scale):
    """q [n, Hq, d], k / v [m, Hkv, d], see bool [n, m] -> (out [n, Hq, d], the sum of p |v| [n, Hq, d],
    the largest scale * sum |q| |k| of each row [n, Hq]): the last two bound rounding errors. Rows
    that see nothing are zero."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, hq, d = q.shape
    rep = hq // k.shape[1]
    out, mag, reach = np.zeros((n, hq, d)), np.zeros((n, hq, d)), np.zeros((n, hq))
    if k.shape[0] == 0:
        return out, mag, reach
    for h in range(hq):
        g = h // rep
        kk, vv = k[:, g], v[:, g]
        used = see.any(0)
        kk, vv = np.where(used[:, None], kk, 0.0), np.where(used[:, None], vv, 0.0)   # nobody's tokens: not read
        s = np.where(see, scale * (q[:, h] @ kk.T), -np.inf)
        top = s.max(1, keepdims=True)
        live = np.isfinite(top)
        p = np.where(see, np.exp(s - np.where(live, top, 0.0)), 0.0)
        tot = p.sum(1, keepdims=True)
        p = p / np.where(tot > 0, tot, 1.0)
        out[:, h], mag[:, h] = p @ vv, p @ np.abs(vv)
        reach[:, h] = (scale * (np.abs(q[:, h]) @ np.abs(kk).T) * see).max(1)
    return out, mag, reach


def cross(q, k, v, q_lens, kv_lens, kv_index=None, key_mask=None, scale=None):
    """Packed cross attention -> (out, mag, reach) as `attend` gives them, packed."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    scale = 1 / np.sqrt(q.shape[2]) if scale is None else scale
    starts = np.concatenate([[0], np.cumsum(kv_lens)]).astype(int)
    parts, at = [], 0
    for i, n in enumerate(q_lens):
        j = i if kv_index is None else kv_index[i]
        a, b = starts[j], starts[j + 1]
        m = np.ones(b - a, bool) if key_mask is None else np.asarray(key_mask[a:b]) != 0
        parts.append(attend(q[at:at + n], k[a:b], v[a:b], np.broadcast_to(m, (n, b - a)), scale))
        at += n
    return tuple(np.concatenate([p[x] for p in parts]) for x in range(3))


def scale_exponent(amax: float) -> int:
    """Smallest e >= -126 with amax <= 448 * 2^e."""
    return -126 if amax == 0 else max(Q.row_scale_exponent(float(amax)), -126)


class Cache:
    """One sequence and tensor of the 8-bit cache: values [tokens, H, d], scales per block and head."""

    def __init__(self, heads: int, d: int):
        self.codes = np.zeros((0, heads, d), np.uint8)
        self.exps = np.zeros((0, heads), int)

    def append(self, rows):
        rows = np.asarray(rows, np.float64)
        old, n = self.codes.shape[0], rows.shape[0]
        if n == 0:
            return
        heads = rows.shape[1]
        blocks = (old + n + BLOCK - 1) // BLOCK
        exps = np.full((blocks, heads), -126)
        exps[:self.exps.shape[0]] = self.exps
        codes = np.concatenate([self.codes, np.zeros((n, *rows.shape[1:]), np.uint8)])
        for b in range(old // BLOCK, blocks):
            lo, hi = b * BLOCK, min((b + 1) * BLOCK, old + n)
            first = max(lo, old)
            for h in range(heads):
                x = rows[first - old:hi - old, h]
                fin = np.where(np.isfinite(x), np.abs(x), 0.0)
                e = 120 if np.isinf(x).any() else scale_exponent(fin.max())
                if first > lo:
                    e = max(e, exps[b, h])
                    kept = Q.decode_table()[codes[lo:first, h].astype(int)] * 2.0 ** (int(exps[b, h]) - e)
                    codes[lo:first, h] = np.where(np.isnan(kept), 0x7F, Q.encode(np.nan_to_num(kept)))
                y = np.clip(np.where(np.isnan(x), 0.0, x) / 2.0 ** e, *((-240, 240) if e == 120 else (-448, 448)))   # 256 * 2^120 is beyond fp32
                codes[first:hi, h] = np.where(np.isnan(x), 0x7F, Q.encode(y))
                exps[b, h] = e
        self.codes, self.exps = codes, exps

    def values(self):
        s = 2.0 ** np.repeat(self.exps, BLOCK, 0)[:self.codes.shape[0]].astype(np.float64)
        return Q.decode_table()[self.codes.astype(int)] * s[:, :, None]


def block_values(k_codes, v_codes, scales):
    """Blocks of a cache as the format lays them out -> keys, values [blocks, 32, H, d] float64."""
    lut = Q.decode_table()
    nb, h, d, _ = v_codes.shape
    k = lut[k_codes.astype(int)].transpose(0, 3, 1, 2, 4).reshape(nb, BLOCK, h, d)
    v = np.empty((nb, BLOCK, h, d))
    for place, tok in enumerate(V_ORDER):
        v[:, tok] = lut[v_codes[..., place].astype(int)]
    s = scales.astype(np.float64)[:, None, :, :, None]
    return k * s[..., 0, :], v * s[..., 1, :]


def group_norm(x, groups, gamma=None, beta=None, eps=1e-5, silu=False):
    """x [N, P, C] -> (y, z before the activation, 1 / sqrt(var + eps) per channel [N, 1, C],
    mean |x| per channel [N, 1, C])."""
    x = np.asarray(x, np.float64)
    n, p, c = x.shape
    z = x.reshape(n, p, groups, c // groups)
    mean = z.mean((1, 3), keepdims=True)
    var = ((z - mean) ** 2).mean((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    y = ((z - mean) * rstd).reshape(n, p, c)
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    wide = lambda t: np.broadcast_to(t, (n, 1, groups, c // groups)).reshape(n, 1, c)
    out = y / (1 + np.exp(-y)) if silu else y
    return out, y, wide(rstd), wide(np.abs(z).mean((1, 3), keepdims=True))
