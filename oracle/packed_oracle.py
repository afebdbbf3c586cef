"""float64 NumPy oracle of the operators beside the paper's: the cache of 4 bits a value, attention over it, and the norm and
rotation of query and key heads.  Written from the definitions in include/sdllm.h alone."""
from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALVES, ADJACENT = 0, 1


def group_codes(x):
    """(e, codes) of groups of 32 along the last axis; e is None-like (255 - 127) where the group is not finite."""
    x = np.asarray(x, np.float64)
    finite = np.isfinite(x).all(-1)
    top = np.where(finite, np.abs(np.where(np.isfinite(x), x, 0)).max(-1), 0.0)
    e = np.full(top.shape, -125)
    for step in range(-125, 125):                 # the smallest that fits
        e = np.where(top >= 7 * 2.0 ** step, step + 1, e)
    a = np.where(finite[..., None], np.abs(x) / 2.0 ** e[..., None].astype(float), 0.0)
    away = np.abs(a[..., None] - MAGNITUDES)
    away = away + np.where(np.arange(8) % 2 == 1, 1e-300, 0)   # a tie goes to the even code
    code = np.zeros(a.shape, int)
    best = away[..., 0]
    for c in (2, 4, 6, 1, 3, 5, 7):
        nearer = away[..., c] < best
        code, best = np.where(nearer, c, code), np.where(nearer, away[..., c], best)
    code = code + 8 * (np.signbit(x) & finite[..., None])
    return np.where(finite, e, 128), code


def group_values(x):
    """What groups of 32 along the last axis read as."""
    e, code = group_codes(x)
    y = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7] * 2.0 ** np.where(e == 128, 0, e)[..., None].astype(float)
    return np.where((e == 128)[..., None], np.nan, y)


def cache_values(k, v):
    """Rows [.., n, d] of keys and values as the cache holds them."""
    *lead, n, d = np.shape(k)
    kv = group_values(np.reshape(k, (*lead, n, d // 32, 32))).reshape(*lead, n, d)
    pad = -n % 32
    w = np.concatenate([np.asarray(v, np.float64), np.zeros((*lead, pad, d))], -2)
    w = np.swapaxes(w.reshape(*lead, (n + pad) // 32, 32, d), -1, -2)
    return kv, np.swapaxes(group_values(w), -1, -2).reshape(*lead, n + pad, d)[..., :n, :]


def cache_bytes(k, v):
    """One (batch, KV head): the tiles [ceil(n / 32), 34 d] of rows [n, d], byte for byte."""
    n, d = np.shape(k)
    tiles = -(-n // 32)
    out = np.zeros((tiles, 34 * d), np.uint8)
    for t in range(tiles):
        kt, vt = np.zeros((32, d)), np.zeros((32, d))
        m = min(32, n - 32 * t)
        kt[:m], vt[:m] = k[32 * t:32 * t + m], v[32 * t:32 * t + m]
        e, code = group_codes(kt.reshape(32, d // 32, 32))
        for r in range(32):
            for g in range(d // 32):
                out[t, 32 * d + r * (d // 32) + g] = e[r, g] + 127
                for c in range(32):
                    out[t, (g * 32 + r) * 16 + c // 2] |= code[r, g, c] << 4 * (c % 2)
        e, code = group_codes(vt.T)
        for ch in range(d):
            out[t, 33 * d + ch] = e[ch] + 127
            mm, rest = divmod(ch, d // 32)
            i, j = divmod(rest, 2)
            for r in range(32):
                a, h, p = r // 8, r // 4 % 2, r % 4
                nib = 4 * a + p
                out[t, 16 * d + ((i * 2 + h) * 32 + mm) * 16 + 8 * j + nib // 2] |= code[ch, r] << 4 * (nib % 2)
    return out


def attention(q, k, v, scale):
    """(out, mean): softmax(scale q k^T) v of rows [n, d], and the same over |v| (what errors of the probabilities are measured in)."""
    with np.errstate(invalid="ignore"):
        a = scale * (q @ k.T)
        p = np.exp(a - a.max(-1, keepdims=True))
        p = p / p.sum(-1, keepdims=True)
        return p @ v, p @ np.abs(v)


def norm_rope(x, weight, inv_freq, positions, *, rot, pairing, norm, eps):
    """[.., n, d] at positions [.., n]."""
    x = np.array(x, np.float64)
    d = x.shape[-1]
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    f = np.arange(rot // 2)
    a, b = (f, f + rot // 2) if pairing == HALVES else (2 * f, 2 * f + 1)
    t = np.asarray(positions, np.float64)[..., None] * np.asarray(inv_freq, np.float64)
    y = x.copy()
    y[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
    y[..., b] = x[..., a] * np.sin(t) + x[..., b] * np.cos(t)
    assert y.shape[-1] == d
    return y
