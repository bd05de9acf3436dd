"""Oracle of the 4-bit cache and of the operators on it.  Test infrastructure only (see the package docstring).

Format: per token, head and group of 32 features, codes 0 .. 15 with a scale s and a zero z in bf16,
    s = bf16((max - min) * (1 / 15)), 0 where that is below 2^-100;  z = bf16(min - 16 s)
    code = rint((x - z) / s) - 16, clamped to 0 .. 15 (0 where s = 0);  held: bf16(s (16 + code) + z)
after NaN -> 0 and clamping to +-2^124.  The inputs are fp32 numbers and the steps before z's and s's rounding to bf16, and the
quotient before rint, are rounded to fp32, as the definition of a code at a border; everything else is exact in fp64.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
TOP, LEAST = 2.0 ** 124, 2.0 ** -100


def bf16(x):
    """fp64 -> the nearest bf16 number (ties to even), as fp64."""
    m, e = np.frexp(np.asarray(x, np.float64))
    return np.ldexp(np.rint(m * 256.0), e - 8)


def quantise(x):
    """fp32 [.., 32 k] -> codes [.., 32 k], s and z [.., k] (fp64 that holds bf16 numbers)."""
    x = np.asarray(x, np.float32)
    x = np.clip(np.where(np.isnan(x), np.float32(0), x), np.float32(-TOP), np.float32(TOP))
    x = x.reshape(x.shape[:-1] + (-1, GROUP))
    lo, hi = x.min(-1), x.max(-1)
    s = bf16((hi - lo) * (np.float32(1) / np.float32(15)))
    s = np.where(s < LEAST, 0.0, s)
    z = bf16(lo - np.float32(16) * s.astype(np.float32))
    safe = np.where(s > 0, s, 1.0).astype(np.float32)[..., None]
    q = (x - z.astype(np.float32)[..., None]) / safe
    code = np.where(s[..., None] > 0, np.clip(np.rint(q) - 16, 0, 15), 0)
    return code.reshape(code.shape[:-2] + (-1,)).astype(np.int64), s, z


def value(code, s, z):
    c = code.reshape(code.shape[:-1] + (-1, GROUP))
    return bf16(s[..., None] * (16 + c) + z[..., None]).reshape(code.shape)


def held(x):
    """What the cache holds for fp32 features [.., 32 k], fp64."""
    return value(*quantise(x))


def paths(n, parents=None):
    """For rows 0 .. n-1: the rows on the path to each (itself last).  parents[i] = row of row i's parent (i >= 1)."""
    out = []
    for i in range(n):
        if parents is None:
            out.append(list(range(i + 1)))
        else:
            out.append([0] if i == 0 else out[int(parents[i])] + [i])
    return out


def rotate(x, pos, theta):
    """Rotary embedding of [.., dh] features at position pos, rotate-half pairing, fp64."""
    dh = x.shape[-1]
    ang = pos * theta ** (-2.0 * np.arange(dh // 2) / dh)
    c, s = np.cos(ang), np.sin(ang)
    x1, x2 = x[..., :dh // 2], x[..., dh // 2:]
    return np.concatenate([x1 * c - x2 * s, x2 * c + x1 * s], -1)


def attend(q, k, v, n_cached, see):
    """q [R, H, dh], k and v [T, Hkv, dh] (the cached tokens, then the step's rows), see[i] = the step's rows that row i sees.
    fp64 -> out [R, H, dh], and the mean distance of the values from it under the row's weights, [R, H, dh]."""
    R, H, dh = q.shape
    g = H // k.shape[1]
    out, spread = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(R):
        at = list(range(n_cached)) + [n_cached + j for j in see[i]]
        for h in range(H):
            x = k[at, h // g] @ q[i, h] / np.sqrt(dh)
            p = np.exp(x - x.max())
            p /= p.sum()
            out[i, h] = p @ v[at, h // g]
            spread[i, h] = p @ np.abs(v[at, h // g] - out[i, h])
    return out, spread
