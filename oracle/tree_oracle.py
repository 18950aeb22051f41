"""fp64 oracle of serving drafted trees: rotary positions, rows held in 8 bits, attention of a tree over a cache, the commit of
a branch.  Plain numpy from the definitions, one sequence, head and token at a time; shares nothing with the library."""
from __future__ import annotations

import math

import numpy as np

TOP = {"int8": 127.0, "fp8": 448.0}


def frequencies(base, rot_dim, scaling="none", by=1.0, context=0.0, low=1.0, high=4.0):
    """(radians a position of every pair, factor of cos and sin)"""
    theta, factor = [], 1.0
    if scaling == "base":
        base = base * by ** (rot_dim / (rot_dim - 2.0))
    pair_that_turns = lambda times: rot_dim * math.log(context / (times * 2 * math.pi)) / (2 * math.log(base))
    if scaling == "ramp":
        first = max(0, math.floor(pair_that_turns(high)))
        last = min(rot_dim - 1, math.ceil(pair_that_turns(low)))
        factor = 0.1 * math.log(by) + 1.0
    for i in range(rot_dim // 2):
        t = base ** (-2.0 * i / rot_dim)
        if scaling == "linear":
            t /= by
        elif scaling in ("bands", "ramp"):
            if scaling == "bands":
                keep = (context * t / (2 * math.pi) - low) / (high - low)
            else:
                keep = 1.0 - (i - first) / max(1e-3, last - first)
            keep = min(1.0, max(0.0, keep))
            t = keep * t + (1.0 - keep) * t / by
        theta.append(t)
    return np.array(theta), factor


def rotate(x, positions, theta, style, factor=1.0):
    """x [..., dh] with positions [...] (broadcast against its leading axes): the first 2 len(theta) elements turn."""
    y = np.array(x, np.float64)
    r = 2 * len(theta)
    a = np.asarray(positions, np.float64)[..., None] * theta
    c, s = factor * np.cos(a), factor * np.sin(a)
    for i in range(r // 2):
        j, k = (i, i + r // 2) if style == "half" else (2 * i, 2 * i + 1)
        u, v = np.array(x[..., j], np.float64), np.array(x[..., k], np.float64)
        y[..., j] = u * c[..., i] - v * s[..., i]
        y[..., k] = v * c[..., i] + u * s[..., i]
    return y


def e4m3_values():
    """The 256 values of the 8-bit float with 4 exponent and 3 mantissa bits that has no infinities."""
    out = np.empty(256)
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        if e == 15 and m == 7:
            v = math.nan
        out[code] = -v if code & 128 else v
    return out


def row_scale(x, store):
    """fp32 scales of fp32 rows (the definition is in fp32)."""
    x = np.asarray(x, np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        top = np.max(np.abs(x), axis=-1)
        s = top / np.float32(TOP[store])
        s = np.where(s < np.float32(2.0 ** -126), np.float32(1.0), s)
        return np.where(np.isfinite(x).all(-1), s, np.float32(np.nan)).astype(np.float32)


def int8_codes(x, scale):
    x = np.asarray(x, np.float32)
    ok = np.isfinite(scale)[..., None]
    q = np.rint(np.where(ok, x, np.float32(0.0)) / np.where(ok, scale[..., None], np.float32(1.0)))
    return np.clip(q, -127, 127).astype(np.int8)


def tree_attention(q, k, v, pos, visible, scale):
    """q [B,n,Hq,dh]; k, v [B,Hkv,cap,dh]; pos [B]; visible [B][n] of ints.  Returns (out [B,n,Hq,dh], weight of the rows'
    magnitudes sum_j P |v|, which rounding errors are measured in)."""
    B, n, Hq, dh = q.shape
    Hkv = k.shape[1]
    out, mag = np.zeros((B, n, Hq, dh)), np.zeros((B, n, Hq, dh))
    for b in range(B):
        for t in range(n):
            rows = list(range(pos[b])) + [pos[b] + j for j in range(n) if visible[b][t] >> j & 1]
            if not rows:
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                s = (k[b, g, rows] @ np.asarray(q[b, t, h], np.float64)) * scale
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, t, h] = p @ v[b, g, rows]
                mag[b, t, h] = p @ np.abs(v[b, g, rows])
    return out, mag


def commit(cache, pos, path, accepted):
    """cache [L,B,H,cap,...]; returns a copy with the accepted rows moved together."""
    new = cache.copy()
    for b in range(cache.shape[1]):
        for j in range(accepted[b]):
            new[:, b, :, pos[b] + j] = cache[:, b, :, pos[b] + path[b][j]]
    return new
