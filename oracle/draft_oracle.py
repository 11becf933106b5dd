"""Plain definitions, in 64 bits, of the operators on caches of 16 or 8 bits and on drafted tokens (test infrastructure only)."""
from __future__ import annotations

import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


def to_bf16(x):
    """Nearest bf16 (halves to even) of values in 64 bits that fit, by way of fp32 as the operators round them."""
    b = np.asarray(x, dtype=np.float64).astype(np.float32)
    u = b.view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isfinite(b), r, b).astype(np.float64)


def to_e4m3(x):
    """Nearest e4m3 value, halves to even: steps of 2^(e - 3) in [2^e, 2^(e + 1)), of 2^-9 below 2^-6."""
    x = np.asarray(x, dtype=np.float64)
    e = np.maximum(np.frexp(np.where(x == 0, 1.0, x))[1] - 1, -6)
    step = np.ldexp(1.0, e - 3)
    return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def quantise(x, fmt):
    """Codes and scales (both float64) of heads x [..., D]: every step in fp32, as defined."""
    x = np.asarray(x, dtype=np.float64).astype(np.float32)
    with np.errstate(all="ignore"):
        a = np.abs(x).max(-1)
        scale = np.maximum(a * np.float32(1.0 / TOP[fmt]), np.float32(2.0 ** -64))
        y = (x * (np.float32(1.0) / scale)[..., None]).astype(np.float64)
    fine = np.isfinite(x).all(-1)
    y = np.where(fine[..., None], y, 0.0)
    codes = np.rint(y) if fmt == "int8" else to_e4m3(y)
    return codes, np.where(fine, scale.astype(np.float64), np.nan)


def rows_of(lens, offsets):
    """[(sequence, number in it, rows of it)] of every row that is no padding."""
    if offsets is None:
        return [(b, 0, 1) for b in range(len(lens))]
    return [(b, i, int(offsets[b + 1] - offsets[b])) for b in range(len(lens)) for i in range(int(offsets[b + 1] - offsets[b]))]


def turn(x, pos, theta, gain, eps):
    """Head norm (gain None: none) and rotary embedding of heads x [..., D]; also the size of the terms that were added."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    if gain is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain
    ang = pos * float(theta) ** (-2.0 * np.arange(d // 2) / d)
    c, s = np.cos(ang), np.sin(ang)
    a, b = x[..., :d // 2], x[..., d // 2:]
    size = np.concatenate([np.abs(a) + np.abs(b)] * 2, -1)
    return np.concatenate([a * c - b * s, b * c + a * s], -1), size


def append(qkv, table, lens, offsets, positions, Hq, Hkv, gq, gk, eps, theta):
    """q [rows, Hq, D] in 64 bits, the size of its terms, and [(page, slot, keys [Hkv, D] in bf16, values)] of every row."""
    D = qkv.shape[1] // (Hq + 2 * Hkv)
    q, size, put = np.zeros((len(qkv), Hq, D)), np.zeros((len(qkv), Hq, D)), []
    for r, (b, i, m) in enumerate(rows_of(lens, offsets)):
        x = qkv[r].reshape(-1, D)
        t = int(lens[b]) - m + i
        pos = t if positions is None else int(positions[r])
        q[r], size[r] = turn(x[:Hq], pos, theta, gq, eps)
        put.append((int(table[b, t // 16]), t % 16, to_bf16(turn(x[Hq:Hq + Hkv], pos, theta, gk, eps)[0]), x[Hq + Hkv:]))
    return q, size, put


def visible(n, m, i, bits):
    """Which of a sequence's n tokens its drafted token i sees; bits: its mask as a whole number, None for tokens 0 .. i."""
    see = np.ones(n, dtype=bool)
    for j in range(m):
        see[n - m + j] = j <= i if bits is None else bool(bits >> j & 1)
    return see


def attend(q, k, v, table, lens, offsets, mask, scale=None, v_scales=None):
    """out [rows, Hq, D], lse [rows, Hq], per row and head the largest sum of |products| of a score, sum_j p_j |v_j|, and (with v_scales)
    max_j (p_j scale_j) * sum_j |code_j|.  k, v: what the cache stands for, in 64 bits.  mask: [rows] whole numbers or None."""
    rows, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    scale = scale or 1.0 / math.sqrt(D)
    out, lse = np.zeros(q.shape), np.full((rows, Hq), -np.inf)
    size, spread, codes = np.zeros((rows, Hq)), np.zeros(q.shape), np.zeros(q.shape)
    for r, (b, i, m) in enumerate(rows_of(lens, offsets)):
        n = int(lens[b])
        see = np.nonzero(visible(n, m, i, None if mask is None else mask[r]))[0]
        if len(see) == 0:
            continue
        pages, slots = table[b, see // 16], see % 16
        for g in range(Hkv):
            kk, vv = k[pages, g, slots], v[pages, g, slots]
            for h in range(g * G, g * G + G):
                s = kk @ q[r, h] * scale
                top = s.max()
                p = np.exp(s - top)
                lse[r, h] = top + np.log(p.sum())
                p /= p.sum()
                out[r, h], spread[r, h] = p @ vv, p @ np.abs(vv)
                if v_scales is not None:
                    vs = v_scales[pages, g, slots]
                    codes[r, h] = (p * vs).max() * (np.abs(vv) / vs[:, None]).sum(0)
                size[r, h] = (np.abs(kk) @ np.abs(q[r, h])).max() * scale
    return out, lse, size, spread, codes
