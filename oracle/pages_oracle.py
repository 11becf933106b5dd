"""Plain definitions of the page-sparse decode attention operators, in numpy and 64 bits.

TEST INFRASTRUCTURE ONLY, like the rest of this package: nothing of the library is imported here.  Each
function follows the operator's definition step by step, one head and one page at a time; bf16 tensors
come as float64 arrays of their values.
"""
from __future__ import annotations

import numpy as np

PAGE = 16
E_MIN, E_MAX = -60, 50


def to_bf16(x: np.ndarray) -> np.ndarray:
    """float64 -> float32 -> bf16 (both to nearest even), as float64 values."""
    with np.errstate(over="ignore"):
        u = np.asarray(x, dtype=np.float64).astype(np.float32).view(np.uint32).astype(np.uint64)
    nan = (u & 0x7FFFFFFF) > 0x7F800000
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint32) << 16
    out = r.astype(np.uint32).view(np.float32).astype(np.float64)
    return np.where(nan, np.nan, out)


def rows_of(seq_lens, q_offsets=None):
    """[(row, sequence, position)] of a call."""
    if q_offsets is None:
        return [(b, b, int(n) - 1) for b, n in enumerate(seq_lens)]
    out = []
    for b, n in enumerate(seq_lens):
        m = int(q_offsets[b + 1]) - int(q_offsets[b])
        out += [(int(q_offsets[b]) + i, b, int(n) - m + i) for i in range(m)]
    return out


def exponent(a: float) -> int:
    """Smallest e in [E_MIN, E_MAX] with a <= 127 * 2^e (E_MAX where there is none)."""
    e = E_MIN
    while e < E_MAX and a > 127.0 * 2.0 ** e:
        e += 1
    return e


def page_bounds(keys: np.ndarray):
    """keys [tokens][D], the stored ones of one page and head -> (codes int8 [D/8][2][8], scales uint8 [D/32])."""
    D = keys.shape[1]
    codes, scales = np.zeros((D // 8, 2, 8), dtype=np.int8), np.zeros(D // 32, dtype=np.uint8)
    hi, lo = np.zeros(D), np.zeros(D)
    for d in range(D):
        col = keys[:, d][~np.isnan(keys[:, d])]
        if col.size:
            hi[d], lo[d] = col.max(), col.min()
    for c in range(D // 32):
        e = exponent(max(np.abs(hi[32 * c:32 * c + 32]).max(), np.abs(lo[32 * c:32 * c + 32]).max()))
        scales[c] = e + 127
        for d in range(32 * c, 32 * c + 32):
            codes[d // 8, 0, d % 8] = int(min(127.0, max(-127.0, np.ceil(hi[d] / 2.0 ** e))))
            codes[d // 8, 1, d % 8] = int(min(127.0, max(-127.0, np.floor(lo[d] / 2.0 ** e))))
    return codes, scales


def page_scores(q: np.ndarray, codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """q [G][D]; codes int8 [pages][D/8][2][8], scales uint8 [pages][D/32] -> float32 [pages]."""
    n, G, D = codes.shape[0], q.shape[0], q.shape[1]
    hi = codes[:, :, 0].reshape(n, D).astype(np.int64)
    lo = codes[:, :, 1].reshape(n, D).astype(np.int64)
    q = np.where(np.isnan(q), 0.0, q)
    best = np.full(n, -np.inf, dtype=np.float32)
    for h in range(G):
        s = None
        for c in range(D // 32):
            x = q[h, 32 * c:32 * c + 32]
            f = exponent(np.abs(x).max())
            z = np.clip(np.rint(x / 2.0 ** f), -127, 127).astype(np.int64)
            i = (z * np.where(z > 0, hi[:, 32 * c:32 * c + 32], lo[:, 32 * c:32 * c + 32])).sum(1)
            v = (i.astype(np.float64) * 2.0 ** (scales[:, c].astype(np.float64) - 127 + f)).astype(np.float32)
            s = v if s is None else (s + v).astype(np.float32)
        best = np.maximum(best, s)
    return best


def page_select(q, codes, scales, page_table, seq_lens, top, sink, window, q_offsets=None):
    """q [rows][Hq][D]; codes / scales with leading [num_pages][Hkv] -> (list int32 [rows][Hkv][top], count int32 [rows][Hkv]);
    rows of no sequence keep list -2 and count -2."""
    rows, Hq, _ = q.shape
    Hkv = codes.shape[1]
    G = Hq // Hkv
    lst, cnt = np.full((rows, Hkv, top), -2, dtype=np.int32), np.full((rows, Hkv), -2, dtype=np.int32)
    for r, b, pos in rows_of(seq_lens, q_offsets):
        n = pos // PAGE + 1
        for g in range(Hkv):
            if n <= top:
                take = list(range(n))
            else:
                pg = page_table[b, :n]
                s = page_scores(q[r, g * G:(g + 1) * G], codes[pg, g], scales[pg, g])
                mid = sorted(range(sink, n - window), key=lambda j: (-s[j], j))[:top - sink - window]
                take = sorted(list(range(sink)) + mid + list(range(n - window, n)))
            lst[r, g] = -1
            lst[r, g, :len(take)] = take
            cnt[r, g] = len(take)
    return lst, cnt


def attn_pages(q, k_cache, v_cache, page_table, seq_lens, page_list, page_count, q_offsets=None, sm_scale=None):
    """-> (out [rows][Hq][D], lse [rows][Hq], slack): slack [rows][Hq] = (largest sum_d |q_d K_jd| * scale, tokens,
    sum_j p_j |V_j| [D]) of every row and head, for the error bounds of a 32-bit computation."""
    rows, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(D) if not sm_scale else sm_scale
    out, lse = np.zeros((rows, Hq, D)), np.full((rows, Hq), -np.inf)
    mag, num, absv = np.zeros((rows, Hq)), np.zeros((rows, Hq)), np.zeros((rows, Hq, D))
    for r, b, pos in rows_of(seq_lens, q_offsets):
        for g in range(Hkv):
            ks, vs = [], []
            for e in page_list[r, g, :max(0, page_count[r, g])]:
                if e < 0 or e > pos // PAGE or not 0 <= page_table[b, e] < k_cache.shape[0]:
                    continue
                m = min(PAGE, pos - e * PAGE + 1)
                ks.append(k_cache[page_table[b, e], g, :m])
                vs.append(v_cache[page_table[b, e], g, :m])
            if not ks:
                continue
            k, v = np.concatenate(ks), np.concatenate(vs)
            for h in range(g * G, (g + 1) * G):
                s = scale * (k @ q[r, h])
                p = np.exp(s - s.max())
                out[r, h] = (p @ v) / p.sum()
                lse[r, h] = s.max() + np.log(p.sum())
                mag[r, h] = scale * (np.abs(k) @ np.abs(q[r, h])).max()
                num[r, h] = len(s)
                absv[r, h] = (p @ np.abs(v)) / p.sum()
    return out, lse, (mag, num, absv)


def rope_append(qkv, k_cache, v_cache, page_table, seq_lens, Hq, Hkv, w_qn, w_kn, eps, theta, q_offsets=None):
    """qkv [rows][(Hq+2Hkv)*D] -> (q [rows][Hq][D] not rounded, NaN for rows of no sequence; size [rows][Hq][D] = |a| + |b| of
    each rotary pair).  k_cache / v_cache ([num_pages][Hkv][16][D]) get the rows' keys (rounded to fp32, then bf16) and values."""
    D = k_cache.shape[3]
    half = D // 2
    x = qkv.reshape(qkv.shape[0], Hq + 2 * Hkv, D)
    q = np.full((qkv.shape[0], Hq, D), np.nan)
    size = np.zeros_like(q)

    def turn(v, w, pos):
        if w is not None:
            v = v / np.sqrt((v * v).mean() + eps) * w
        ang = pos * float(theta) ** (-2.0 * np.arange(half) / D)
        a, b = v[:half], v[half:]
        return (np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)]),
                np.tile(np.abs(a) + np.abs(b), 2))

    for r, b, pos in rows_of(seq_lens, q_offsets):
        for h in range(Hq):
            q[r, h], size[r, h] = turn(x[r, h], w_qn, pos)
        page = page_table[b, pos // PAGE]
        for g in range(Hkv):
            k_cache[page, g, pos % PAGE] = to_bf16(turn(x[r, Hq + g], w_kn, pos)[0])
            v_cache[page, g, pos % PAGE] = x[r, Hq + Hkv + g]
    return q, size
