"""Plain statements of the cache operators for the tests: rotary rotation and quantisation, reading back, and HCCS
attention over a paged int8 cache.

TEST INFRASTRUCTURE, not part of the product.  numpy only, one token or row at a time, int64 for everything that is
an integer and 80-bit floats for the rotation; shares no code with the CUDA library.
"""
from __future__ import annotations

import numpy as np


def rotate(x, pos, freq, interleaved, scale):
    """x [tokens, heads, d] rotated by the positions, in extended precision; the angle is rounded to fp64 once."""
    y = np.asarray(x, dtype=np.longdouble).copy()
    half = len(freq)
    for t in range(y.shape[0]):
        for i in range(half):
            angle = np.longdouble(np.float64(int(pos[t])) * np.float64(freq[i]))
            c, s = np.cos(angle) * np.longdouble(scale), np.sin(angle) * np.longdouble(scale)
            ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            a, b = y[t, :, ia].copy(), y[t, :, ib].copy()
            with np.errstate(invalid="ignore"):
                y[t, :, ia] = a * c - b * s
                y[t, :, ib] = b * c + a * s
    return y


def quantise(y, step):
    """Codes of y [tokens, heads, d] with one step per head: nearest, ties to even, clamped; NaN -> 0."""
    with np.errstate(invalid="ignore"):
        z = np.rint(y / np.asarray(step, dtype=np.float32).astype(np.longdouble)[None, :, None])
    z = np.where(np.isnan(z), 0, np.clip(z, -128, 127))
    return z.astype(np.int8)


def write(pool, codes, slots):
    """A copy of the pool [pages, heads, page, d] with the codes [tokens, heads, d] at their slots (negative: skipped)."""
    out = pool.copy()
    page = pool.shape[2]
    for t, s in enumerate(slots):
        if 0 <= s < pool.shape[0] * page:
            out[s // page, :, s % page] = codes[t]
    return out


def sequence(pool, table_row, n):
    """The first n tokens of a sequence, [n, heads, d]."""
    page = pool.shape[2]
    return np.stack([pool[table_row[j // page], :, j % page] for j in range(n)]) if n else np.zeros((0,) + pool.shape[1:2] + pool.shape[3:], pool.dtype)


def rho16(z, clb):
    return 32767 >> (int(z).bit_length() - 1) if clb else 32767 // int(z)


def attend(q, k_pool, v_pool, table, q_start, kv_len, theta, mult, shift, tree=None):
    """Per row (token, head): (sum_j s_j V_j int64 [T, Hq, d], Z int64 [T, Hq], seen keys int64 [T, Hq])."""
    T, hq, d = q.shape
    hkv = k_pool.shape[1]
    g = hq // hkv
    num, zs, cnt = np.zeros((T, hq, d), np.int64), np.zeros((T, hq), np.int64), np.zeros((T, hq), np.int64)
    for b in range(len(kv_len)):
        s0, s1, n = int(q_start[b]), int(q_start[b + 1]), int(kv_len[b])
        k = sequence(k_pool, table[b], n).astype(np.int64)
        v = sequence(v_pool, table[b], n).astype(np.int64)
        for t in range(s0, s1):
            new = np.arange(n) - (n - (s1 - s0))
            if tree is None:
                seen = new <= t - s0
            else:
                words = [int(w) & 0xFFFFFFFF for w in tree[t]]
                bits = sum(w << (32 * i) for i, w in enumerate(words))
                seen = np.array([j < 0 or (bits >> int(j)) & 1 == 1 for j in new], dtype=bool)
            if not seen.any():
                continue
            for h in range(hq):
                big, slope, reach = (int(c) for c in theta[h])
                acc = k[seen, h // g] @ q[t, h].astype(np.int64)
                x = np.clip((acc * int(mult[h]) + (1 << (shift - 1))) >> shift, -128, 127)
                s = big - slope * np.minimum(x.max() - x, reach)
                num[t, h], zs[t, h], cnt[t, h] = s @ v[seen, h // g], s.sum(), seen.sum()
    return num, zs, cnt


def integer_output(num, zs, cnt, clb):
    """rho * sum s V of the int16 path; rows without keys are zeros."""
    out = np.zeros(num.shape, np.int64)
    for t in range(num.shape[0]):
        for h in range(num.shape[1]):
            if cnt[t, h]:
                out[t, h] = num[t, h] * rho16(zs[t, h], clb)
    return out
