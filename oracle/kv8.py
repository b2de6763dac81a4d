"""The 8-bit paged KV cache in 64 bits: writing, reading back and decode attention, written from its definition.

A cache is held as the values of its codes [n_blocks, 2, n_kv_heads, 128, head_dim] and its scales
[n_blocks, 2, n_kv_heads, 4], float64 numpy arrays.  value = code * 2^e with the smallest e >= -100 for which the
largest magnitude of the 32 positions that share the scale is at most top * 2^e.
"""
from __future__ import annotations

import numpy as np

PAGE, BLOCK = 128, 32
TOP = {"e4m3": 448.0, "int8": 127.0}


def to_grid(x, fmt):
    """The nearest value that a code stands for (|x| at most the format's top), ties to even."""
    if fmt == "int8":
        return np.rint(x)
    _, e = np.frexp(np.maximum(np.abs(x), 2.0 ** -6))  # |x| = f 2^e, 1/2 <= f < 1: three bits behind the first
    step = np.ldexp(1.0, e - 4)
    return np.rint(x / step) * step


def exponent(amax, fmt):
    e = -100
    if amax > 0:
        e = max(e, int(np.floor(np.log2(amax / TOP[fmt]))) - 1)
    while amax > TOP[fmt] * 2.0 ** e:
        e += 1
    return e


def write(codes, scales, fmt, table_row, pos0, k, v):
    """Tokens k, v [n, n_kv_heads, head_dim] become positions pos0 .. of the sequence whose blocks table_row names (in place)."""
    for kv, x in ((0, np.asarray(k, np.float64)), (1, np.asarray(v, np.float64))):
        p, end = pos0, pos0 + len(x)
        while p < end:
            stop = min(end, (p // BLOCK + 1) * BLOCK)
            page, a, b = table_row[p // PAGE], p % PAGE, p % PAGE + stop - p
            part, base = a // BLOCK, a // BLOCK * BLOCK
            for h in range(x.shape[1]):
                new, old = x[p - pos0:stop - pos0, h], scales[page, kv, h, part]
                if not np.isfinite(new).all() or (a > base and not np.isfinite(old)):
                    scales[page, kv, h, part] = np.nan
                    continue
                e = exponent(np.abs(new).max(), fmt)
                if a > base:
                    eo = int(np.frexp(old)[1]) - 1
                    if eo < e:
                        codes[page, kv, h, base:a] = to_grid(codes[page, kv, h, base:a] * 2.0 ** (eo - e), fmt)
                    e = max(e, eo)
                codes[page, kv, h, a:b] = to_grid(new * 2.0 ** -e, fmt)
                scales[page, kv, h, part] = 2.0 ** e
            p = stop


def read(codes, scales, table_row, a, b):
    """Positions a .. b of a sequence: k, v [b - a, n_kv_heads, head_dim]."""
    p = np.arange(a, b)
    page, slot = np.asarray(table_row)[p // PAGE], p % PAGE
    x = codes[page, :, :, slot] * scales[page, :, :, slot // BLOCK][..., None]
    return x[:, 0], x[:, 1]


def attention(q, k, v):
    """One query row q [n_heads, hd] over k, v [n, n_kv_heads, hd]: out [n_heads, hd], lse [n_heads], and per head the
    largest sum over dims of |q k| / sqrt(hd) and the sum of p |v| (what errors are bounded by)."""
    H, hd = q.shape
    if len(k) == 0:
        return np.zeros((H, hd)), np.full(H, -np.inf), np.zeros(H), np.zeros((H, hd))
    G = H // k.shape[1]
    out, lse, mag, pv = np.empty((H, hd)), np.empty(H), np.empty(H), np.empty((H, hd))
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        s = kh @ q[h] / np.sqrt(hd)
        m = s.max()
        e = np.exp(s - m)
        p = e / e.sum()
        out[h], lse[h] = p @ vh, m + np.log(e.sum())
        mag[h], pv[h] = (np.abs(kh) @ np.abs(q[h])).max() / np.sqrt(hd), p @ np.abs(vh)
    return out, lse, mag, pv
