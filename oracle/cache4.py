"""Oracle of the 4-bit cache, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Groups of 32 dims are
rounded to E2M1 values under a power-of-two scale by comparing with every value
there is; bytes are packed and unpacked one element at a time by the layout's
formula.
"""
from __future__ import annotations

import numpy as np

from .serve import CACHE_BLOCK, cache_attend

__all__ = ["E2M1", "cache4_scale", "cache4_round", "cache4_byte", "cache4_values", "cache4_write",
           "cache4_rows", "cache4_prompt"]

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def cache4_scale(top):
    """Exponent of the least power of two s with top <= 7 s, within -100 .. 120."""
    e = -100
    while e < 120 and top > 7.0 * 2.0 ** e:
        e += 1
    return e


def cache4_round(x):
    """x [..., 128] -> codes [..., 128] (0 .. 15) and scale bytes [..., 4]."""
    x = np.asarray(x, np.float64)
    g = x.reshape(-1, GROUP)
    codes, e = np.zeros(g.shape, np.int64), np.zeros(len(g), np.int64)
    for i, row in enumerate(g):
        if not np.isfinite(row).all():
            e[i] = 255
            continue
        exp = cache4_scale(np.abs(row).max())
        e[i] = exp + 127
        far = np.abs(np.abs(row)[:, None] / 2.0 ** exp - E2M1)
        near = far == far.min(1, keepdims=True)  # two for a tie: the even code of them
        even = near & (np.arange(8) % 2 == 0)
        codes[i] = np.where(near.sum(1) > 1, even.argmax(1), near.argmax(1)) + 8 * np.signbit(row)
    return codes.reshape(x.shape), e.reshape(*x.shape[:-1], -1)


def cache4_byte(which, token, dim):
    """Where an element of a (block, head) lies: byte, and 0 (low half) or 1."""
    i = dim // 2
    if which:
        return 256 * (token // 4) + 16 * (i // 4) + 4 * (token % 4) + i % 4, dim % 2
    return 64 * token + i, dim % 2


def _places():
    at = np.array([[[cache4_byte(w, t, d) for d in range(128)] for t in range(CACHE_BLOCK)] for w in range(2)])
    return at[..., 0], at[..., 1]


def cache4_values(cache, scales, which):
    """cache [n, H, 64, 64] and scales [n, H, 2, 64, 4] bytes -> values [n, H, 64, 128]."""
    n, H = cache.shape[:2]
    at, half = (a[which] for a in _places())
    c = np.asarray(cache, np.int64).reshape(n, H, -1)[:, :, at] >> (4 * half) & 15
    e = np.repeat(np.asarray(scales, np.float64)[:, :, which], GROUP, -1)
    v = np.where(c >= 8, -1.0, 1.0) * E2M1[c & 7] * 2.0 ** (e - 127)
    return np.where(e == 255, np.nan, v)


def cache4_write(x, slots, cache, scales, which):
    """x [T, H, 128] to its slots.  -> new bytes"""
    cache, scales = np.array(cache), np.array(scales)
    flat = cache.reshape(*cache.shape[:2], -1)
    at, half = (a[which] for a in _places())
    codes, e = cache4_round(x)
    for t, slot in enumerate(slots):
        if not 0 <= slot < cache.shape[0] * CACHE_BLOCK:
            continue
        blk, off = divmod(int(slot), CACHE_BLOCK)
        scales[blk, :, which, off] = e[t]
        for h in range(cache.shape[1]):
            for d in range(128):
                b = flat[blk, h, at[off, d]]
                flat[blk, h, at[off, d]] = (b & (15 if half[off, d] else 240)) | codes[t, h, d] << (4 * half[off, d])
    return cache, scales


def cache4_rows(values, tables, cu, starts, T):
    """Rows [T, H, 128] of the requests' tokens, and which of them belong to one."""
    out, mine = np.zeros((T, values.shape[1], 128)), np.zeros(T, bool)
    for b in range(len(cu) - 1):
        for t in range(cu[b], cu[b + 1]):
            mine[t] = True
            p = starts[b] + t - cu[b]
            blk = tables[b][p // CACHE_BLOCK] if 0 <= p < len(tables[b]) * CACHE_BLOCK else -1
            if 0 <= blk < len(values):
                out[t] = values[blk, :, p % CACHE_BLOCK]
    return out, mine


def cache4_prompt(q, k, v, tables, lens, cu):
    """q [T, H_q, 128], values k, v [n, H_kv, 64, 128].  -> out (zero for tokens
    of no request), mass and size as for cache_attend"""
    out, mass, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    one = np.ones((*k.shape[:2], 2))
    for b in range(len(lens)):
        rows = slice(cu[b], cu[b + 1])
        if cu[b + 1] > cu[b]:
            o, m, s = cache_attend(q[rows].transpose(1, 0, 2)[None], k, v, one, tables[b:b + 1], lens[b:b + 1])
            out[rows], mass[rows], size[rows] = o[0].transpose(1, 0, 2), m[0].transpose(1, 0, 2), s[0].T
    return out, mass, size
