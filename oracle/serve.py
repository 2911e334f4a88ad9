"""Oracle of the serving operators around the index, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain statements of
rotary positions with several axes, block tables, the 8-bit cache and the
attentions that read it or a whole prompt; loops over requests, heads and
queries, no blocking.
"""
from __future__ import annotations

import numpy as np

from .saki import ROPE_THETA, fp8_round

__all__ = ["rope_axes", "block_tables", "cache_write", "cache_rows", "cache_attend", "prompt_attend",
           "CACHE_BLOCK"]

CACHE_BLOCK = 64


def rope_axes(x, pos, sections, theta: float = ROPE_THETA, inverse: bool = False):
    """x [T, H, d]; pos [axes, T]: pair (m, m + d/2) turned by
    pos[axis(m)] * theta^(-2m/d), the first sections[0] pairs by axis 0 and so on."""
    x = np.asarray(x, np.float64)
    half = x.shape[-1] // 2
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = np.asarray(pos, np.float64)[axis].T * theta ** (-np.arange(half) / half)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1.0 if inverse else 1.0)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, a * s + b * c], -1)


def block_tables(ctx, new, free, tables):
    """Requests in order, tokens in order: a token whose block is not there
    takes the next free one.  -> tables, slots, pos, cu, lens, counts"""
    tables = np.array(tables, np.int64)
    rows = tables.shape[1]
    slots, pos, cu, lens = [], [], [0], []
    taken = lacking = 0
    for b, (c, n) in enumerate(zip(ctx, new)):
        c, n = min(max(int(c), 0), rows * CACHE_BLOCK), max(int(n), 0)
        have = -(-c // CACHE_BLOCK)
        need = -(-(c + n) // CACHE_BLOCK)
        for blk in range(have, need):
            if blk < rows and taken < len(free):
                tables[b, blk] = free[taken]
                taken += 1
                have = blk + 1
            else:
                lacking += 1
        lens.append(min(c + n, have * CACHE_BLOCK))
        for p in range(c, c + n):
            blk, off = divmod(p, CACHE_BLOCK)
            slots.append(tables[b, blk] * CACHE_BLOCK + off if blk < have else -1)
            pos.append(p)
        cu.append(cu[-1] + n)
    return tables, np.array(slots, np.int64), np.array(pos, np.int64), np.array(cu), np.array(lens), \
        np.array([taken, lacking])


def _scale(top):
    """The least power of two s >= 2^-100 with top <= 448 s."""
    e = -100
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def cache_write(x, slots, codes, scales):
    """x [T, H, d] to codes [n_blocks, H, 64, d] (their values) and scales
    [n_blocks, H].  -> new codes, scales"""
    x = np.asarray(x, np.float64)
    codes, scales = np.array(codes, np.float64), np.array(scales, np.float64)
    n_slots = codes.shape[0] * CACHE_BLOCK
    t = 0
    while t < len(slots):
        if not 0 <= slots[t] < n_slots:
            t += 1
            continue
        blk, first = divmod(int(slots[t]), CACHE_BLOCK)
        n = 1
        while t + n < len(slots) and slots[t + n] > slots[t + n - 1] and slots[t + n] // CACHE_BLOCK == blk:
            n += 1
        at = np.asarray(slots[t:t + n]) % CACHE_BLOCK
        for h in range(x.shape[1]):
            s = _scale(np.abs(x[t:t + n, h]).max())
            if first:
                s = max(s, scales[blk, h])
                if s > scales[blk, h]:
                    codes[blk, h, :first] = fp8_round(codes[blk, h, :first] * (scales[blk, h] / s))
            codes[blk, h, at] = fp8_round(x[t:t + n, h] / s)
            scales[blk, h] = s
        t += n
    return codes, scales


def cache_rows(codes, scales, table, n, h):
    """The first n rows of a request and head: values [n, d], and which of
    them a valid table entry holds."""
    out, ok = np.zeros((n, codes.shape[-1])), np.zeros(n, bool)
    for j in range(n):
        blk = table[j // CACHE_BLOCK] if j // CACHE_BLOCK < len(table) else -1
        if 0 <= blk < codes.shape[0]:
            out[j] = codes[blk, h, j % CACHE_BLOCK] * scales[blk, h]
            ok[j] = True
    return out, ok


def _softmax_sum(q, k, v):
    s = k @ q / np.sqrt(q.size)
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ v, p


def cache_attend(q, k_codes, v_codes, scales, tables, lens, top_idx=None):
    """q [B, H_q, Q, d], codes [n_blocks, H_kv, 64, d] (values), scales
    [n_blocks, H_kv, 2].  -> out, and for each row the sums of p |v| and the
    largest sum of |q_e k_e| / sqrt(d), which error bounds are made of."""
    q = np.asarray(q, np.float64)
    B, H, Q, d = q.shape
    G = H // k_codes.shape[1]
    out, mass, size = np.zeros_like(q), np.zeros_like(q), np.zeros((B, H, Q))
    for b in range(B):
        n = max(0, min(int(lens[b]), len(tables[b]) * CACHE_BLOCK))
        for h in range(H):
            k, ok = cache_rows(k_codes, scales[..., 0], tables[b], n, h // G)
            v, _ = cache_rows(v_codes, scales[..., 1], tables[b], n, h // G)
            for i in range(Q):
                end = max(0, min(n, int(lens[b]) - Q + i + 1))
                pick = np.arange(end)
                if top_idx is not None:
                    pick = np.asarray(top_idx[b, h, i])
                    pick = pick[(pick >= 0) & (pick < end)]
                pick = pick[ok[pick]]
                if pick.size:
                    out[b, h, i], p = _softmax_sum(q[b, h, i], k[pick], v[pick])
                    mass[b, h, i] = p @ np.abs(v[pick])
                    size[b, h, i] = (np.abs(k[pick]) @ np.abs(q[b, h, i])).max() / np.sqrt(d)
    return out, mass, size


def prompt_attend(q, k, v, cu):
    """q [T, H_q, d], k, v [T, H_kv, d], prompt b at rows [cu[b], cu[b+1]).
    -> out (zero outside the prompts), mass and size as for cache_attend"""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    G = q.shape[1] // k.shape[1]
    out, mass, size = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2])
    for a, e in zip(cu[:-1], cu[1:]):
        for h in range(q.shape[1]):
            kk, vv = k[a:e, h // G], v[a:e, h // G]
            for i in range(e - a):
                out[a + i, h], p = _softmax_sum(q[a + i, h], kk[:i + 1], vv[:i + 1])
                mass[a + i, h] = p @ np.abs(vv[:i + 1])
                size[a + i, h] = (np.abs(kk[:i + 1]) @ np.abs(q[a + i, h])).max() / np.sqrt(q.shape[-1])
    return out, mass, size
