"""Float64 oracle of the growing paged cache: where a chunk's tokens lie, what a write
leaves there, and the attention of a chunk over its request's cache.  Plain loops over
requests and tokens; arrays are numpy, values float64."""
from __future__ import annotations

import numpy as np

from .c2kv_oracle import rope_rotate


def places(tok_off, kv_len, block_table, page_size, n_pages, n_tokens):
    """{row: (request, cache index, page, offset)} of the chunk rows that have a place.
    page is None where the block table names none."""
    out = {}
    for b in range(len(kv_len)):
        r0, r1 = int(tok_off[b]), int(tok_off[b + 1])
        for i in range(max(r0, 0), min(r1, n_tokens)):
            n = r1 - r0
            j = int(kv_len[b]) - n + (i - r0)
            if j < 0 or j // page_size >= block_table.shape[1]:
                continue
            page = int(block_table[b, j // page_size])
            out[i] = (b, j, page if 0 <= page < n_pages else None, j % page_size)
    return out


def turned(x, pos, base):
    """Rows x [n][H][D] turned to pos [n] (None: as they are)."""
    x = np.asarray(x, np.float64)
    if pos is None:
        return x
    return np.stack([rope_rotate(x[i], int(pos[i]), base) for i in range(len(x))]) \
        if len(x) else x


def int8_scale(x):
    """Scale of each row over the last axis: max |x| / 127, 1 for zeros."""
    s = np.abs(x).max(-1) / 127.0
    return np.where(s == 0, 1.0, s)


def cached(k_pages, v_pages, table_row, length):
    """Keys and values [length][H][D] of one request and which of them exist."""
    n_pages, H, PS, D = k_pages.shape
    k, v = np.zeros((length, H, D)), np.zeros((length, H, D))
    there = np.zeros(length, bool)
    for j in range(length):
        if j // PS >= len(table_row):
            continue
        p = int(table_row[j // PS])
        if 0 <= p < n_pages:
            k[j], v[j], there[j] = k_pages[p, :, j % PS], v_pages[p, :, :, j % PS], True
    return k, v, there


def attend(q, pos, k_pages, v_pages, tok_off, kv_len, block_table, base, scale=None):
    """(out, lse, has) of each row of q [n][Hq][D]: token t of request b sees the cache
    indices j <= kv_len[b] - n_b + t that exist; `has` marks the rows of some request."""
    n, Hq, D = q.shape
    Hkv = k_pages.shape[1]
    scale = scale or 1.0 / np.sqrt(D)
    q = turned(q, pos, base)
    out, lse = np.zeros((n, Hq, D)), np.full((n, Hq), -np.inf)
    has = np.zeros(n, bool)
    for b in range(len(kv_len)):
        r0, r1 = int(tok_off[b]), int(tok_off[b + 1])
        k, v, there = cached(k_pages, v_pages, block_table[b], max(int(kv_len[b]), 0))
        for i in range(r0, min(r1, n)):
            has[i] = True
            sees = max(int(kv_len[b]) - (r1 - r0) + (i - r0) + 1, 0)
            at = np.flatnonzero(there[:sees])
            if not len(at):
                continue
            for h in range(Hq):
                g = h // (Hq // Hkv)
                s = k[at, g] @ q[i, h] * scale
                p = np.exp(s - s.max())
                out[i, h] = p @ v[at, g] / p.sum()
                lse[i, h] = s.max() + np.log(p.sum())
    return out, lse, has
