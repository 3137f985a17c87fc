"""The operators around the paged cache (include/rsr_cache.h) by their definitions, in float64 and Python integers."""
from __future__ import annotations

import math

import numpy as np


def _trees(start, tokens, most):
    """(request, first row, number of new tokens) of the requests that have rows."""
    for r in range(len(start) - 1):
        first = int(start[r])
        n = min(most, min(int(start[r + 1]), tokens) - first)
        if first >= 0 and n > 0:
            yield r, first, n


def attention(q, k, v, cache_k, cache_v, table, held, start, mask, heads, scale, max_new, round_to=None):
    """``q [tokens][heads * dim]``, ``k``, ``v [tokens][kv_heads * dim]``, caches ``[pages][kv_heads][page_size][dim]`` (all
    float64).  ``round_to(x)``: what the cache's type makes of the new keys and values.  Returns the result, NaN in rows of no
    request, and the same sum with |v| and the largest scale * sum |q| |k| behind every value, for bounds."""
    pages, kv_heads, size, dim = cache_k.shape
    tokens = q.shape[0]
    k, v = (round_to(k), round_to(v)) if round_to else (k, v)
    out = np.full((tokens, heads, dim), np.nan)
    spread, steep, seen_most = np.zeros_like(out), np.zeros((tokens, heads)), 0
    for r, first, n in _trees(start, tokens, max_new):
        have = min(max(int(held[r]), 0), table.shape[1] * size)
        slots = [(int(table[r, t // size]), t % size) for t in range(have) if 0 <= table[r, t // size] < pages]
        page, offset = (np.array([s[i] for s in slots], dtype=np.int64) for i in (0, 1))
        for i in range(n):
            bits = int(mask[first + i]) if mask is not None else (1 << (i + 1)) - 1
            new = [first + j for j in range(n) if bits >> j & 1]
            seen_most = max(seen_most, len(slots) + len(new))
            for a in range(heads):
                b = a // (heads // kv_heads)
                cut = slice(b * dim, (b + 1) * dim)
                K = np.concatenate([cache_k[page, b, offset], k[new, cut]])
                V = np.concatenate([cache_v[page, b, offset], v[new, cut]])
                x = q[first + i, a * dim:(a + 1) * dim]
                if not len(K):
                    out[first + i, a] = 0.0
                    continue
                s = (K @ x) * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[first + i, a], spread[first + i, a] = w @ V, w @ np.abs(V)
                steep[first + i, a] = (np.abs(K) @ np.abs(x)).max() * abs(scale)
    flat = (tokens, heads * dim)
    return out.reshape(flat), spread.reshape(flat), np.repeat(steep, dim, axis=1).reshape(flat), seen_most


def masks(parent, start, tokens):
    """(mask, depth) as lists, None in rows of no request."""
    mask, depth = [None] * tokens, [None] * tokens
    for _, first, n in _trees(start, tokens, tokens):
        for i in range(n):
            if i >= 64:
                mask[first + i], depth[first + i] = 0, -1
                continue
            up = int(parent[first + i])
            hangs = 0 <= up < i
            mask[first + i] = 1 << i | (mask[first + up] if hangs else 0)
            depth[first + i] = depth[first + up] + 1 if hangs else 0
    return mask, depth


def slots(held, add, table, page_size, free, count, max_slots):
    """(slots, table, start, now, left) for the next add[r] tokens of every request."""
    table, free = np.array(table), [int(x) for x in free[:max(0, count)]]
    left, found, start, now = max(0, count), [], [], []
    for r in range(len(held)):
        have, more = max(0, int(held[r])), max(0, int(add[r]))
        start.append(min(len(found), max_slots))
        kept = have
        before = min(math.ceil(have / page_size), table.shape[1])
        for c in range(before, min(math.ceil((have + more) / page_size), table.shape[1])):
            left -= 1
            table[r, c] = free.pop() if free else -1
        for t in range(have, have + more):
            page = int(table[r, t // page_size]) if t // page_size < table.shape[1] else -1
            found.append(page * page_size + t % page_size if page >= 0 else -1)
            # (a page that the request gave up holds no token, but its place in the request is counted)
            kept += t // page_size < table.shape[1] and (page >= 0 or t // page_size < before)
        now.append(kept)
    start.append(min(len(found), max_slots))
    found = (found + [-1] * max_slots)[:max_slots]
    return found, table, start, now, left


def append(cache, x, rows, slots, round_to):
    """The cache ``[pages][kv_heads][page_size][dim]`` with the rows ``x [nrows][kv_heads * dim]`` in their slots."""
    cache = cache.copy()
    pages, heads, size, dim = cache.shape
    for i, slot in enumerate(slots):
        row = i if rows is None else int(rows[i])
        if 0 <= slot < pages * size and 0 <= row < x.shape[0]:
            cache[slot // size, :, slot % size] = round_to(x[row]).reshape(heads, dim)
    return cache
