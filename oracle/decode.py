"""The operators on both sides of the attention (include/rsr_decode.h) by their definitions, in 64 bits and more and in Python integers."""
from __future__ import annotations

import math

import numpy as np


def rotate(x, position, frequency, head_dim, eps=None, weight=None, pairs=False):
    """``x [tokens][heads * head_dim]`` (float64).  Returns the result and, for bounds, |y_a| + |y_b| behind every value.  Angles and
    their functions in the longest type that numpy has."""
    tokens = x.shape[0]
    y = x.reshape(tokens, -1, head_dim).astype(np.longdouble)
    if eps is not None:
        with np.errstate(invalid="ignore", divide="ignore"):
            y = y / np.sqrt((y * y).sum(2, keepdims=True) / head_dim + np.longdouble(eps))
            y = y * (1 if weight is None else np.asarray(weight, np.longdouble))
    half = 0 if frequency is None else len(frequency)
    out, size = y.copy(), np.abs(y)
    for j in range(half):
        a, b = (2 * j, 2 * j + 1) if pairs else (j, j + half)
        t = np.asarray(position).astype(np.longdouble)[:, None] * np.longdouble(frequency[j])
        c, s = np.cos(t), np.sin(t)
        out[:, :, a], out[:, :, b] = y[:, :, a] * c - y[:, :, b] * s, y[:, :, a] * s + y[:, :, b] * c
        size[:, :, a] = size[:, :, b] = np.abs(y[:, :, a]) + np.abs(y[:, :, b])
    return out.reshape(tokens, -1).astype(np.float64), size.reshape(tokens, -1).astype(np.float64)


def sample(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """(token, probability, kept) of one row of scores (float64)."""
    x = np.asarray(logits, np.float64)
    if np.isnan(x).any():
        return -1, math.nan, 0
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if not len(order):
        return -1, 0.0, 0
    if not temperature > 0:
        return int(order[0]), 1.0, 1
    x = x[order].astype(np.longdouble)
    if np.isfinite(x[0]):
        with np.errstate(under="ignore"):
            weight = np.exp((x - x[0]) / np.longdouble(temperature))
    else:
        weight = (x == x[0]).astype(np.longdouble)
    total = weight.cumsum()
    kept = top_k if 0 < top_k < len(x) else len(x)
    if top_p < 1:
        kept = min(kept, 1 + int((total < max(top_p, 0) * total[kept - 1]).sum()))
    if min_p > 0:
        kept = min(kept, int((weight >= min(min_p, 1)).sum()))
    u = min(uniform, 1 - 2.0**-24) if uniform > 0 else 0.0
    at = min(int((total <= u * total[kept - 1]).sum()), kept - 1)
    return int(order[at]), float(weight[at] / total[kept - 1]), kept


def keep(drafted, chosen, parent, start, tokens):
    """(rows, found, add, first); ``parent`` None: chains."""
    rows, add, first = [], [], []
    for r in range(len(start) - 1):
        begin = int(start[r])
        n = min(64, min(int(start[r + 1]), tokens) - begin) if begin >= 0 else 0
        first.append(min(len(rows), tokens))
        at, before = (0 if n > 0 else None), len(rows)
        while at is not None:
            rows.append(begin + at)
            want = int(chosen[begin + at])
            hangs = (lambda j: j - 1) if parent is None else (lambda j: int(parent[begin + j]))
            at = next((j for j in range(at + 1, n) if hangs(j) == at and int(drafted[begin + j]) == want), None) if want >= 0 else None
        add.append(len(rows) - before)
    first.append(min(len(rows), tokens))
    rows = (rows + [-1] * tokens)[:tokens]
    return rows, [int(chosen[i]) if i >= 0 else -1 for i in rows], add, first
