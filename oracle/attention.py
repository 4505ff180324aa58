"""fp64 oracle of the attention layer over a paged cache, in numpy, one
sequence, node and head at a time, from the definitions:

  append   y = x / sqrt(mean(x^2) + eps) * w, pairs turned by the angle whose
           cosine and sine a table holds for the node's position; keys and
           values to the cache rows len + j;
  verify   o_j = sum_i p_ji v_i, p_j = softmax_i(scale q_j . k_i), i over the
           committed rows and the nodes of j's root path;
  commit   cache row len + t <- row len + path[t], t rising, from a copy;
  copy     the first rows of page dst <- page src, from a copy.

A cache is [layers][pages][kv heads][page size][D] or one layer of it.
"""
from __future__ import annotations

import numpy as np


def root_path(parent, j):
    out = []
    while j >= 0:
        out.append(int(j))
        j = int(parent[j])
    return out[::-1]


def row_of(table, r, page):
    return int(table[r // page]), int(r % page)


def rotate(x, cos, sin, layout):
    """One head x [D], turned by len(cos) angles."""
    y = np.array(x, np.float64)
    h = len(cos)
    for i in range(h):
        a, b = (i, i + h) if layout == "half" else (2 * i, 2 * i + 1)
        y[a] = x[a] * cos[i] - x[b] * sin[i]
        y[b] = x[b] * cos[i] + x[a] * sin[i]
    return y


def transform(x, pos, norm, eps, rope, layout):
    """One head x [D] of a node at position pos."""
    y = np.asarray(x, np.float64)
    if norm is not None:
        y = y / np.sqrt(np.mean(y * y) + eps) * np.asarray(norm, np.float64)
    if rope is not None:
        h = rope.shape[1] // 2
        row = np.asarray(rope[pos], np.float64)
        y = rotate(y, row[:h], row[h:], layout)
    return y


def append(q, k, v, parent, table, lens, k_cache, v_cache, *, q_norm=None, k_norm=None, eps=0.0, rope=None,
           layout="half"):
    """(q_out, k_cache, v_cache), the caches of one layer as fp64 copies."""
    B, n, hq, D = q.shape
    page = k_cache.shape[2]
    out = np.empty((B, n, hq, D))
    kc, vc = np.array(k_cache, np.float64), np.array(v_cache, np.float64)
    for b in range(B):
        for j in range(n):
            pos = int(lens[b]) + len(root_path(parent[b], j)) - 1
            pg, row = row_of(table[b], int(lens[b]) + j, page)
            for h in range(hq):
                out[b, j, h] = transform(q[b, j, h], pos, q_norm, eps, rope, layout)
            for h in range(k.shape[2]):
                kc[pg, h, row] = transform(k[b, j, h], pos, k_norm, eps, rope, layout)
                vc[pg, h, row] = v[b, j, h]
    return out, kc, vc


def verify(q, k_cache, v_cache, parent, table, lens, scale=None):
    """(o, a): the outputs, and sum_i p_ji |v_i| for the bounds of rounded weights."""
    B, n, hq, D = q.shape
    hkv, page = k_cache.shape[1:3]
    scale = D ** -0.5 if scale is None else scale
    o, a = np.empty((B, n, hq, D)), np.empty((B, n, hq, D))
    for b in range(B):
        length = int(lens[b])
        where = [row_of(table[b], r, page) for r in range(length + n)]
        pg, row = np.array([w[0] for w in where]), np.array([w[1] for w in where])
        for j in range(n):
            see = np.array(list(range(length)) + [length + x for x in root_path(parent[b], j)])
            for h in range(hq):
                c = h // (hq // hkv)
                keys = np.asarray(k_cache[pg[see], c, row[see]], np.float64)
                vals = np.asarray(v_cache[pg[see], c, row[see]], np.float64)
                s = scale * (keys @ np.asarray(q[b, j, h], np.float64))
                p = np.exp(s - s.max())
                p /= p.sum()
                o[b, j, h] = p @ vals
                a[b, j, h] = p @ np.abs(vals)
    return o, a


def commit(cache, path, accepted, table, lens):
    """A pool's bits (any dtype) [layers][pages][kv heads][page][D] after the move."""
    out = cache.copy()
    page = cache.shape[3]
    for b in range(len(lens)):
        for t in range(int(accepted[b])):
            sp, sr = row_of(table[b], int(lens[b]) + int(path[b][t]), page)
            dp, dr = row_of(table[b], int(lens[b]) + t, page)
            out[:, dp, :, dr] = cache[:, sp, :, sr]
    return out


def page_copy(cache, src, dst, rows=None):
    out = cache.copy()
    for i, (s, d) in enumerate(zip(src, dst)):
        r = cache.shape[3] if rows is None else int(rows[i])
        out[:, d, :, :r] = cache[:, s, :, :r]
    return out
