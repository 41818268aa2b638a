"""Oracle of the paged KV cache: the step's plan as a plain account, the write and the attention in fp64, from their
definitions (test infrastructure only)."""
from __future__ import annotations

import numpy as np


def plan(table, length, parent, ring, state, new, page, rows):
    """The step as a plain account, sequence by sequence. Returns (table, length, ring, state, cu, slots, positions)."""
    table, length, ring = table.copy(), length.astype(np.int64), ring.copy()
    first, spare = (int(x) for x in state)
    pages, n = len(ring), np.maximum(new, 0).astype(np.int64)
    cu = np.concatenate([[0], np.cumsum(n)])
    slots, positions = np.full(rows, -1, np.int64), np.full(rows, -1, np.int64)
    take = first
    old = table.copy()
    for i in range(len(new)):
        for k in range(-(-length[i] // page), -(-(length[i] + n[i]) // page)):
            table[i, k] = ring[take % pages]
            take += 1
        at = length[i] + np.arange(n[i])
        slots[cu[i]:cu[i + 1]] = table[i, at // page].astype(np.int64) * page + at % page
        before = length[parent[i]] + n[parent[i]] if parent[i] >= 0 else 0
        positions[cu[i]:cu[i + 1]] = at + before
    back = 0
    for i in np.flatnonzero(new < 0):
        for k in range(-(-length[i] // page)):
            ring[(first + spare + back) % pages] = old[i, k]
            back += 1
    taken = take - first
    out = np.where(new < 0, 0, length + n)
    return table, out, ring, np.array([(first + taken) % pages, spare - taken + back]), cu, slots, positions


def attention(q, k_of, v_of, parent, length, new, scale, group):
    """q [rows, Hq, d]; k_of(i), v_of(i): all tokens of sequence i after the step, [tokens, Hkv, d]. Returns
    (o, lse, mag, size): mag = sum_j p_j |v_j| like o, size = max_j scale sum |q| |k_j| like lse, for error bounds."""
    rows, hq, d = q.shape
    o, mag = np.zeros_like(q), np.zeros_like(q)
    lse, size = np.zeros((hq, rows)), np.zeros((hq, rows))
    cu = np.concatenate([[0], np.cumsum(np.maximum(new, 0))])
    for i in range(len(new)):
        a, b = cu[i], cu[i + 1]
        if a == b:
            continue
        k, v = k_of(i), v_of(i)
        before = int(length[i])
        if parent[i] >= 0:
            kp, vp = k_of(parent[i]), v_of(parent[i])
            k, v, before = np.concatenate([kp, k]), np.concatenate([vp, v]), before + len(kp)
        seen = np.arange(len(k))[None] <= before + np.arange(b - a)[:, None]
        for h in range(hq):
            x, kh, vh = q[a:b, h], k[:, h // group], v[:, h // group]
            s = np.where(seen, scale * (x @ kh.T), -np.inf)
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            z = p.sum(1, keepdims=True)
            p /= z
            o[a:b, h], mag[a:b, h] = p @ vh, p @ abs(vh)
            lse[h, a:b] = (top + np.log(z))[:, 0]
            size[h, a:b] = np.where(seen, scale * (abs(x) @ abs(kh).T), 0).max(1)
    return o, lse, mag, size
