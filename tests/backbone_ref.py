"""The language backbone's operators restated in numpy and 64 bits, request by request, for the GPU tests."""
from __future__ import annotations

import numpy as np

# half a unit in the last place, relative to the value
UNIT = {"bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def step_plan(held, base, new, parent, ring, ring_in, table, page, max_rows, mask_words):
    """cu, req, slot, pos, mask, ring, ring_out, table, status."""
    held, base, new = (np.asarray(a, np.int64) for a in (held, base, new))
    ring, table = np.array(ring, np.int64), np.array(table, np.int64)
    n, places, cols = len(held), len(ring), table.shape[1]
    head, count = int(ring_in[0]), int(ring_in[1])
    ok = (held >= 0) & (base >= 0) & (new >= 0)
    have, need = -(-held // page), -(-(base + new) // page)
    fits = ok & (have <= cols) & (need <= cols)
    status = (0 if ok.all() else 8) | (0 if (fits | ~ok).all() else 2)
    grow = np.where(fits, np.maximum(need - have, 0), 0)
    back = np.where(fits, np.maximum(have - need, 0), 0)
    if np.where(ok, new, 0).sum() > max_rows:
        status |= 4
    if not (0 <= head < places and 0 <= count <= places):
        status |= 8
    elif grow.sum() > count:
        status |= 1
    elif count - grow.sum() + back.sum() > places:
        status |= 8
    cu = np.zeros(n + 1, np.int64)
    req, slot = np.full(max_rows, -1), np.full(max_rows, -1)
    pos, mask = np.zeros(max_rows, np.int64), np.zeros((max_rows, mask_words), np.uint32)
    if status:
        return cu, req, slot, pos, mask, ring, np.array([head, count]), table, status
    cu[1:] = np.cumsum(new)
    taken, put = head, head + count
    given = []
    for i in range(n):
        for k in range(have[i], need[i]):
            table[i, k] = ring[taken % places]
            taken += 1
        for k in range(need[i], have[i]):
            given.append((put % places, table[i, k]))
            put += 1
        for j in range(new[i]):
            r, at = cu[i] + j, base[i] + j
            req[r], slot[r] = i, table[i, at // page] * page + at % page
            line = [j]
            if parent is None:
                line = list(range(j + 1))
            else:
                while 0 <= parent[cu[i] + line[-1]] < line[-1]:
                    line.append(int(parent[cu[i] + line[-1]]))
            pos[r] = base[i] + len(line) - 1
            for k in line:
                if k < 32 * mask_words:
                    mask[r, k // 32] |= np.uint32(1) << np.uint32(k % 32)
    for at, page_id in given:
        ring[at] = page_id
    return cu, req, slot, pos, mask, ring, np.array([taken % places, put - taken]), table, 0


def _pairs(rot, interleaved):
    f = np.arange(rot // 2)
    return (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)


def rope(x, weight, pos, freq, axis, rot, interleaved, eps):
    """x [rows, heads, dim], pos [axes, rows]."""
    y = np.array(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    if rot:
        a = (np.asarray(pos, np.float64)[axis] * np.asarray(freq, np.float64)[:, None]).T[:, None]
        i, j = _pairs(rot, interleaved)
        u, v = y[..., i].copy(), y[..., j].copy()
        y[..., i], y[..., j] = u * np.cos(a) - v * np.sin(a), v * np.cos(a) + u * np.sin(a)
    return y


def rope_backward(g, x, weight, pos, freq, axis, rot, interleaved, eps):
    """dx, dweight."""
    y = rope(g, None, -np.asarray(pos, np.int64), freq, axis, rot, interleaved, eps)
    if weight is None:
        return y, None
    x, w = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    u = y * w
    return r * u - x * r ** 3 * (u * x).mean(-1, keepdims=True), (y * x * r).sum((0, 1))


def attention(q, k_new, v_new, k_cache, v_cache, table, lengths, cu, sees, scale):
    """out, lse and sum_j p_j |v_j| / sum_j p_j (for error bounds); caches [pages, page, heads, dim], sees(i, n):
    which new rows each of request i's n new rows sees.  What a row does not see is left out of its sums."""
    rows, heads, dim = q.shape
    group, page = heads // k_cache.shape[2], k_cache.shape[1]
    out, size, lse = np.zeros(q.shape), np.zeros(q.shape), np.full((rows, heads), -np.inf)
    for i in range(len(lengths)):
        lo, hi, n = cu[i], cu[i + 1], int(lengths[i])
        at = np.arange(n)
        pages = np.asarray(table[i])[at // page]
        vis = sees(i, hi - lo)
        for h in range(heads):
            kc, vc = (c[pages, at % page, h // group].astype(np.float64) for c in (k_cache, v_cache))
            for r in range(lo, hi):
                new = np.nonzero(vis[r - lo])[0] + lo
                k = np.concatenate([kc, k_new[new, h // group].astype(np.float64)])
                v = np.concatenate([vc, v_new[new, h // group].astype(np.float64)])
                if not len(k):
                    continue
                s = k @ q[r, h].astype(np.float64) * scale
                m = s.max()
                p = np.exp(s - m)
                lse[r, h] = m + np.log(p.sum())
                out[r, h] = p @ v / p.sum()
                size[r, h] = p @ np.abs(v) / p.sum()
    return out, lse, size


def ancestors(parent):
    """Which nodes of one tree each node sees: itself and its ancestors."""
    n = len(parent)
    m = np.zeros((n, n), bool)
    for j in range(n):
        m[j, j] = True
        if 0 <= parent[j] < j:
            m[j] |= m[parent[j]]
    return m


def words(vis, mask_words):
    """Rows of truth values packed into int32 words."""
    out = np.zeros((vis.shape[0], mask_words), np.uint32)
    for r, k in zip(*np.nonzero(vis)):
        out[r, k // 32] |= np.uint32(1) << np.uint32(k % 32)
    return out.view(np.int32)
