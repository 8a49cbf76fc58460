"""The paged cache's operators in float64 numpy, a position or a page at a time."""
from __future__ import annotations

import math

import numpy as np


def _spans(kv_len, new_start, max_new, table, page_size, n_new):
    """(b, first row, rows computed, position of the first) of each sequence; the
    rows are of the packed axis (b * max_new + i without new_start)."""
    most = table.shape[1] * page_size
    for b in range(table.shape[0]):
        kv = min(max(int(kv_len[b]), 0), most)
        if new_start is None:
            s, count = b * max_new, max_new
        else:
            s = min(max(int(new_start[b]), 0), n_new)
            count = min(max(int(new_start[b + 1]), s), n_new) - s
        yield b, s, min(count, max_new), kv - count


def _page(table, b, pos, page_size, n_pages):
    p = int(table[b, pos // page_size])
    return p if 0 <= p < n_pages else -1


def _row(pool, layout, page, slot):
    """[H][D] of a position, of one layer's pool."""
    return pool[page, :, slot] if layout else pool[page, slot]


def paged_attention(q, k_pages, v_pages, table, kv_len, o, new_start=None, max_new=None, window=0, scale=None,
                    layout=0):
    """o [rows][H_q][D] with the rows of the new tokens computed (q alike), and the
    pair (sum of softmax |v|, largest scale sum |q k|) of every element, for
    error bounds."""
    o, mag, smax = o.copy(), np.zeros(o.shape), np.zeros(o.shape)
    n_pages, D = k_pages.shape[0], q.shape[-1]
    H_kv, ps = (k_pages.shape[1], k_pages.shape[2]) if layout else (k_pages.shape[2], k_pages.shape[1])
    G = q.shape[1] // H_kv
    scale = scale or 1 / math.sqrt(D)
    max_new = q.shape[0] if max_new is None else max_new
    for b, s, n, at in _spans(kv_len, new_start, max_new, table, ps, q.shape[0]):
        for i in range(n):
            u = at + i
            see = [v for v in range(max(0, u - window + 1) if window else 0, u + 1)
                   if _page(table, b, v, ps, n_pages) >= 0]
            if not see:
                o[s + i] = 0
                continue
            where = [(_page(table, b, v, ps, n_pages), v % ps) for v in see]
            K = np.stack([_row(k_pages, layout, *w) for w in where])      # [N][H_kv][D]
            V = np.stack([_row(v_pages, layout, *w) for w in where])
            for h in range(q.shape[1]):
                x = scale * (K[:, h // G] @ q[s + i, h])
                p = np.exp(x - x.max())
                p /= p.sum()
                o[s + i, h] = p @ V[:, h // G]
                mag[s + i, h] = p @ np.abs(V[:, h // G])
                smax[s + i, h] = scale * (np.abs(K[:, h // G]) @ np.abs(q[s + i, h])).max()
    return o, mag, smax


def _ready(x, gain, eps, inv_freq, pos, interleaved):
    """One head row normed and turned."""
    x = x.copy()
    if gain is not None:
        x = x / math.sqrt((x * x).mean() + eps) * gain
    if inv_freq is not None:
        for r, f in enumerate(inv_freq):
            i, j = (2 * r, 2 * r + 1) if interleaved else (r, r + len(inv_freq))
            c, s = math.cos(pos * float(f)), math.sin(pos * float(f))
            x[i], x[j] = x[i] * c - x[j] * s, x[j] * c + x[i] * s
    return x


def cache_append(q, k, v, q_out, k_pages, v_pages, table, kv_len, new_start=None, max_new=None, q_gain=None,
                 k_gain=None, eps=1e-6, inv_freq=None, interleaved=False, positions=None, layout=0):
    """(q_out, k_pages, v_pages) after the call: rows [L][rows][heads][D], pools
    [L][n_pages] x page, gains [L][D]."""
    q_out = None if q is None else q_out.copy()
    k_pages, v_pages = k_pages.copy(), v_pages.copy()
    L, n_pages = k_pages.shape[:2]
    ps = k_pages.shape[3] if layout else k_pages.shape[2]
    some = q if k is None else k
    max_new = some.shape[1] if max_new is None else max_new
    for b, s, n, at in _spans(kv_len, new_start, max_new, table, ps, some.shape[1]):
        for i in range(n):
            u = at + i
            turn = u if positions is None else int(positions[s + i])
            page = _page(table, b, u, ps, n_pages) if u >= 0 else -1
            for l in range(L):
                if q is not None:
                    for h in range(q.shape[2]):
                        q_out[l, s + i, h] = _ready(q[l, s + i, h], None if q_gain is None else q_gain[l], eps, inv_freq,
                                                    turn, interleaved)
                if k is not None and page >= 0:
                    for h in range(k.shape[2]):
                        _row(k_pages[l], layout, page, u % ps)[h] = _ready(
                            k[l, s + i, h], None if k_gain is None else k_gain[l], eps, inv_freq, turn, interleaved)
                        _row(v_pages[l], layout, page, u % ps)[h] = v[l, s + i, h]
    return q_out, k_pages, v_pages


def cache_reorder(k_pages, v_pages, table, source, keep, want, layout=0):
    """(k_pages, v_pages, new table, missing)."""
    pools = [k_pages.copy(), v_pages.copy()]
    n_pages, ps = k_pages.shape[1], k_pages.shape[3] if layout else k_pages.shape[2]
    B, M = table.shape
    rows, whole, part = [], set(), {}
    for b, s in enumerate(source):
        k = min(max(int(keep[b]), 0), M * ps) if 0 <= s < B else 0
        w = max(min(int(want[b]), M * ps), k)
        ids = [int(p) if 0 <= p < n_pages else -1 for p in (table[s] if 0 <= s < B else [])][:-(-k // ps)]
        rows.append((ids, k, -(-w // ps)))
        whole |= set(ids[:k // ps])
        if k % ps and ids[-1] >= 0:
            part.setdefault(ids[-1], b)
    free = [p for p in range(n_pages) if p not in whole and p not in part]
    new, missing = np.full((len(rows), M), -1, np.int32), 0

    def give():
        nonlocal missing
        if free:
            return free.pop(0)
        missing += 1
        return -1

    for b, (ids, k, need) in enumerate(rows):
        ids = list(ids)
        if k % ps and ids[-1] >= 0 and (ids[-1] in whole or part[ids[-1]] != b):
            to = give()
            if to >= 0:
                for pool, orig in zip(pools, (k_pages, v_pages)):
                    if layout:
                        pool[:, to, :, :k % ps] = orig[:, ids[-1], :, :k % ps]
                    else:
                        pool[:, to, :k % ps] = orig[:, ids[-1], :k % ps]
            ids[-1] = to
        while len(ids) < need:
            ids.append(give())
        new[b, :len(ids)] = ids
    return pools[0], pools[1], new, missing


def cache_compact(k_pages, v_pages, table):
    """(k_pages, v_pages, new table, used)."""
    pools = [k_pages.copy(), v_pages.copy()]
    n_pages = k_pages.shape[1]
    held = sorted({int(p) for p in table.ravel() if 0 <= p < n_pages})
    n = len(held)
    free = [p for p in range(n) if p not in set(held)]
    to = {p: p for p in held}
    for p in held:
        if p >= n:
            to[p] = free.pop(0)
            for pool, orig in zip(pools, (k_pages, v_pages)):
                pool[:, to[p]] = orig[:, p]
    new = np.array([[to.get(int(p), -1) for p in row] for row in table], np.int32).reshape(table.shape)
    return pools[0], pools[1], new, n
