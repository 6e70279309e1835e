"""fp64 numpy oracle of the inference calls: rotary positions with several axes, new tokens written to a paged cache,
attention over it, and the bookkeeping of its pages.  Written from the definitions, with plain loops; shares no code with the
HIP path."""
import math

import numpy as np


def rotary(x, positions, sections, theta, inverse=False):
    """x [rows, heads, d], positions [n_axes, rows]: pair (i, i + d/2) turned by positions[axis of i] * theta^(-2i/d)."""
    x = np.asarray(x, dtype=np.float64)
    rows, _, d = x.shape
    y = np.empty_like(x)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    assert len(axis) == d // 2
    for i, a in enumerate(axis):
        angle = np.asarray(positions[a], dtype=np.float64) * theta ** (-2.0 * i / d) * (-1 if inverse else 1)
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[:, :, i] = x[:, :, i] * c - x[:, :, i + d // 2] * s
        y[:, :, i + d // 2] = x[:, :, i + d // 2] * c + x[:, :, i] * s
    return y


def new_rows(lengths, cu_new=None):
    """(row, sequence, token number) of every new token."""
    out = []
    for s, n in enumerate(lengths):
        first, last = (s, s + 1) if cu_new is None else (cu_new[s], cu_new[s + 1])
        out += [(r, s, n - (last - first) + r - first) for r in range(first, last)]
    return out


def append(k_pool, v_pool, table, page_size, lengths, cu_new, k, v):
    """Pools [n_pages, heads, page_size, d] changed in place."""
    for r, s, c in new_rows(lengths, cu_new):
        if c < 0:
            continue
        page = table[s][c // page_size]
        if 0 <= page < len(k_pool):
            k_pool[page, :, c % page_size] = k[r]
            v_pool[page, :, c % page_size] = v[r]


def attention(q, k_pool, v_pool, table, page_size, lengths, cu_new, scale):
    """q [rows, Hq, d] -> (O [rows, Hq, d], LSE [Hq, rows], size) with NaN in rows that belong to no sequence; size: a bound of
    sum |q_i k_i| scale over the visible keys, and of |v|, by row and head, for tolerances."""
    rows, hq, d = q.shape
    hkv = k_pool.shape[1]
    o, lse = np.full((rows, hq, d), np.nan), np.full((hq, rows), np.nan)
    s_size, v_size = np.zeros((rows, hq)), np.zeros((rows, hq))
    for r, s, c in new_rows(lengths, cu_new):
        at = [(table[s][j // page_size], j % page_size) for j in range(c + 1)]
        at = [(p, j) for p, j in at if 0 <= p < len(k_pool)]
        for h in range(hq):
            if not at:
                o[r, h], lse[h, r] = 0.0, -math.inf
                continue
            p, j = np.array(at).T
            k, v = k_pool[p, h // (hq // hkv), j].astype(np.float64), v_pool[p, h // (hq // hkv), j].astype(np.float64)
            x = k @ q[r, h].astype(np.float64) * scale
            top = x.max()
            e = np.exp(x - top)
            lse[h, r] = top + math.log(e.sum())
            o[r, h] = e @ v / e.sum()
            s_size[r, h], v_size[r, h] = (np.abs(k) @ np.abs(q[r, h].astype(np.float64)) * scale).max(), np.abs(v).max()
    return o, lse, s_size, v_size


class Pages:
    """Which sequences hold which pages, as sets: what the bookkeeping has to agree with."""

    def __init__(self, n_pages, page_size):
        self.n_pages, self.page_size, self.held = n_pages, page_size, {}

    def holders(self, page):
        return sum(pages.count(page) for pages in self.held.values())

    def used(self):
        return {p for pages in self.held.values() for p in pages}
