"""Plain float64 oracle of the packed prefill, the paged append with its rotation and the paged attention.

Written from the definitions in include/samkv.h, one sequence and one head at a time, in numpy; nothing here imports the
library.  Arrays are [heads, tokens, d]; pages are [n_pages, Hkv, page_size, d].
"""
from __future__ import annotations

import numpy as np


def spans(n_seq, n_rows, max_new, max_len, cu=None, lens=None):
    """(first row, rows, tokens) of every sequence under the bounds that the header states."""
    out = []
    for s in range(n_seq):
        if cu is None:
            first, n = s * max_new, max_new
        else:
            first = min(max(int(cu[s]), 0), n_rows)
            n = min(max(min(max(int(cu[s + 1]), 0), n_rows) - first, 0), max_new)
        out.append((first, n, n if lens is None else min(max(int(lens[s]), 0), max_len)))
    return out


def attend_rows(q, k, v, scale):
    """q [n, d] are the newest rows of the m keys k, v [m, d]: row t sees keys 0 .. m - n + t.  Returns out, lse, and for error
    bounds the same average of |v| and the largest sum of |q_c k_c| over the row's keys."""
    n, d = q.shape
    m = k.shape[0]
    out, lse = np.zeros((n, d)), np.full(n, -np.inf)
    mean_abs, size = np.zeros((n, d)), np.zeros(n)
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    for t in range(n):
        seen = m - n + t + 1
        if seen < 1:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            s = scale * (k[:seen] @ q[t])
            top = s.max()
            w = np.exp(s - top)
            total = w.sum()
            out[t] = (w[:, None] * v[:seen]).sum(0) / total
            mean_abs[t] = (w[:, None] * np.abs(v[:seen])).sum(0) / total
            lse[t] = top + np.log(total)
            size[t] = (np.abs(k[:seen]) @ np.abs(q[t])).max()
    return out, lse, mean_abs, size


class Attention:
    """Outputs of a batch and what an implementation may be off by; rows of no sequence are not `written`."""

    def __init__(self, hq, n_rows, d):
        self.out, self.lse = np.zeros((hq, n_rows, d)), np.full((hq, n_rows), -np.inf)
        self.mean_abs, self.size = np.zeros((hq, n_rows, d)), np.zeros((hq, n_rows))
        self.seen, self.written = np.zeros(n_rows, int), np.zeros(n_rows, bool)

    def put(self, h, first, n, m, results):
        for to, x in zip((self.out, self.lse, self.mean_abs, self.size), results):
            to[h, first:first + n] = x
        self.seen[first:first + n] = np.maximum(m - n + 1 + np.arange(n), 0)
        self.written[first:first + n] = True


def prefill(q, k, v, cu, max_len, scale):
    hq, n_rows, d = q.shape
    group = hq // k.shape[0]
    r = Attention(hq, n_rows, d)
    for first, n, _ in spans(len(cu) - 1, n_rows, max_len, max_len, cu):
        rows = slice(first, first + n)
        for h in range(hq):
            r.put(h, first, n, n, attend_rows(q[h, rows], k[h // group, rows], v[h // group, rows], scale))
    return r


def cached(pages, table_row, m, g):
    """[m, d]: the first m slots of a sequence, KV head g."""
    size = pages.shape[2]
    slots = np.arange(m)
    page = np.clip(np.asarray(table_row)[slots // size], 0, pages.shape[0] - 1)
    return pages[page, g, slots % size]


def paged_attention(k_pages, v_pages, table, lens, max_len, q, scale, max_new, cu=None):
    hq, n_rows, d = q.shape
    group = hq // k_pages.shape[1]
    r = Attention(hq, n_rows, d)
    for s, (first, n, m) in enumerate(spans(len(table), n_rows, max_new, max_len, cu, lens)):
        for h in range(hq):
            g = h // group
            r.put(h, first, n, m, attend_rows(q[h, first:first + n], cached(k_pages, table[s], m, g),
                                              cached(v_pages, table[s], m, g), scale))
    return r


def rotate(x, pos, inv_freq, interleaved):
    """x [heads, d] turned by pos * inv_freq[i], pair by pair."""
    y = x.astype(np.float64).copy()
    half = len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = float(pos) * float(inv_freq[i])
        c, s = np.cos(angle), np.sin(angle)
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
    return y


def append(k_pages, v_pages, table, lens, max_len, k_new, v_new, max_new, cu=None, inv_freq=None, interleaved=False,
           positions=None, q=None, q_out=None):
    """Returns new float64 copies of k_pages, v_pages and q_out (None without q)."""
    k_pages, v_pages = k_pages.astype(np.float64), v_pages.astype(np.float64)
    q_out = None if q is None else q_out.astype(np.float64)
    size = k_pages.shape[2]
    turn = (lambda x, pos: x.astype(np.float64)) if inv_freq is None else (lambda x, pos: rotate(x, pos, inv_freq, interleaved))
    for s, (first, n, m) in enumerate(spans(len(table), k_new.shape[1], max_new, max_len, cu, lens)):
        for t in range(n):
            i, slot = first + t, m - n + t
            pos = max(slot, 0) if positions is None else int(positions[i])
            if q is not None:
                q_out[:, i] = turn(q[:, i], pos)
            if slot < 0 or not 0 <= table[s][slot // size] < len(k_pages):
                continue
            k_pages[table[s][slot // size], :, slot % size] = turn(k_new[:, i], pos)
            v_pages[table[s][slot // size], :, slot % size] = v_new[:, i]
    return k_pages, v_pages, q_out
