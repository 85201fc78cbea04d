"""Serving from a paged cache in 64 bits, from the definitions: norm, rotation,
storing in pages, causal attention over pages.  NumPy, one loop per sequence;
pages out of range hold nothing."""
from __future__ import annotations

import numpy as np

D = 128


def norm(x, w, eps):
    """w x / sqrt(mean(x^2) + eps) over the last axis."""
    x = np.asarray(x, np.float64)
    return np.asarray(w, np.float64) * x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def pair_axes(sections):
    """Position axis of each of the 64 pairs."""
    return np.repeat(np.arange(len(sections)), sections)


def rotate(x, positions, theta, sections=(64,), interleaved=False):
    """x [..., tokens, heads, 128] turned by positions [axes, tokens]."""
    x = np.asarray(x, np.float64)
    half = D // 2
    angle = np.asarray(positions, np.float64)[pair_axes(sections)].T * theta ** (-np.arange(half) / half)
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]  # [tokens, 1, 64]
    y = np.empty_like(x)
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        y[..., 0::2], y[..., 1::2] = ya, yb
    else:
        y[..., :half], y[..., half:] = ya, yb
    return y


def place(page_table, s, j, page_size, n_pages):
    """Row of the pool of token j of sequence s, or None where its page is none."""
    if j < 0 or j // page_size >= page_table.shape[1]:
        return None
    page = int(page_table[s, j // page_size])
    return page * page_size + j % page_size if 0 <= page < n_pages else None


def length(seq_lens, s, max_len):
    return min(max(int(seq_lens[s]), 0), max_len)


def new_places(page_table, seq_lens, cu_new, page_size, n_pages, max_len):
    """Row of the pool of every new token (None: dropped)."""
    rows = []
    for s in range(len(cu_new) - 1):
        n, at = int(cu_new[s + 1] - cu_new[s]), length(seq_lens, s, max_len)
        rows += [place(page_table, s, at - n + t, page_size, n_pages) for t in range(n)]
    return rows


def visible_rows(page_table, s, count, page_size, n_pages):
    """(token indices, pool rows) of the first `count` tokens of sequence s that lie in pages."""
    got = [(j, place(page_table, s, j, page_size, n_pages)) for j in range(count)]
    got = [(j, r) for j, r in got if r is not None]
    return np.array([j for j, _ in got], np.int64), np.array([r for _, r in got], np.int64)


def attention(q, k, v, page_table, seq_lens, cu_new, max_len, scale, group):
    """q [total_new, q_heads, 128], k, v [kv_heads, n_pages, page, 128] of one layer, 64 bits.  Returns out, and
    per output sum_j p_j |v_j|, the number of keys and max_j scale sum_c |q_c k_jc| (what errors scale with)."""
    n_pages, page = k.shape[1:3]
    kf, vf = k.reshape(k.shape[0], -1, D), v.reshape(v.shape[0], -1, D)
    out = np.zeros(q.shape, np.float64)
    weight = np.zeros(q.shape, np.float64)
    keys = np.zeros(q.shape[:2], np.int64)
    dot = np.zeros(q.shape[:2], np.float64)
    for s in range(len(cu_new) - 1):
        n, size = int(cu_new[s + 1] - cu_new[s]), length(seq_lens, s, max_len)
        at, rows = visible_rows(page_table, s, size, page, n_pages)
        for t in range(n):
            m = int(np.searchsorted(at, size - n + t, side="right"))
            if m == 0:
                continue
            i = int(cu_new[s]) + t
            for h in range(k.shape[0]):
                g = slice(h * group, (h + 1) * group)
                kr, vr = kf[h, rows[:m]], vf[h, rows[:m]]
                x = scale * (q[i, g] @ kr.T)
                p = np.exp(x - x.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[i, g] = p @ vr
                weight[i, g] = p @ np.abs(vr)
                keys[i, g] = m
                dot[i, g] = scale * (np.abs(q[i, g]) @ np.abs(kr).T).max(-1)
    return out, weight, keys, dot
