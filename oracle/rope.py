"""Rotary positions in extended precision, pair by pair (Su et al. 2021)."""
from __future__ import annotations

import numpy as np


def angles(positions, turns):
    """Angles in radians, [tokens, pairs], reduced to a turn in 80-bit arithmetic."""
    t = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(turns, dtype=np.longdouble)[None, :]
    return ((t - np.rint(t)) * (2 * np.longdouble("3.14159265358979323846264"))).astype(np.float64)


def rotate(x, positions, turns, scale: float = 1.0, interleaved: bool = False, inverse: bool = False):
    """x [tokens, heads, d] with the pairs of its first 2 * len(turns) channels turned."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    n = len(turns)
    a = angles(positions, turns)
    if inverse:
        a = -a
    for i in range(n):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        c, s = scale * np.cos(a[:, i])[:, None], scale * np.sin(a[:, i])[:, None]
        y[:, :, p] = x[:, :, p] * c - x[:, :, q] * s
        y[:, :, q] = x[:, :, p] * s + x[:, :, q] * c
    return y


def pair_norms(x, n: int, interleaved: bool = False):
    """Per channel the length of its pair (the channel's own size where it is not rotated)."""
    x = np.asarray(x, dtype=np.float64)
    r = np.abs(x)
    for i in range(n):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, n + i)
        r[:, :, p] = r[:, :, q] = np.hypot(x[:, :, p], x[:, :, q])
    return r


def append(k_pages, v_pages, k, v, q_counts, kv_lens, page_lists):
    """Copies of the pools with each request's new tokens at the end of its keys."""
    kp, vp = np.array(k_pages), np.array(v_pages)
    P = kp.shape[1]
    t = 0
    for n, L, pages in zip(q_counts, kv_lens, page_lists):
        for j in range(L - n, L):
            kp[pages[j // P], j % P] = k[t]
            vp[pages[j // P], j % P] = v[t]
            t += 1
    return kp, vp
