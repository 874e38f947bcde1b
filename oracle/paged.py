"""fp64 NumPy oracle of the rotation by positions with several axes and of attention over a cache of pages.

Written from the definitions: angles per pair, one softmax per row over the keys that it sees.  Nothing here is shared with
the library.
"""
from __future__ import annotations

import numpy as np


def rotate_axes(x, positions, pairs, theta=10000.0, halves=True, shared=True, inverse=False):
    """x [..., n, d], positions [axes, n] -> the rotated copy, fp64."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    P, p = sum(pairs), 0
    for a, count in enumerate(pairs):
        for i in range(count):
            rate = theta ** (-(p / P) if shared else -(i / count))
            angle = np.asarray(positions[a], dtype=np.float64) * rate * (-1.0 if inverse else 1.0)
            u, v = (p, p + P) if halves else (2 * p, 2 * p + 1)
            y[..., u] = x[..., u] * np.cos(angle) - x[..., v] * np.sin(angle)
            y[..., v] = x[..., u] * np.sin(angle) + x[..., v] * np.cos(angle)
            p += 1
    return y


def sees(p, length, causal, window, n_sink):
    """Which of the tokens 0 .. length - 1 the token at place p sees."""
    j = np.arange(max(length, 0))
    ok = np.ones(j.shape, dtype=bool)
    if causal:
        ok &= j <= p
    if window:
        ok &= (j > p - window) | (j < n_sink)
    return ok


def slots(lengths, cu, s, page_tokens, table, n_pages):
    """(page, place in it) of every token of sequence s, None where there is no page."""
    most = table.shape[1] * page_tokens
    out = []
    for j in range(min(int(lengths[s]), most)):
        page = int(table[s, j // page_tokens])
        out.append((page, j % page_tokens) if 0 <= page < n_pages else None)
    return out


def append(K_pages, V_pages, K_new, V_new, cu, lengths, table):
    """The pages after the new tokens' keys and values (already rotated) are in them; pages [n, heads_kv, tokens, d]."""
    K, V = K_pages.copy(), V_pages.copy()
    for s in range(len(lengths)):
        m = int(cu[s + 1] - cu[s])
        for i in range(m):
            j = int(lengths[s]) - m + i
            if j < 0 or j >= table.shape[1] * K.shape[2]:
                continue
            page = int(table[s, j // K.shape[2]])
            if 0 <= page < K.shape[0]:
                K[page, :, j % K.shape[2]] = K_new[cu[s] + i]
                V[page, :, j % K.shape[2]] = V_new[cu[s] + i]
    return K, V


def attend(Q, K_pages, V_pages, cu, lengths, table, causal=True, window=0, n_sink=0, scale=None):
    """Q [rows, heads, d] -> O, lse2 [heads, rows], spread = sum_j p_j |v_j| and, per (row, head), the largest sum_f |q_f k_f| and
    the keys seen: what rounding bounds are made of.  Rows of no sequence: NaN."""
    n, H, d = Q.shape
    P, Hk = K_pages.shape[2], K_pages.shape[1]
    scale = 1.0 / np.sqrt(d) if not scale else scale
    O, spread = np.full((n, H, d), np.nan), np.full((n, H, d), np.nan)
    lse2, size, count = np.full((H, n), np.nan), np.zeros((n, H)), np.zeros(n, dtype=int)
    for s in range(len(lengths)):
        m = int(cu[s + 1] - cu[s])
        if m == 0:
            continue
        at = slots(lengths, cu, s, P, table, K_pages.shape[0])
        held = np.array([a is not None for a in at], dtype=bool)
        pages = np.array([a[0] if a else 0 for a in at], dtype=int)
        inside = np.array([a[1] if a else 0 for a in at], dtype=int)
        for i in range(m):
            row, p = int(cu[s]) + i, int(lengths[s]) - m + i
            ok = np.nonzero(sees(p, len(at), causal, window, n_sink) & held)[0]
            count[row] = len(ok)
            for h in range(H):
                if len(ok) == 0:
                    O[row, h], spread[row, h], lse2[h, row] = 0.0, 0.0, np.inf
                    continue
                k, v = K_pages[pages[ok], h * Hk // H, inside[ok]], V_pages[pages[ok], h * Hk // H, inside[ok]]
                logit = (k @ Q[row, h]) * scale
                size[row, h] = (np.abs(k) @ np.abs(Q[row, h])).max() * scale
                top = logit.max()
                w = np.exp(logit - top)
                lse2[h, row] = (np.log(w.sum()) + top) / np.log(2.0)
                O[row, h] = (w / w.sum()) @ v
                spread[row, h] = (w / w.sum()) @ np.abs(v)
    return O, lse2, spread, size, count
