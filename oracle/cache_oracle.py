"""fp64 oracle of the operators around the verification step: appending to the cache with rotation,
attention of new tokens over the cache, sampling.  One function per definition (include/svf_cache.h,
include/svf_rules.h), numpy on the CPU, loops over sequences, heads and rows."""
from __future__ import annotations

import math

import numpy as np


def sequences(seq_lens, new_rows, new_lens, max_seq_len, max_new, n_rows):
    """(sequence, cached tokens, first row, new tokens) of the sequences that take part."""
    out = []
    for b, (L, r, n) in enumerate(zip(seq_lens, new_rows, new_lens)):
        n = min(n, max_new, n_rows - r, max_seq_len - L)
        if L >= 0 and 0 <= r < n_rows and n > 0:
            out.append((b, int(L), int(r), int(n)))
    return out


def place(t, b, table, page_size):
    """(page, slot) of place t of sequence b."""
    return (b, t) if page_size == 0 else (int(table[b][t // page_size]), t % page_size)


def rotate(x, position, inv_freq, interleaved, scale=1.0):
    """x fp64 [..., d]: the leading 2 * len(inv_freq) channels turned by position * inv_freq."""
    half = len(inv_freq)
    y = x.copy()
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = np.cos(position * inv_freq), np.sin(position * inv_freq)
    y[..., a] = scale * (x[..., a] * c - x[..., b] * s)
    y[..., b] = scale * (x[..., b] * c + x[..., a] * s)
    return y


def attend(q, K, V, table, page_size, seqs, G, scale, window=0):
    """q [n_rows][Hq][d], K, V [pages][slots][Hkv][d], fp64.  For every (row, head) of a sequence: the output, the
    log-sum-exp, the weighted sum of |V|, and the largest scaled sum of |q_c k_c| of its tokens."""
    n_rows, Hq, d = q.shape
    out, mag = np.zeros_like(q), np.zeros_like(q)
    lse, size = np.zeros((n_rows, Hq)), np.zeros((n_rows, Hq))
    for b, L, r, n in seqs:
        at = [place(t, b, table, page_size) for t in range(L + n)]
        pg, sl = np.array([a[0] for a in at]), np.array([a[1] for a in at])
        for h in range(Hq):
            k, v = K[pg, sl, h // G], V[pg, sl, h // G]
            for j in range(n):
                lo = max(0, L + j + 1 - window) if window else 0
                ks, vs = k[lo:L + j + 1], v[lo:L + j + 1]
                x = ks @ q[r + j, h] * scale
                m = x.max()
                w = np.exp(x - m)
                out[r + j, h] = w @ vs / w.sum()
                mag[r + j, h] = w @ np.abs(vs) / w.sum()
                lse[r + j, h] = m + math.log(w.sum())
                size[r + j, h] = (np.abs(ks) @ np.abs(q[r + j, h])).max() * scale
    return out, lse, mag, size


def kept(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens that one row of logits (fp64) keeps, in descending order, their weights, and how near the nearest
    token was to the top-p border (share of the top-k mass)."""
    x = np.where(np.isnan(x), -np.inf, x)
    if not temperature > 0:
        temperature, top_k = 1.0, 1
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        z = np.where(x == top, 0.0, (x - top) / temperature)
    z = np.where((x == -np.inf) & (top > -np.inf), -np.inf, z)      # (whatever the temperature)
    w = np.exp(z)
    if top_k > 0:
        order = order[:top_k]
    gap = np.inf
    if top_p < 1:
        mass = np.cumsum(w[order])
        before = np.concatenate(([0.0], mass[:-1]))
        gap = np.abs(before[1:] - top_p * mass[-1]).min(initial=np.inf) / mass[-1]
        keep = before < top_p * mass[-1]
        keep[0] = True
        order = order[keep]
    if min_p > 0:
        order = order[x[order] >= min(top, top + temperature * math.log(min_p))]
    order = order[x[order] > -np.inf]
    return order, w[order], gap


def draw(order, w, u, V):
    """(token, cumulative weights by index, target)."""
    full = np.zeros(V)
    full[order] = w
    cdf = np.cumsum(full)
    target = u * cdf[-1]
    return int(min(np.searchsorted(cdf, target, side="right"), order.max())), cdf, target
