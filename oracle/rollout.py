"""Rollouts and clipping, in fp64 from their definitions: keys and values written to a paged cache, attention of new tokens over
it, tokens drawn from logits, gradients clipped by the norm of all of them.  Axes as in the library's tensors.
"""
from __future__ import annotations

import numpy as np


def rotated(x, position, table, pairs):
    """x [h] turned by column `position` of table [r, N_pos] (r/2 cosines, then r/2 sines)."""
    if table is None:
        return x.copy()
    y, r = x.copy(), table.shape[0]
    for i in range(r // 2):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, i + r // 2)
        c, s = table[i, position], table[r // 2 + i, position]
        y[a], y[b] = x[a] * c - x[b] * s, x[a] * s + x[b] * c
    return y


def slot_of(position, b, pages, P, n_pages):
    """Where a position of sequence b lies along the cache's second axis (pages [max_pages, N_b]), or None."""
    if position < 0 or position >= pages.shape[0] * P:
        return None
    page = pages[position // P, b]
    return int(page) * P + position % P if 0 <= page < n_pages else None


def new_tokens(count, b, N_s):
    return N_s if count is None else min(max(int(count[b]), 0), N_s)


def cache_append(QKV, K, V, P, N_h, pages, start, count=None, table=None, pairs=False):
    """(K, V) [h, n_pages * P, N_kv] with the new tokens' keys and values; QKV [(N_h + 2 N_kv) h, N_s, N_b]."""
    K, V = K.copy(), V.copy()
    h, _, N_kv = K.shape
    for b in range(QKV.shape[2]):
        for s in range(new_tokens(count, b, QKV.shape[1])):
            p = int(start[b]) + s
            at = slot_of(p, b, pages, P, K.shape[1] // P)
            if at is None or (table is not None and p >= table.shape[1]):
                continue
            for j in range(N_kv):
                K[:, at, j] = rotated(QKV[(N_h + j) * h:(N_h + j + 1) * h, s, b], p, table, pairs)
                V[:, at, j] = QKV[(N_h + N_kv + j) * h:(N_h + N_kv + j + 1) * h, s, b]
    return K, V


def cache_attention(QKV, K, V, B, P, N_h, scale, pages, start, count=None, table=None, pairs=False, window=0):
    """(B, bound): B [N_h h, N_s, N_b] with the new tokens' columns overwritten; bound: for each element sum_k P |V|, then the largest
    sum_i |K| |Q| scale and |V| among the keys of its row (what errors of a product in fewer bits are measured against)."""
    B = B.copy()
    h, _, N_kv = K.shape
    mass, reach, largest = np.zeros_like(B), np.zeros_like(B), np.zeros_like(B)
    for b in range(QKV.shape[2]):
        for s in range(new_tokens(count, b, QKV.shape[1])):
            p = int(start[b]) + s
            seen = [slot_of(k, b, pages, P, K.shape[1] // P) for k in range(max(0, p - window + 1) if window else 0, p + 1)]
            seen = [k for k in seen if k is not None]
            if table is not None and p >= table.shape[1]:
                seen = []
            for j in range(N_h):
                rows = slice(j * h, (j + 1) * h)
                if not seen:
                    B[rows, s, b] = 0.0
                    continue
                q, g = rotated(QKV[rows, s, b], p, table, pairs), j // (N_h // N_kv)
                k, v = K[:, seen, g], V[:, seen, g]
                e = scale * (k.T @ q)
                w = np.exp(e - e.max())
                w /= w.sum()
                B[rows, s, b] = v @ w
                mass[rows, s, b] = np.abs(v) @ w
                reach[rows, s, b] = scale * (np.abs(k).T @ np.abs(q)).max()
                largest[rows, s, b] = np.abs(v).max()
    return B, (mass, reach, largest)


def sample_token(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log-probability) drawn from the logits x with the random number u."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    if x.max() == -np.inf:
        return -1, 0.0
    if x.max() == np.inf:
        x = np.where(x == np.inf, 0.0, -np.inf)
    shifted = x - x.max()
    logp = shifted - np.log(np.exp(shifted).sum())
    if temperature == 0.0:
        token = int(np.argmax(shifted == 0.0))
        return token, float(logp[token])
    e = np.exp(shifted / temperature)
    order = np.lexsort((np.arange(len(x)), -x))          # falling logits, among equals rising numbers
    order = order[:top_k] if top_k else order
    if top_p < 1.0:
        mass = np.cumsum(e[order])
        order = order[:int(np.argmax(mass >= top_p * mass[-1])) + 1]
    kept = np.sort(order[e[order] >= min_p])
    mass = np.cumsum(e[kept])
    u = 0.0 if not u >= 0.0 else min(float(u), 1.0 - 2.0 ** -24)
    token = int(kept[np.argmax(mass > u * mass[-1])])
    return token, float(logp[token])


def clip_grad_norm(G, max_norm, eps):
    """(clipped gradients, norm)"""
    norm = float(np.sqrt(sum(np.square(g.astype(np.float64)).sum() for g in G)))
    factor = min(1.0, max_norm / (norm + eps)) if np.isfinite(norm) else 1.0
    return [g.astype(np.float64) * factor for g in G], norm
