"""fp64 oracle of the paged key-value cache (TEST INFRASTRUCTURE ONLY): numpy, one sequence and one head at a time, nothing blocked.

Only ``tests/`` may import this module.  It imports nothing from the HIP package.

Slot j of a sequence is row j % P of page table[j // P]; a page outside [0, n_pages) is not there.

Pins: ``tests/test_oracle_paged_pins.py``.
"""
from __future__ import annotations

import math

import numpy as np


def rope(x, position, theta, style=0):
    """x [..., d] turned by position: pair i by the angle position * theta^(-2i/d); pairs (i, i + d/2), or (2i, 2i + 1)."""
    x = np.asarray(x, np.float64)
    d = x.shape[-1]
    a = float(position) * float(theta) ** (-2.0 * np.arange(d // 2) / d)
    first, second = (np.arange(0, d, 2), np.arange(1, d, 2)) if style else (np.arange(d // 2), np.arange(d // 2, d))
    y = np.empty_like(x)
    y[..., first] = x[..., first] * np.cos(a) - x[..., second] * np.sin(a)
    y[..., second] = x[..., first] * np.sin(a) + x[..., second] * np.cos(a)
    return y


def slots(table_row, P, n, n_pages):
    """(page, row, there) of the first n slots."""
    j = np.arange(n)
    page = np.asarray(table_row)[j // P] if n else np.zeros(0, int)
    return page, j % P, (page >= 0) & (page < n_pages)


def attend(q, position, K, V, there, theta, style=0):
    """q [H, d] pre-RoPE; K, V [n, H_kv, d] (K rotated); there [n].  Returns (out [H, d], p [H, n])."""
    H, d = q.shape
    n, H_kv = K.shape[:2]
    q = rope(q, position, theta, style)
    out, p = np.zeros((H, d)), np.zeros((H, n))
    if not np.any(there):
        return out, p
    for h in range(H):
        g = h // (H // H_kv)
        x = (K[there, g] @ q[h]) / math.sqrt(d)
        e = np.exp(x - x.max())
        p[h, there] = e / e.sum()
        out[h] = p[h, there] @ V[there, g]
    return out, p


def list_weights(p, lists):
    """Softmax weights [H, n] added up over the query heads of each of `lists` lists."""
    return p.reshape(lists, p.shape[0] // lists, -1).sum(axis=1)


def evict(weights, pos, position, n_keep, n_sink, n_recent):
    """One list of n slots: for each slot of the shortened list, the slot that it is taken from."""
    n = len(weights)
    if n <= n_keep:
        return list(range(n))

    def rank(j):
        protected = int(pos[j]) < n_sink or int(pos[j]) > int(position) - n_recent
        w = float(weights[j])
        return (0 if protected else 1, 0.0 if protected else (math.inf if math.isnan(w) else -w), 1 if math.isnan(w) and not protected else 0, j)

    kept = set(sorted(range(n), key=rank)[:n_keep])
    late = [j for j in range(n_keep, n) if j in kept]
    return [j if j in kept else late.pop(0) for j in range(n_keep)]
