"""Attention weights of cache rows, and eviction by them (oracle; test infrastructure only)."""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64, kv_head


def attend(q_bits, k, v, scale=None):
    """One query row [Hq, d] (bf16 bits) over k, v [n, Hkv, d] (float64): (out [Hq, d], the rows' weights
    averaged over the q-heads [n])."""
    q = bf16_bits_to_f64(q_bits)
    Hq, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, weight = np.zeros((Hq, d)), np.zeros(len(k))
    for h in range(Hq):
        g = kv_head(h, Hq, k.shape[1])
        s = scale * (k[:, g] @ q[h])
        p = np.exp(s - s.max())
        p /= p.sum()
        out[h] = p @ v[:, g]
        weight += p
    return out, weight / Hq


def kept_rows(weight, head, tail, budget):
    """Rows that stay, ascending: the first `head`, the last `tail`, and the heaviest others up to `budget` in
    all (of equal weights the lower row; NaN as -infinity)."""
    n = len(weight)
    if n <= budget:
        return np.arange(n)
    head = min(head, n)
    tail = min(tail, n - head)
    w = np.asarray(weight, np.float64)
    w = np.where(np.isnan(w), -np.inf, w)
    order = sorted(range(head, n - tail), key=lambda r: (-w[r], r))
    chosen = order[:max(budget - head - tail, 0)]
    return np.array(sorted(list(range(head)) + chosen + list(range(n - tail, n))), np.int64)
