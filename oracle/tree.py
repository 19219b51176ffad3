"""Steps over drafted tokens (oracle; test infrastructure only): trees given by parent places, the attention of their
nodes, the path that chosen tokens confirm, and the logits a sampler is given."""
from __future__ import annotations

import numpy as np

from .attention import kv_head


def path_of(parent, i):
    """Node i and its ancestors, upwards."""
    path = [i]
    while parent[path[-1]] >= 0:
        path.append(int(parent[path[-1]]))
    return path


def attend(q, k, v, k_new, v_new, parent, scale=None):
    """q [n, Hq, d]; cache rows k, v [L, Hkv, d]; nodes' rows k_new, v_new [n, Hkv, d] (all float64) -> [n, Hq, d]."""
    n, Hq, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out = np.empty((n, Hq, d))
    for i in range(n):
        own = sorted(path_of(parent, i))
        kk, vv = np.concatenate([k, k_new[own]]), np.concatenate([v, v_new[own]])
        for h in range(Hq):
            g = kv_head(h, Hq, kk.shape[1])
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (kk[:, g] @ q[i, h])
                p = np.exp(s - s.max())
                out[i, h] = (p / p.sum()) @ vv[:, g]
    return out


def accepted(parent, token, chosen):
    """(path, the token after it) from node 0 on; ([], -1) without nodes.  A negative choice is no token."""
    if len(parent) == 0:
        return [], -1
    path = [0]
    while True:
        step = [j for j in range(len(parent)) if parent[j] == path[-1] and token[j] == chosen[path[-1]] >= 0]
        if not step:
            return path, int(chosen[path[-1]])
        path.append(step[0])


def logits_row(x, prompt, generated, rep, presence, frequency, biases, allowed):
    """One row [V] (float32) after penalties, biases and mask, every operation rounded to 32 bits: (row, best token, its
    value).  biases: (token, value) pairs, the last one of a token counts; allowed: bool [V] or None."""
    x = x.astype(np.float32).copy()
    V = len(x)
    count = np.zeros(V, np.int64)
    for t in generated:
        if 0 <= t < V:
            count[t] += 1
    seen = count > 0
    seen[[t for t in prompt if 0 <= t < V]] = True
    f = np.float32
    with np.errstate(all="ignore"):
        x[seen] = np.where(x[seen] > 0, x[seen] / f(rep), x[seen] * f(rep))
        some = count > 0
        x[some] = x[some] - (f(presence) + f(frequency) * count[some].astype(np.float32))
        for t, v in dict(biases).items():
            if 0 <= t < V:
                x[t] = x[t] + f(v)
    if allowed is not None:
        x[~allowed] = -np.inf
    y = np.where(np.isnan(x), -np.inf, x)
    best = int(np.argmax(y))
    return (x, best, y[best]) if y[best] > -np.inf else (x, -1, f(-np.inf))
