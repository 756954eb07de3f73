"""CPU oracle for generating on the fused cache: appending to it, attention of single tokens over it, logits and log
probabilities.

TEST INFRASTRUCTURE ONLY, like the other oracle files.  A request's cache is an array [slots, KV heads, d] here; pages are a
matter of the tests, which spread it over a pool.  Pinned by tests/test_oracle_generate.py.
"""
from __future__ import annotations

import numpy as np

from . import a3_oracle as ora


def turn(x, positions, base, layout, storage="exact"):
    """Rows [n, heads, d] turned to their positions; (cos, sin) as the path stores them, in float32."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    angle = np.asarray(positions, dtype=np.float64)[:, None] * ora.rope_theta(d, base)[None]
    c, s = (f(angle).astype(np.float32).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    a, b = ora.rope_pairs(d, layout)
    y = np.empty_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return ora.store(y, storage)


def attend(q, k, v, scale):
    """One token: q [Hq, d] over the n slots k, v [n, Hkv, d].  No slots: zeros."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros_like(q)
    out = np.empty_like(q)
    group = q.shape[0] // k.shape[1]
    for h in range(q.shape[0]):
        s = k[:, h // group] @ q[h] * scale
        with np.errstate(invalid="ignore"):
            w = np.exp(s - s.max())
        out[h] = (w / w.sum()) @ v[:, h // group]
    return out


def log_probs(x):
    """log softmax of rows; NaN where a row has no distribution (NaN, +inf, or nothing but -inf in it)."""
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        m = x.max(-1, keepdims=True)
        return x - m - np.log(np.exp(x - m).sum(-1, keepdims=True))


def given(lp, tokens):
    """Log probabilities of tokens [n, m]; -inf for a token that is not in the vocabulary."""
    tokens = np.asarray(tokens)
    inside = (tokens >= 0) & (tokens < lp.shape[-1])
    return np.where(inside, np.take_along_axis(lp, np.where(inside, tokens, 0), -1), -np.inf)


def entropy(lp):
    p = np.exp(lp)
    return -np.where(p > 0, p * np.where(p > 0, lp, 0.0), p).sum(-1)


def top(x, n):
    """Indexes of the n largest, largest first, equal ones by the lower index, NaN behind everything else."""
    x = np.asarray(x, dtype=np.float64)
    i = np.arange(x.shape[-1])
    return np.stack([np.lexsort((i, -np.where(np.isnan(r), 0, r), np.isnan(r)))[:n] for r in x]).astype(np.int32).reshape(len(x), n)
