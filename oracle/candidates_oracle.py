"""CPU oracle for following several candidates of one request: attention of drafted trees, the accepted path, cache rows moved, and the
best continuations of beams.

TEST INFRASTRUCTURE ONLY, like the other oracle files.  Caches are arrays [slots, KV heads, d] here; pages are a matter of the tests.
Pinned by tests/test_oracle_candidates.py.
"""
from __future__ import annotations

import numpy as np

from . import generate_oracle as gen


def ancestors(parents):
    """seen[j, t]: t is j itself or one of its ancestors."""
    n = len(parents)
    seen = np.eye(n, dtype=bool)
    for j in range(n):
        p = parents[j]
        while p >= 0:
            seen[j, p] = True
            p = parents[p]
    return seen


def pack(seen, words):
    """Bit t % 32 of word t / 32, int32 [rows, words]."""
    out = np.zeros((len(seen), words), dtype=np.uint32)
    for j, t in zip(*np.nonzero(seen)):
        out[j, t // 32] |= np.uint32(1) << np.uint32(t % 32)
    return out.view(np.int32)


def tree_attend(q, k, v, n_before, seen, scale, there=None):
    """Rows q [n, Hq, d] over the slots k, v [n_before + n, Hkv, d]: the first n_before of them, and those of the tree that seen [n, n]
    says.  there: the slots that exist."""
    there = np.ones(len(k), dtype=bool) if there is None else there
    out = []
    for j in range(len(q)):
        mine = np.concatenate([np.ones(n_before, dtype=bool), seen[j]])[:len(k)] & there
        out.append(gen.attend(q[j], k[mine], v[mine], scale))
    return np.stack(out) if out else np.zeros_like(q)


def follow(picked, tokens, parents, max_path):
    """Path of one tree, as row numbers."""
    path = [0] if len(tokens) else []
    while path and len(path) < max_path:
        hit = [c for c in range(path[-1] + 1, len(tokens)) if parents[c] == path[-1] and tokens[c] == picked[path[-1]]]
        if not hit:
            break
        path.append(hit[0])
    return path


def move(cache, moves):
    """cache[r]: the rows of request r, a list of arrays.  moves: sets of (source request, slot, target request, slot, slots); those of a
    set at once for every slot of the run.  Returns the new rows."""
    new = [c.copy() for c in cache]
    for s in moves:
        for o in range(max([m[4] for m in s] + [0])):
            held = [(m, new[m[0]][m[1] + o].copy()) for m in s if o < m[4]]
            for m, x in held:
                new[m[2]][m[3] + o] = x
    return new


def beams(x, score, done, end, n_best):
    """x [beams, vocab] of one group.  (score, beam, token) lists of n_best, -inf, -1, -1 where there is none.  Tokens of one beam whose worths
    a double holds as equal go by their logits."""
    got = []
    for b, row in enumerate(np.asarray(x, dtype=np.float64)):
        if not np.isfinite(score[b]):
            continue
        if done is not None and done[b]:
            got.append((-float(score[b]), b, 0.0, end))
            continue
        lp = gen.log_probs(row[None])[0]
        if np.isnan(lp).any():
            continue
        total = float(score[b]) + lp
        best = np.lexsort((np.arange(len(row)), -row))[:n_best]
        got += [(-total[t], b, -row[t], int(t)) for t in best if total[t] > -np.inf]
    got = sorted(got)[:n_best]
    got += [(np.inf, -1, 0.0, -1)] * (n_best - len(got))
    return np.array([-g[0] for g in got]), np.array([g[1] for g in got]), np.array([g[3] for g in got])
