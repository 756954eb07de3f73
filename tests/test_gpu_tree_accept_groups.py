"""Accepted paths in buffers made for more trees and rows: what lies behind the last group and the last row stays as it was, eager, on another
stream and replayed.  Whole numbers, so equal."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from paper_2511_17560_amd import api
from gpu_util import idev

pytestmark = pytest.mark.gpu
OUT, KEEP = ("picked", "count", "next_token", "path", "src_slot", "dst_slot"), -1234


def _case(rng, rows, vocab):
    trees = [[-1] + [int(rng.integers(max(0, (j - 1) // 3), j)) for j in range(1, n)] for n in rows]
    tokens, parents = rng.integers(0, vocab, sum(rows)), np.concatenate(trees)
    start = np.concatenate([[0], np.cumsum(rows)])
    x = rng.standard_normal((sum(rows), vocab)).astype(np.float32)
    for g, t in enumerate(trees):
        for j in range(len(t)):
            children = [c for c in range(j + 1, len(t)) if t[c] == j]
            if children and rng.random() < 0.8:
                x[start[g] + j, tokens[start[g] + rng.choice(children)]] = 30.0
    return trees, tokens, parents, start, x


@pytest.mark.parametrize("given", [False, True])
def test_nothing_behind_the_last(given):
    rng = np.random.default_rng(3)
    rows, lens, vocab, max_path = [7, 1, 16, 4], [3, 0, 700, -5], 4001, 9
    n, groups = sum(rows), len(rows)
    out = api.TreeAccepted(groups + 5, n + 40, max_path, 0 if given else vocab)
    x, tokens, parents = torch.zeros((n, vocab), device="cuda"), idev(np.zeros(n)), idev(np.zeros(n))
    start, length = idev(np.concatenate([[0], np.cumsum(rows)])), idev(lens)
    call = lambda stream=None: api.a3_tree_accept(None if given else x, tokens, parents, start, length, n, max(rows), out, stream=stream)
    call()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        call()
    for turn in range(3):
        trees, tok, par, at, logits = _case(rng, rows, vocab)
        picked = logits.argmax(-1)
        x.copy_(torch.from_numpy(logits))
        tokens.copy_(idev(tok))
        parents.copy_(idev(par))
        for run in (graph.replay, call, lambda: call(side)):
            for name in OUT:
                getattr(out, name).fill_(KEEP)
            if given:
                out.picked[:n].copy_(idev(picked))
            torch.cuda.synchronize()
            run()
            torch.cuda.synchronize()
            got = {name: getattr(out, name).cpu().numpy() for name in OUT}
            assert np.array_equal(got["picked"][:n], picked) and (got["picked"][n:] == KEEP).all()
            for name in OUT[1:]:
                assert (got[name][groups:] == KEEP).all(), name
            for g, t in enumerate(trees):
                rows_of = slice(at[g], at[g + 1])
                path = cand.follow(picked[rows_of], tok[rows_of], t, max_path)
                none = [-1] * (max_path - len(path))
                assert got["count"][g] == len(path) and got["next_token"][g] == picked[at[g] + path[-1]]
                assert got["path"][g].tolist() == path + none
                assert got["src_slot"][g].tolist() == [max(lens[g], 0) + p for p in path] + none
                assert got["dst_slot"][g].tolist() == [max(lens[g], 0) + m for m in range(len(path))] + none
