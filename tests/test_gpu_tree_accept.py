"""Accepted paths of drafted trees, against the oracle: whole numbers, so equal."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from oracle import generate_oracle as gen
from paper_2511_17560_amd import api
from gpu_util import idev

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _tree(rng, n):
    return [-1] + [int(rng.integers(max(0, (j - 1) // 3), j)) for j in range(1, n)]


def _case(rng, rows, vocab, dtype, agree=0.8):
    """Logits [n, vocab] (as stored) with the largest at one child's token in `agree` of the rows that have one."""
    trees = [_tree(rng, n) if n else [] for n in rows]
    tokens = rng.integers(0, vocab, sum(rows))
    x = rng.standard_normal((sum(rows), vocab)).astype(np.float32) * 2
    at = 0
    for t in trees:
        for j in range(len(t)):
            children = [c for c in range(len(t)) if t[c] == j]
            if children and rng.random() < agree:
                x[at + j, tokens[at + rng.choice(children)]] = 30.0
        at += len(t)
    return trees, tokens, torch.from_numpy(x).to(TYPES[dtype])


def _expect(picked, tokens, trees, lens, max_path, max_rows=None):
    out, at = dict(count=[], path=[], next_token=[], src_slot=[], dst_slot=[]), 0
    for t, n in zip(trees, lens):
        m = min(len(t), max_rows or len(t))
        path = cand.follow(picked[at:at + m], tokens[at:at + m], t[:m], max_path)
        none = [-1] * (max_path - len(path))
        out["count"].append(len(path))
        out["path"].append(path + none)
        out["next_token"].append(picked[at + path[-1]] if path else -1)
        out["src_slot"].append([n + p for p in path] + none)
        out["dst_slot"].append([n + i for i in range(len(path))] + none)
        at += len(t)
    return {k: np.array(v) for k, v in out.items()}


def _check(out, want, picked=None):
    torch.cuda.synchronize()
    for name, w in want.items():
        got = getattr(out, name).cpu().numpy()
        assert np.array_equal(got[:len(w)], w), name
    if picked is not None:
        assert np.array_equal(out.picked.cpu().numpy()[:len(picked)], picked)


def _call(logits, tokens, trees, lens, max_path=16, max_rows=None, extra=0):
    rows = [len(t) for t in trees]
    n = sum(rows) + extra
    out = api.TreeAccepted(len(trees), n, max_path, 0 if logits is None else logits.shape[1])
    for t in (out.picked, out.count, out.next_token, out.path, out.src_slot, out.dst_slot):
        t.fill_(-77)
    out.ws.fill_(255)
    parent = idev(np.concatenate([np.asarray(t, dtype=np.int32) for t in trees] + [np.zeros(extra, np.int32)]))
    start = idev(np.concatenate([[0], np.cumsum(rows)]))
    return api.a3_tree_accept(logits, idev(np.concatenate([tokens, np.zeros(extra, np.int64)])), parent, start, idev(lens), n, max_rows or max(max(rows), 1), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(1, [3]), (2, [5, 1, 9]), (17, [1]), (501, [16, 0, 7, 64]), (4099, [30] * 5), (32003, [8, 64, 1, 5]), (128256, [16]),
                                        (152064, [3, 12]), (1000, [200, 1024, 65]), (4096, [1] * 300)])
def test_paths(vocab, rows, dtype):
    rng = np.random.default_rng(vocab + len(rows))
    trees, tokens, x = _case(rng, rows, vocab, dtype)
    lens = rng.integers(0, 9000, len(rows))
    picked = gen.top(x.double().numpy(), 1)[:, 0]
    for max_path in (16, 1, 64):
        out = _call(x.cuda(), tokens, trees, lens, max_path)
        _check(out, _expect(picked, tokens, trees, lens, max_path), picked)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ties_zeros_nan_and_infinities(dtype):
    """Equal logits: the lowest index; -0 is 0; NaN is below -inf; rows that start anywhere an element can, apart from each other."""
    vocab = 3001
    x = np.full((10, vocab), -5.0, dtype=np.float32)
    x[0, [7, 2000, 2999]] = 3.0
    x[1] = 0.0
    x[1, :5] = -0.0
    x[2] = np.nan
    x[3] = np.nan
    x[3, 2500] = -np.inf
    x[4] = -np.inf
    x[5, [1500, 1501]] = np.inf
    x[6, 0] = np.nan
    x[6, 3000] = -4.0
    x[7, ::2] = np.nan
    x[8] = -np.finfo(np.float32).max if dtype == "f32" else float(torch.finfo(torch.bfloat16).min)
    x[9, vocab - 1] = 1e-30
    want = np.array([7, 0, 0, 2500, 0, 1500, 3000, 1, 0, 3000])
    assert np.array_equal(gen.top(x.astype(np.float64), 1)[:, 0], want)
    for shift in range(9):
        wide = torch.full((10, vocab + 13), float("inf"), dtype=TYPES[dtype], device="cuda")
        part = wide[:, shift:shift + vocab]
        part.copy_(torch.from_numpy(x))
        out = _call(part, np.zeros(10, np.int64), [[-1] + [99] * 9], [5])
        _check(out, dict(count=np.array([1]), next_token=want[:1]), want)


def test_children_parents_and_bounds_that_are_no_tree():
    """Only rows behind the last with exactly its number as their parent go on; the first of equal ones; a parent behind its child, or
    outside, is never met.  Bounds out of order: an empty group.  Rows behind max_rows are not looked at."""
    picked = np.array([5, 5, 5, 5, 5, 5, 5, 5])
    parents, tokens = [-1, 0, 0, 7, 1, -9, 2 ** 31 - 1, 4], np.array([0, 4, 5, 5, 5, 5, 5, 5])
    out = api.TreeAccepted(3, 8, 5)
    for start, most, want in (([0, 8, 8, 8], 8, [[0, 2], [], []]), ([3, 1, 8, 9], 8, [[], [0, 1, 3], []]), ([0, 2, -1, 8], 8, [[0], [], []]),
                              ([0, 8, 8, 8], 2, [[0], [], []]), ([2 ** 31 - 1, -2 ** 31, 0, 8], 8, [[], [], [0, 2]])):
        out.picked.copy_(idev(picked))
        api.a3_tree_accept(None, idev(tokens), idev(parents), idev(start), idev([10, 20, 30]), 8, most, out)
        _check(out, dict(count=np.array([len(w) for w in want]), path=np.array([w + [-1] * (5 - len(w)) for w in want]),
                         next_token=np.array([5 if w else -1 for w in want]),
                         src_slot=np.array([[L + p for p in w] + [-1] * (5 - len(w)) for w, L in zip(want, (10, 20, 30))])), picked)


def test_rows_of_no_group_are_picked_and_long_paths_cut():
    rng = np.random.default_rng(4)
    n, vocab = 80, 700
    trees, tokens = [list(range(-1, n - 1))], rng.integers(0, vocab, n)
    x = torch.randn(n + 4, vocab)
    x[torch.arange(n - 1), torch.from_numpy(tokens[1:])] = 20.0
    picked = gen.top(x.double().numpy(), 1)[:, 0]
    for max_path in (1, 7, 63, 64):
        out = _call(x.cuda(), tokens, trees, [40], max_path, extra=4)
        want = _expect(picked, tokens, trees, [40], max_path)
        assert want["count"][0] == max_path
        _check(out, want, picked)


def test_fewer_rows_than_the_buffers_on_another_stream_and_captured():
    """Buffers made for more; a captured call follows logits and trees as they are at each replay."""
    rng = np.random.default_rng(6)
    rows, vocab = [9, 16, 4], 5003
    out = api.TreeAccepted(8, 100, 12, vocab)
    n, most = sum(rows), 16
    x, tokens, parent = torch.empty((n, vocab), device="cuda"), idev(np.zeros(n)), idev(np.zeros(n))
    start, lens = idev(np.concatenate([[0], np.cumsum(rows)])), idev([3, 700, 0])
    call = lambda: api.a3_tree_accept(x, tokens, parent, start, lens, n, most, out)
    x.zero_()
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    side = torch.cuda.Stream()
    for i in range(4):
        trees, tok, logits = _case(rng, rows, vocab, "f32", agree=0.5 + 0.15 * i)
        x.copy_(logits)
        tokens.copy_(idev(tok))
        parent.copy_(idev(np.concatenate(trees)))
        picked = gen.top(logits.double().numpy(), 1)[:, 0]
        want = _expect(picked, tok, trees, [3, 700, 0], 12)
        for t in (out.count, out.path, out.picked, out.next_token):
            t.fill_(-5)
        graph.replay()
        _check(out, want, picked)
        out.count.fill_(-5)
        torch.cuda.synchronize()
        api.a3_tree_accept(x, tokens, parent, start, lens, n, most, out, stream=side)
        side.synchronize()
        _check(out, want, picked)
        assert bool((out.path[3:] != 0).all()) or i == 0                 # groups behind the last: not written
