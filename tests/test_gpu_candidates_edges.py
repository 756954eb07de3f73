"""Picks, moves and beams where pieces of rows, lists and pools meet: whole numbers are equal; worths have the tolerance of
tests/test_gpu_beam_select.py."""
import numpy as np
import pytest
import torch

from paper_2511_17560_amd import api
from gpu_util import idev
from test_gpu_beam_select import _check as check_beams, _select
from test_gpu_paged_move import _call as move, _check as check_moves, _layers, _snapshot

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,rows", [(1, 2), (3, 3), (7, 7), (9, 9), (8191, 64), (8192, 64), (8193, 64), (16385, 64), (32003, 64), (40000, 2100), (128256, 3)])
def test_picks_at_every_border(vocab, rows, dtype):
    """The largest logit at the ends of a row, of vectors, of chunks and of slices; a second one, equal, behind it."""
    rng = np.random.default_rng(vocab)
    places = [p for c in range(0, vocab + 8192, 1024) for p in (c - 1, c, c + 1) if 0 <= p < vocab] + [0, vocab - 1, max(vocab - 5, 0), max(vocab - 9, 0)]
    at = rng.choice(places, rows)
    at[:2] = 0, vocab - 1
    x = torch.randn(rows, vocab, device="cuda", generator=torch.Generator(device="cuda").manual_seed(vocab)).clamp_(-3, 3).to(TYPES[dtype])
    i = torch.arange(rows, device="cuda")
    x[i, torch.from_numpy(at).cuda()] = 5.0
    again = np.minimum(at + rng.integers(0, 9000, rows), vocab - 1)
    x[i, torch.from_numpy(again).cuda()] = 5.0
    out = api.TreeAccepted(1, rows, 4, vocab)
    api.a3_tree_accept(x, idev(np.zeros(rows)), idev(np.full(rows, -1)), idev([0, 1]), idev([0]), rows, 1, out)
    torch.cuda.synchronize()
    assert np.array_equal(out.picked.cpu().numpy()[:rows], at)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n_beams,n_best", [(4000, 20, 64), (4000, 3, 64), (4000, 64, 64), (70000, 64, 64), (1200000, 1, 64), (300000, 5, 33), (128256, 4, 8),
                                                  (9001, 11, 2)])
def test_where_the_best_are(vocab, n_beams, n_best, dtype):
    """All of them in one beam, in one slice of it, spread evenly over all lists, or every one equal."""
    rng = np.random.default_rng(vocab + n_beams)
    # (a few logits far ahead, each at its own value, so that candidates differ by more than the worths' error, or are equal)
    def rows(of, places):
        x = np.full((n_beams, vocab), -20.0, dtype=np.float32)
        for j, (b, v) in enumerate(zip(of, places)):
            x[b, v] = 16.0 - 0.125 * j
        return x
    n = min(2 * n_best, 100)
    last = n_beams - 1
    some = rng.choice(vocab, n, replace=False)
    near = (vocab // 2 + rng.permutation(min(vocab // 2, 400))[:n])
    for x, score in ((rows([last] * n, some), np.where(np.arange(n_beams) == last, 0.0, -300.0)),
                     (rows([last] * n, near), np.where(np.arange(n_beams) == last, 0.0, -300.0)),
                     (np.zeros((n_beams, vocab), dtype=np.float32), np.full(n_beams, -1.0)),
                     (np.zeros((n_beams, vocab), dtype=np.float32), -0.5 * np.arange(n_beams))):
        out, stored, s = _select(x, score, n_beams, n_best, dtype=dtype)
        check_beams(out, stored, s, n_beams, n_best)
    # one value ahead in every beam: each beam's first, then the beams' rest in the order of the beams' scores
    x = np.full((n_beams, vocab), -20.0, dtype=np.float32)
    x[np.arange(n_beams), rng.integers(0, vocab, n_beams)] = 10.0
    out, stored, s = _select(x, -0.25 * rng.permutation(n_beams), n_beams, n_best, dtype=dtype)
    check_beams(out, stored, s, n_beams, n_best)


@pytest.mark.parametrize("q8", [False, True])
def test_fewer_workgroups_than_pools_and_heads(q8):
    """Many sets at once: a workgroup goes over several pools and heads with the same slots; sets of every size the kernel has."""
    rng = np.random.default_rng(5)
    for size, n_sets in ((1, 400), (3, 200), (5, 120), (9, 60), (17, 40)):
        n_req = size * n_sets
        pages = _layers([64] * n_req, 3, dtype="bf16", d=128, Hq=3, Hkv=3, q8=q8, page=64, seed=size)
        before = _snapshot(pages)
        sets = []
        for s in range(n_sets):
            at = int(rng.integers(0, 20))                                # (one place for all: nothing is read at another o than it is written)
            sets.append([(s * size + int(rng.integers(0, size)), at, s * size + b, at, int(rng.integers(0, 44))) for b in range(size)])
        move(pages, sets)
        check_moves(pages, before, sets)


def test_runs_as_long_as_a_number_goes():
    """Runs of 2^31 - 1 slots, cut where the pages' table ends; the rest of the tables' slots are moved."""
    pages = _layers([128] * 3, 2, Hq=4, Hkv=2, page=64, slack=0)
    before = _snapshot(pages)
    most = 2 ** 31 - 1
    sets = [[(0, 5, 1, 5, most), (1, 5, 0, 5, most)], [(2, 100, 2, 100, most), (2, most, 2, 0, most)]]
    move(pages, sets, most=most)
    check_moves(pages, before, [[(0, 5, 1, 5, 123), (1, 5, 0, 5, 123)]])
