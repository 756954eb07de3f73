"""Attention of wide drafted trees whose runs of steps go over many pages, items and requests, against the float64 oracle.

Tolerances: those of tests/test_gpu_tree_attention.py, 1e-4 of the largest value for logits and sums in float32, and the output's
rounding to bf16, 2^-8 of the element."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from test_gpu_tree_attention import _values, attend, check, close, filled, test_large_logits_and_a_scale_of_ones_own as large_logits
from test_gpu_tree_attention import test_values_that_are_not_finite as values_that_are_not_finite

pytestmark = pytest.mark.gpu

ROWS = [24, 17, 0, 33, 20, 64, 17, 1, 18, 40, 19, 17]
LENS = [5900, 4097, 10, 3000, 5903, 64, 0, 5936, 1, 2047, 5000, 4160]


@pytest.mark.parametrize("page", [32, 128])
@pytest.mark.parametrize("d,q8", [(128, False), (128, True), (64, False), (64, True)])
def test_long_runs_with_pages_missing(d, q8, page):
    """More than 64 pages an item, pages that are missing in front, in the middle and at the end of a committed part, empty groups and
    short items between long ones; every group sees its own set of the slots."""
    p, held, rng = filled([5940, 5940], [64, 64], d=d, q8=q8, page=page, seed=d + page)
    req = [g % 2 for g in range(len(ROWS))]
    table = p.page_table.cpu().numpy()
    there = np.ones((2, 6004), dtype=bool)
    for no in (0, 5, 6, 4095 // page, 4096 // page + 1, 5900 // page):
        table[1, no] = -1 if no % 2 else p.struct.n_pages
        there[1, no * page:(no + 1) * page] = False
    p.page_table.copy_(torch.from_numpy(table))
    q = _values(rng, "bf16", sum(ROWS), 8, d)
    seen = [rng.random((n, n)) < 0.5 for n in ROWS]
    mask = torch.from_numpy(np.concatenate([cand.pack(s, 2) for s in seen if len(s)])).cuda()
    got, at = attend(p, q, ROWS, LENS, mask, req=req), 0
    for g, (n, m) in enumerate(zip(ROWS, LENS)):
        k, v = (t[:m + n] for t in held[req[g]])
        want = cand.tree_attend(q[at:at + n], k, v, m, seen[g], d ** -0.5, there[req[g]][:m + n])
        close(got[at:at + n], want, np.abs(v).max(), "bf16")
        at += n


def test_the_same_bits_whatever_else_is_in_the_batch_of_one_item_a_workgroup():
    """Two calls on the same data, and one with groups in another order behind it: a group's pieces may be cut elsewhere, its result may
    not leave the tolerance; the same call gives the same bits."""
    rows, lens = [30, 64, 20], [900, 2500, 33]
    p, held, rng = filled(lens, rows)
    q = _values(rng, "bf16", sum(rows), 8, 128)
    first = attend(p, q, rows, lens, None)
    assert np.array_equal(first, attend(p, q, rows, lens, None))
    turned = attend(p, np.concatenate([q[30:], q[:30]]), rows[1:] + rows[:1], lens[1:] + lens[:1], None, req=[1, 2, 0])
    at = 0
    for r in range(3):
        k, v = held[r]
        want = cand.tree_attend(q[at:at + rows[r]], k, v, lens[r], np.tri(rows[r], dtype=bool), 128 ** -0.5)
        close(first[at:at + rows[r]], want, np.abs(v).max(), "bf16")
        to = (at - 30) % sum(rows)
        close(turned[to:to + rows[r]], want, np.abs(v).max(), "bf16")
        at += rows[r]


@pytest.mark.parametrize("rows", [(9, 16), (17, 20)])
@pytest.mark.parametrize("q8", [False, True])
def test_many_groups_of_many_columns(q8, rows):
    """More groups than a workgroup has threads, 36 to 80 columns each, of a few requests."""
    p, held, rng = filled([200, 75, 64], [24, 24, 24], q8=q8, seed=rows[0])
    n_groups = 600
    req = rng.integers(0, 3, n_groups).tolist()
    lens = [int(rng.integers(0, [200, 75, 64][r] + 1)) for r in req]
    size = rng.integers(rows[0], rows[1] + 1, n_groups)
    size[rng.integers(0, n_groups, 40)] = 0
    size = size.tolist()
    q = _values(rng, "bf16", sum(size), 8, 128)
    got = attend(p, q, size, lens, None, req=req, max_rows=rows[1])
    check(p, held, q, got, size, lens, [np.tri(n, dtype=bool) for n in size], req=req)


def test_a_block_of_columns_a_wave():
    values_that_are_not_finite("bf16", 12)
    large_logits("bf16", False, 12)
    large_logits("bf16", True, 12)
