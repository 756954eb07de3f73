"""Values that are not finite in drafted slots of some of many short groups, so that workgroups finish one item after the other: only the rows
that see them get them, in that item alone.

Tolerances: an output is a mean of values with weights of sum 1, so errors are measured against the largest finite value, M: float32 logits and sums
1e-4 M, bf16 adds the output's rounding, 2^-8 of the element."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from paper_2511_17560_amd import api
from gpu_util import idev, to_dev, to_host
from paged_util import make_pages, put
import a3_synth as synth

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,rows_lo,rows_hi", [("f32", 128, 9, 20), ("f32", 128, 33, 40), ("f32", 64, 9, 16), ("f32", 64, 17, 40), ("bf16", 128, 9, 16),
                                                     ("bf16", 128, 20, 40), ("f32", 128, 1, 8)])
def test_many_short_groups(dtype, d, rows_lo, rows_hi):
    rng = np.random.default_rng(d + rows_hi)
    n_groups, Hq, Hkv = 300, 8, 2
    value = lambda *s: synth.round_to_storage(rng.standard_normal(s, dtype=np.float32), dtype).astype(np.float64)
    rows, lens = rng.integers(rows_lo, rows_hi + 1, n_groups), rng.integers(0, 60, n_groups)
    p = make_pages((rows + lens).tolist(), dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, page=32, seed=2)
    held, seen = [], []
    for r, (n, m) in enumerate(zip(rows, lens)):
        k, v = value(m + n, Hkv, d), value(m + n, Hkv, d)
        if r % 3 == 1:
            for t in rng.integers(0, n, 2):
                v[m + t, rng.integers(0, Hkv), rng.integers(0, d, 3)] = [np.nan, np.inf, -np.inf]
        held.append(put(p, r, 0, k, v))
        seen.append(rng.random((n, n)) < 0.5)
    mask = torch.from_numpy(np.concatenate([cand.pack(s, 2) for s in seen])).cuda()
    q, start = value(rows.sum(), Hq, d), np.concatenate([[0], np.cumsum(rows)])
    out = torch.empty(q.shape, dtype=api.torch_dtype(dtype), device="cuda")
    most = int(rows.max())
    ws, got = p.tree_workspace(n_groups, most), []
    for _ in range(3):
        out.fill_(9.0)
        api.a3_tree_attention(p, to_dev(q, dtype), idev(start), None, idev(lens), mask, len(q), most, out, ws)
        torch.cuda.synchronize()
        got.append(to_host(out))
    assert np.array_equal(got[0], got[1], equal_nan=True) and np.array_equal(got[0], got[2], equal_nan=True)
    odd = 0
    for g, (n, m) in enumerate(zip(rows, lens)):
        k, v = held[g]
        mine = got[0][start[g]:start[g + 1]]
        bad = ~np.isfinite(v)
        with np.errstate(invalid="ignore"):
            want = cand.tree_attend(q[start[g]:start[g + 1]], k, np.where(bad, 0.0, v), m, seen[g], d ** -0.5)
            for j in range(n):
                for t in np.nonzero(seen[g][j])[0]:
                    for h in range(Hkv):
                        add = np.where(bad[m + t, h], v[m + t, h], 0.0)
                        want[j, h * Hq // Hkv:(h + 1) * Hq // Hkv] += add
        fine = np.isfinite(want)
        odd += int((~fine).sum())
        assert np.array_equal(mine[~fine], want[~fine], equal_nan=True), g
        tol = 1e-4 * np.abs(v[~bad]).max() + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
        assert np.isfinite(mine[fine]).all() and np.all(np.abs(mine[fine] - want[fine]) <= np.broadcast_to(tol, want.shape)[fine]), g
    assert odd > 100
