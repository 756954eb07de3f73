"""Attention of drafted trees over a paged cache, against the float64 oracle on what the cache holds.

Tolerances: as for single tokens (tests/test_gpu_paged_attention.py).  An output is a mean of values with weights of sum 1, so errors
are measured against the largest value seen, M: float32 logits and sums 1e-4 M, bf16 adds the output's rounding, 2^-8 of the element."""
import numpy as np
import pytest
import torch

from oracle import candidates_oracle as cand
from paper_2511_17560_amd import api
from gpu_util import idev, to_dev, to_host
from paged_util import make_pages, put
import a3_synth as synth

pytestmark = pytest.mark.gpu


def _values(rng, dtype, *shape):
    return synth.round_to_storage(rng.standard_normal(shape, dtype=np.float32), dtype).astype(np.float64)


def tree(rng, n):
    """Parents of a random tree of n, in front of their children."""
    return [-1] + [int(rng.integers(max(0, (j - 1) // 3), j)) for j in range(1, n)]


def filled(lens, rows, seed=0, **kw):
    """Pages of requests of lens[r] committed slots and rows[r] drafted ones, all written; what is behind them is NaN."""
    rng = np.random.default_rng(seed)
    p = make_pages([n + m for n, m in zip(lens, rows)], seed=seed, **kw)
    s = p.struct
    held = []
    for r, (n, m) in enumerate(zip(lens, rows)):
        k, v = (_values(rng, p.dtype, n + m, s.n_kv_heads, s.head_dim) for _ in range(2))
        held.append(put(p, r, 0, k, v) if n + m else (k, v))
    return p, held, rng


def masks(trees, words=None):
    """Packed rows [sum of rows, words] of the trees' ancestors."""
    words = words or max(-(-max(len(t) for t in trees) // 32), 1)
    rows = [cand.pack(cand.ancestors(t), words) for t in trees]
    return torch.from_numpy(np.concatenate(rows)).cuda()


def attend(p, q, rows, lens, mask, req=None, max_rows=None, extra=0, ws=None, out=None):
    """One call on q [sum rows + extra, Hq, d]; rows behind the last group have to stay 9."""
    n, most = len(q), max_rows or max(max(rows), 1)
    start = idev(np.concatenate([[0], np.cumsum(rows)]))
    out = torch.full(q.shape, 9.0, dtype=api.torch_dtype(p.dtype), device="cuda") if out is None else out
    ws = p.tree_workspace(len(rows), most).fill_(255) if ws is None else ws           # whatever the workspace held
    api.a3_tree_attention(p, to_dev(q, p.dtype), start, None if req is None else idev(req), idev(lens), mask, n, most, out, ws)
    torch.cuda.synchronize()
    return to_host(out)


def close(got, want, top, dtype):
    tol = 1e-4 * top + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    assert np.all(np.abs(got - want) <= tol), float((np.abs(got - want) - tol).max() / top)


def check(p, held, q, got, rows, lens, seen, req=None, scale=None):
    """seen[g] [rows, rows]: what each row sees of its tree."""
    s, at = p.struct, 0
    for g, (n, m) in enumerate(zip(rows, lens)):
        k, v = (t[:m + n] for t in held[g if req is None else req[g]])
        if n:
            want = cand.tree_attend(q[at:at + n], k, v, m, seen[g][:n, :n], scale or s.head_dim ** -0.5)
            close(got[at:at + n], want, max(np.abs(v).max(), 1e-30) if len(v) else 1.0, p.dtype)
        at += n


FORMS = [("bf16", 128, 32, 8), ("bf16", 128, 7, 1), ("bf16", 64, 16, 1), ("bf16", 64, 5, 5), ("f32", 64, 8, 8), ("f32", 128, 12, 4)]
LENS = [0, 0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 255, 511, 1000, 2049]
ROWS = [1, 5, 1, 17, 3, 2, 16, 32, 1, 12, 64, 7, 1, 33, 20, 9, 4]


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", FORMS)
def test_trees(dtype, d, Hq, Hkv, q8):
    """Committed parts from nothing to a few thousand, trees of 1 to 64 across every boundary a tile or a page can have."""
    p, held, rng = filled(LENS, ROWS, dtype=dtype, d=d, Hq=Hq, Hkv=Hkv, q8=q8)
    trees = [tree(rng, n) for n in ROWS]
    q = _values(rng, dtype, sum(ROWS), Hq, d)
    got = attend(p, q, ROWS, LENS, masks(trees))
    check(p, held, q, got, ROWS, LENS, [cand.ancestors(t) for t in trees])


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", FORMS)
def test_chains(dtype, d, Hq, Hkv, q8):
    p, held, rng = filled(LENS, ROWS, dtype=dtype, d=d, Hq=Hq, Hkv=Hkv, q8=q8, seed=1)
    q = _values(rng, dtype, sum(ROWS), Hq, d)
    got = attend(p, q, ROWS, LENS, None)
    check(p, held, q, got, ROWS, LENS, [np.tri(n, dtype=bool) for n in ROWS])


@pytest.mark.parametrize("dtype,Hq,Hkv,rows", [("bf16", 8, 2, [1]), ("bf16", 4, 1, [5]), ("bf16", 4, 4, [16]), ("bf16", 16, 2, [3, 0, 4]), ("bf16", 8, 2, [16, 9]),
                                               ("bf16", 8, 2, [17, 31]), ("bf16", 8, 2, [33, 64, 1]), ("bf16", 8, 2, [65, 130]), ("bf16", 32, 2, [40, 8]),
                                               ("bf16", 7, 1, [200]), ("bf16", 2, 2, [1024, 3]), ("f32", 8, 2, [17, 40]), ("f32", 4, 4, [300])])
def test_sizes_of_groups(dtype, Hq, Hkv, rows):
    """Groups on both sides of every number of rows at which a kernel or a tile changes, long enough to be cut."""
    lens = [3000, 700, 77][:len(rows)]
    d = 128 if dtype == "bf16" else 64
    p, held, rng = filled(lens, rows, dtype=dtype, d=d, Hq=Hq, Hkv=Hkv)
    q = _values(rng, dtype, sum(rows), Hq, d)
    seen = [rng.random((n, n)) < 0.4 for n in rows]                     # any set of the tree's slots, its own or not
    words = -(-max(rows) // 32)
    mask = torch.from_numpy(np.concatenate([cand.pack(s, words) for s in seen if len(s)])).cuda()
    check(p, held, q, attend(p, q, rows, lens, mask), rows, lens, seen)
    check(p, held, q, attend(p, q, rows, lens, None), rows, lens, [np.tri(n, dtype=bool) for n in rows])


@pytest.mark.parametrize("page", [32, 64, 128, 1024])
@pytest.mark.parametrize("q8", [False, True])
def test_page_sizes(page, q8):
    lens, rows = [5, page - 3, page, 2 * page + 7, 1500], [7, 7, 1, 40, 20]
    p, held, rng = filled(lens, rows, page=page, q8=q8, seed=page)
    trees = [tree(rng, n) for n in rows]
    q = _values(rng, "bf16", sum(rows), 8, 128)
    check(p, held, q, attend(p, q, rows, lens, masks(trees)), rows, lens, [cand.ancestors(t) for t in trees])


@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_one_long_request_beside_short_ones(dtype, q8):
    d = 128 if dtype == "bf16" else 64
    lens, rows = [3, 20011, 1, 0, 700], [2, 14, 30, 1, 5]
    p, held, rng = filled(lens, rows, dtype=dtype, d=d, Hq=4, Hkv=2, q8=q8)
    trees = [tree(rng, n) for n in rows]
    q = _values(rng, dtype, sum(rows), 4, d)
    seen = [cand.ancestors(t) for t in trees]
    check(p, held, q, attend(p, q, rows, lens, masks(trees)), rows, lens, seen)
    one = attend(p, q[2:16], [14], [20011], masks(trees[1:2]), req=[1])         # alone: the whole chip on it
    check(p, held, q[2:16], one, [14], [20011], seen[1:2], req=[1])


@pytest.mark.parametrize("n_groups", [65, 300, 700])
def test_many_groups_that_share_requests(n_groups):
    """More groups than there are requests, some empty, some of requests that do not exist, lengths of their own; rows of no group."""
    lens, most = [257, 40, 1, 130], 6
    p, held, rng = filled(lens, [most] * 4, Hq=4, Hkv=2, d=64)
    req = rng.integers(0, 4, n_groups)
    rows, n = rng.integers(0, most + 1, n_groups), np.array([rng.integers(0, lens[r] + 1) for r in req])
    named = np.where(rng.random(n_groups) < 0.2, rng.choice([-1, 4, 2 ** 31 - 1, -2 ** 31], n_groups), req)
    q = _values(rng, "bf16", int(rows.sum()) + 3, 4, 64)
    got = attend(p, q, rows, n, None, req=named, max_rows=most)
    off = np.concatenate([np.repeat(named != req, rows), [True] * 3])
    assert np.all(got[off] == 9.0)
    ok = named == req
    keep = np.concatenate([np.repeat(ok, rows), [False] * 3])
    check(p, held, q[keep], got[keep], rows[ok].tolist(), n[ok].tolist(), [np.tri(m, dtype=bool) for m in rows[ok]], req=req[ok].tolist())


def test_rows_that_see_nothing():
    """A new request whose masks leave rows empty: zeros; a mask without the row's own bit; committed slots alone."""
    for dtype, d in (("bf16", 128), ("f32", 64)):
        lens, rows = [0, 64, 0], [6, 40, 70]
        p, held, rng = filled(lens, rows, dtype=dtype, d=d, Hq=4, Hkv=2)
        q = _values(rng, dtype, sum(rows), 4, d)
        seen = [np.zeros((n, n), bool) for n in rows]
        seen[0][2, [0, 5]] = True                        # one row sees a later one and not itself
        seen[2][69, 69] = seen[2][3, 64] = True
        mask = torch.from_numpy(np.concatenate([cand.pack(s, 3) for s in seen])).cuda()
        got = attend(p, q, rows, lens, mask)
        empty = np.ones(sum(rows), bool)
        empty[2] = empty[46 + 69] = empty[46 + 3] = False
        empty[6:46] = False
        assert np.all(got[empty] == 0.0)
        check(p, held, q, got, rows, lens, seen)


def test_bits_behind_the_tree_are_not_looked_at():
    lens, rows = [100, 30], [5, 37]
    p, held, rng = filled(lens, rows, Hq=4, Hkv=2)
    q = _values(rng, "bf16", sum(rows), 4, 128)
    mask = torch.full((sum(rows), 4), -1, dtype=torch.int32, device="cuda")
    check(p, held, q, attend(p, q, rows, lens, mask, max_rows=128), rows, lens, [np.ones((n, n), bool) for n in rows])


def test_bounds_lengths_and_pages_that_do_not_exist():
    p, held, rng = filled([186, 186], [6, 6], slack=0)                  # 192 slots, three pages of 64
    table = p.page_table.cpu().numpy()
    q = _values(rng, "bf16", 12, 8, 128)
    tri = np.tri(6, dtype=bool)
    for bad in (-1, p.struct.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.copy()
        t[1, 1] = bad
        p.page_table.copy_(torch.from_numpy(t))
        got = attend(p, q, [6, 6], [186, 186], None)
        check(p, held, q[:6], got[:6], [6], [186], [tri])
        k, v = held[1]
        there = np.ones(192, bool)
        there[64:128] = False
        close(got[6:], cand.tree_attend(q[6:], k, v, 186, tri, 128 ** -0.5, there), np.abs(v).max(), "bf16")
        # committed part negative: none; up to the table's end and beyond: the tree's slots are cut off
        got = attend(p, q, [6, 6], [-5, 2 ** 31 - 1], None, req=[0, 0])
        check(p, held, q[:6], got[:6], [6], [0], [tri])
        want = cand.tree_attend(q[6:], *held[0], 192, tri, 128 ** -0.5)
        close(got[6:], want, np.abs(held[0][1]).max(), "bf16")
        got = attend(p, q, [6, 6], [189, 191], None, req=[0, 0])
        for i, n in ((0, 189), (1, 191)):
            close(got[6 * i:6 * i + 6], cand.tree_attend(q[6 * i:6 * i + 6], *held[0], n, tri, 128 ** -0.5), np.abs(held[0][1]).max(), "bf16")
    p.page_table.copy_(torch.from_numpy(table))
    # bounds that are not in order or outside the rows: such a group has no rows; more rows than max_rows: the rest stays
    for start in ([0, -1, 6], [0, 13, 6], [7, 3, 12], [0, 2 ** 31 - 1, -2 ** 31]):
        out = torch.full(q.shape, 9.0, dtype=torch.bfloat16, device="cuda")
        api.a3_tree_attention(p, to_dev(q, "bf16"), idev(start), None, idev([186, 186]), None, 12, 6, out, p.tree_workspace(2, 6))
        torch.cuda.synchronize()
        if start == [7, 3, 12]:
            assert bool((out[:3] == 9.0).all()) and bool((out[9:] == 9.0).all())
            check(p, held, q[3:9], to_host(out)[3:9], [6], [186], [tri], req=[1])
        else:
            assert bool((out == 9.0).all())
    got = attend(p, q, [6, 6], [186, 186], None, max_rows=4)
    assert np.all(got[4:6] == 9.0) and np.all(got[10:] == 9.0)
    check(p, held, q[:4], got[:4], [4], [186], [tri])
    check(p, held, q[6:10], got[6:10], [4], [186], [tri], req=[1])
    p.page_table.fill_(-1)                                              # no page at all: nothing seen
    assert np.all(attend(p, q, [6, 6], [186, 186], None) == 0.0)


@pytest.mark.parametrize("dtype,rows", [("bf16", 6), ("bf16", 20), ("bf16", 60), ("f32", 6), ("f32", 40)])
def test_values_that_are_not_finite(dtype, rows):
    """NaN and infinities in one branch's keys and values reach the rows that see it, and no others; so in the committed part all."""
    d = 128 if dtype == "bf16" else 64
    lens = [300, 61]
    p, held, rng = filled(lens, [rows] * 2, dtype=dtype, d=d, Hq=4, Hkv=2)
    q = _values(rng, dtype, 2 * rows, 4, d)
    seen = rng.random((rows, rows)) < 0.5
    bad_v, bad_k, bad_i = 1, 3, 4                                       # tree slots: a NaN value, a NaN key, an infinite value
    seen[:, [bad_v, bad_k, bad_i]] = False
    seen[0, bad_v] = seen[2, bad_k] = seen[5, bad_i] = True
    for r in range(2):
        k, v = (t.copy() for t in held[r])
        v[lens[r] + bad_v, 0, 7], v[lens[r] + bad_i, 1, 9], k[lens[r] + bad_k, 1, 3] = np.nan, np.inf, np.nan
        put(p, r, 0, k, v)
    mask = torch.from_numpy(np.concatenate([cand.pack(seen, 2)] * 2)).cuda()
    got = attend(p, q, [rows] * 2, lens, mask)
    for r in range(2):
        k, v = held[r]                                                  # finite everywhere: as every row but three sees it
        want, x = cand.tree_attend(q[r * rows:(r + 1) * rows], k, v, lens[r], seen, d ** -0.5), got[r * rows:(r + 1) * rows]
        odd = np.zeros(x.shape, bool)
        odd[0, :2, 7], odd[2, 2:], odd[5, 2:, 9] = True, True, True
        close(x[~odd], want[~odd], np.abs(v).max(), dtype)
        assert np.isnan(x[0, :2, 7]).all() and np.isnan(x[2, 2:]).all() and np.isposinf(x[5, 2:, 9]).all()
    # a committed value of NaN: its coordinate, in every row
    k, v = (t.copy() for t in held[0])
    v[17, 1, 3] = np.nan
    put(p, 0, 0, k, v)
    got = attend(p, q[:rows], [rows], lens[:1], masks([tree(rng, rows)], 2))
    assert np.isnan(got[:, 2:, 3]).all() and np.isfinite(got[:, :2]).all() and np.isfinite(np.delete(got[:, 2:], 3, 2)).all()
    # nothing but -inf to see: no distribution
    k[:, 0] = -np.inf
    put(p, 0, 0, k, held[0][1])
    q = np.abs(q) + 0.5
    assert np.isnan(attend(p, q[:rows], [rows], lens[:1], None)[:, :2]).all()


@pytest.mark.parametrize("dtype,q8,rows", [("bf16", False, 3), ("bf16", False, 40), ("bf16", True, 3), ("f32", False, 3), ("f32", False, 40)])
def test_large_logits_and_a_scale_of_ones_own(dtype, q8, rows):
    """Logits of some hundreds, far from each other and from zero: one key has all the weight, or two share it."""
    d, n = 128, 600
    p = make_pages([n + rows] * 2, dtype=dtype, d=d, Hq=4, Hkv=2, q8=q8, sm_scale=1.0)
    rng = np.random.default_rng(9)
    held = []
    for r in range(2):
        k, v = (_values(rng, dtype, n + rows, 2, d) for _ in range(2))
        k[411] = k[33] = 4.0 if r == 0 else -4.0
        held.append(put(p, r, 0, k, v))
    q = np.full((2 * rows, 4, d), 1.0)
    got = attend(p, q, [rows] * 2, [n] * 2, None)
    want0 = np.repeat((held[0][1][33] + held[0][1][411]) / 2, 2, 0)
    for j in range(rows):
        close(got[j], want0, np.abs(held[0][1]).max(), dtype)
    check(p, held, q[rows:], got[rows:], [rows], [n], [np.tri(rows, dtype=bool)], req=[1], scale=1.0)


def test_a_single_row_is_attention_of_a_single_token():
    lens = [1, 64, 500, 3000]
    p, held, rng = filled(lens, [1] * 4)
    q = _values(rng, "bf16", 4, 8, 128)
    got = attend(p, q, [1] * 4, lens, None)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    api.a3_paged_attention(p, to_dev(q, "bf16"), None, idev(np.array(lens) + 1), 4, out, p.workspace(4))
    torch.cuda.synchronize()
    assert np.all(np.abs(got - to_host(out)) <= 1e-3 + 2.0 ** -7 * np.abs(got))


def test_the_same_bits_again_on_another_stream_and_in_place():
    lens, rows = [1000, 5, 64, 3001], [16, 3, 30, 12]
    p, held, rng = filled(lens, rows)
    mask = masks([tree(rng, n) for n in rows])
    q = _values(rng, "bf16", sum(rows), 8, 128)
    a = attend(p, q, rows, lens, mask)
    assert np.array_equal(a, attend(p, q, rows, lens, mask))
    st = torch.cuda.Stream()
    qd, n, ws, start = to_dev(q, "bf16"), idev(lens), p.tree_workspace(4, 30), idev(np.concatenate([[0], np.cumsum(rows)]))
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        api.a3_tree_attention(p, qd, start, None, n, mask, sum(rows), 30, qd, ws)            # out = q
    st.synchronize()
    assert np.array_equal(a, to_host(qd))
    # a workspace and a bound made for more serve fewer
    assert np.array_equal(a, attend(p, q, rows, lens, mask, ws=p.tree_workspace(9, 100).fill_(255)))


def test_captured_with_lengths_and_trees_that_change():
    """A captured call follows bounds, lengths, masks and cache as they are at each replay; two graphs take turns on one workspace."""
    lens, rows, most = [900, 70, 2500], [16, 16, 16], 16
    p, held, rng = filled(lens, rows, Hq=4, Hkv=2)
    q = _values(rng, "bf16", 48, 4, 128)
    qd, n, ws, start = to_dev(q, "bf16"), idev(lens), p.tree_workspace(3, most), idev([0, 16, 32, 48])
    mask = masks([tree(rng, 16)] * 3)
    outs = [torch.empty_like(qd) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    call = lambda out: api.a3_tree_attention(p, qd, start, None, n, mask, 48, most, out, ws)
    call(outs[0])
    torch.cuda.synchronize()
    for g, out in zip(graphs, outs):
        with torch.cuda.graph(g):
            call(out)
    for now, bounds in (([900, 70, 2500], [0, 16, 32, 48]), ([1, 0, 1], [0, 1, 2, 3]), ([0, 0, 0], [0, 0, 16, 20]), ([64, 65, 2049], [0, 5, 21, 37]),
                        ([899, 70, 3], [0, 16, 16, 30])):
        trees = [tree(rng, 16) for _ in range(3)]
        n.copy_(idev(now))
        start.copy_(idev(bounds))
        m = np.zeros((48, 1), np.int32)
        for g in range(3):
            m[bounds[g]:bounds[g + 1]] = cand.pack(cand.ancestors(trees[g]), 1)[:bounds[g + 1] - bounds[g]]
        mask.copy_(torch.from_numpy(m))
        rows = np.diff(bounds).tolist()
        for g, out in zip(graphs, outs):
            out.fill_(9.0)
            g.replay()
            torch.cuda.synchronize()
            got = to_host(out)
            assert np.all(got[bounds[-1]:] == 9.0)
            check(p, held, q, got, rows, now, [cand.ancestors(t) for t in trees])
            out.fill_(9.0)
            call(out)
            torch.cuda.synchronize()
            assert np.array_equal(got, to_host(out))


def test_a_cache_beyond_32_bits():
    """Pools of more than 4 GiB each, a request whose pages lie at both ends."""
    n_pages = (5 << 30) // (8 * 1024 * 128 * 2)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    p = api.Pages(dtype="bf16", n_q_heads=16, n_kv_heads=8, head_dim=128, page_size=1024, n_pages=n_pages, page_table=table, rope_base=1e4,
                  n_pos=8)
    rng = np.random.default_rng(8)
    k, v = (_values(rng, "bf16", 2100, 8, 128) for _ in range(2))
    held = [put(p, 0, 0, k, v)]
    for rows in (7, 50):
        q = _values(rng, "bf16", rows, 16, 128)
        check(p, held, q, attend(p, q, [rows], [2100 - rows], None), [rows], [2100 - rows], [np.tri(rows, dtype=bool)])


def test_two_calls_at_once():
    """Two streams over one cache, each with a workspace of its own."""
    lens, rows = [3000, 17, 900], [12, 3, 20]
    p, held, rng = filled(lens, rows)
    q = [_values(rng, "bf16", sum(rows), 8, 128) for _ in range(2)]
    qd, n, start = [to_dev(x, "bf16") for x in q], idev(lens), idev(np.concatenate([[0], np.cumsum(rows)]))
    out, ws, streams = [torch.empty_like(x) for x in qd], [p.tree_workspace(3, 20) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            api.a3_tree_attention(p, qd[i], start, None, n, None, sum(rows), 20, out[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        check(p, held, q[i], to_host(out[i]), rows, lens, [np.tri(m, dtype=bool) for m in rows])
