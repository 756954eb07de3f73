"""Attention of single tokens over a paged cache, against the float64 oracle on what the cache holds.

Tolerances.  An output is a mean of values with weights of sum 1, so errors are measured against the largest value seen, M.
Logits: a sum of d products in float32, relative to sum |q k| at most d * 2^-24, and the scale; logits here stay below 40 in
sum |q k| * scale, so a logit is off by at most 130 * 40 * 2^-24 = 3.1e-4 in the worst case and, as the roundings are independent,
about sqrt(130) * 40 * 2^-24 = 2.7e-5; a weight's relative error is twice that (its own and the sum's).  fp32: 1e-4 M.  bf16 adds the
output's rounding, 2^-8 of the element: 1e-4 M + 2^-8 |out|."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as gen
from paper_2511_17560_amd import api
from gpu_util import idev, to_dev, to_host
from paged_util import make_pages, parts, put
import a3_synth as synth

pytestmark = pytest.mark.gpu


def _values(rng, dtype, *shape):
    return synth.round_to_storage(rng.standard_normal(shape, dtype=np.float32), dtype).astype(np.float64)


def _filled(lens, seed=0, **kw):
    rng = np.random.default_rng(seed)
    p = make_pages(lens, seed=seed, **kw)
    s = p.struct
    held = []
    for r, n in enumerate(lens):
        k, v = (_values(rng, p.dtype, n, s.n_kv_heads, s.head_dim) for _ in range(2))
        held.append(put(p, r, 0, k, v) if n else (k, v))
    return p, held, rng


def _attend(p, q, lens, req=None, ws=None, out=None):
    n = len(lens)
    out = torch.full(q.shape, 9.0, dtype=api.torch_dtype(p.dtype), device="cuda") if out is None else out
    ws = p.workspace(n).fill_(255) if ws is None else ws          # whatever the workspace held
    api.a3_paged_attention(p, to_dev(q, p.dtype), None if req is None else idev(req), idev(lens), n, out, ws)
    torch.cuda.synchronize()
    return to_host(out)


def _check(got, want, top, dtype):
    tol = 1e-4 * top + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    ok = bool(np.all(np.abs(got - want) <= tol))
    assert ok, float(np.abs(got - want).max() / top)


def _check_rows(p, held, q, got, lens, req=None, scale=None):
    s = p.struct
    for i, n in enumerate(lens):
        k, v = (t[:max(n, 0)] for t in held[i if req is None else req[i]])
        _check(got[i], gen.attend(q[i], k, v, scale or s.head_dim ** -0.5), max(np.abs(v).max(), 1e-30) if n > 0 else 1.0, p.dtype)


FORMS = [("bf16", 128, 32, 8), ("bf16", 128, 7, 1), ("bf16", 64, 16, 1), ("bf16", 64, 5, 5), ("f32", 64, 8, 8), ("f32", 128, 12, 4)]


@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,Hkv", FORMS)
def test_lengths(dtype, d, Hq, Hkv, q8):
    """From nothing to a few thousand, around every boundary a tile or a page can have; behind the ends lies NaN."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 2049]
    p, held, rng = _filled(lens, dtype=dtype, d=d, Hq=Hq, Hkv=Hkv, q8=q8)
    q = _values(rng, dtype, len(lens), Hq, d)
    got = _attend(p, q, lens)
    assert np.all(got[0] == 0.0)
    _check_rows(p, held, q, got, lens)


@pytest.mark.parametrize("page", [32, 64, 128, 256, 1024])
@pytest.mark.parametrize("q8", [False, True])
def test_page_sizes(page, q8):
    lens = [5, page - 1, page, page + 1, 2 * page + 7, 1500]
    p, held, rng = _filled(lens, page=page, q8=q8, seed=page)
    q = _values(rng, "bf16", len(lens), 8, 128)
    _check_rows(p, held, q, _attend(p, q, lens), lens)


@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
def test_one_long_row_beside_short_ones(dtype, q8):
    d = 128 if dtype == "bf16" else 64
    lens = [3, 20011, 1, 0, 700]
    p, held, rng = _filled(lens, dtype=dtype, d=d, Hq=4, Hkv=2, q8=q8)
    q = _values(rng, dtype, len(lens), 4, d)
    _check_rows(p, held, q, _attend(p, q, lens), lens)
    one = _attend(p, q[1:2], [20011], req=[1])                    # alone: the whole chip on it
    _check_rows(p, held, q[1:2], one, [20011], req=[1])


@pytest.mark.parametrize("n_rows", [2, 300, 1100])
def test_rows_that_share_requests(n_rows):
    """Many rows, several of a request with lengths of their own, in any order; a padding row stays as it was."""
    lens = [257, 40, 1, 130]
    p, held, rng = _filled(lens, Hq=4, Hkv=2)
    req = rng.integers(0, 4, n_rows)
    n = np.array([rng.integers(0, lens[r] + 1) for r in req])
    q = _values(rng, "bf16", n_rows, 4, 128)
    named = req.copy()
    named[1], n[1] = -1, 200
    got = _attend(p, q, n, req=named)
    assert np.all(got[1] == 9.0)
    keep = np.arange(n_rows) != 1
    _check_rows(p, held, q[keep], got[keep], n[keep].tolist(), req=req[keep].tolist())


def test_requests_lengths_and_pages_that_do_not_exist():
    """Request outside the table: untouched.  Length beyond the table: cut to it.  A page outside the pool: its slots do not count.
    Negative length: zeros."""
    lens = [192, 192]
    p, held, rng = _filled(lens, slack=0)
    table = p.page_table.cpu().numpy()
    for bad in (-1, p.struct.n_pages, 2 ** 31 - 1, -2 ** 31):
        t = table.copy()
        t[1, 1] = bad
        p.page_table.copy_(torch.from_numpy(t))
        q = _values(rng, "bf16", 6, 8, 128)
        got = _attend(p, q, [192, 2 ** 31 - 1, 2 ** 31 - 1, 150, -5, 10], req=[0, 0, 1, 1, 1, 2])
        _check_rows(p, held, q[:2], got[:2], [192, 192], req=[0, 0])
        for i, n in ((2, 192), (3, 150)):
            k, v = (np.concatenate([t[:64], t[128:n]]) for t in held[1])
            _check(got[i], gen.attend(q[i], k, v, 128 ** -0.5), np.abs(v).max(), "bf16")
        assert np.all(got[4] == 0.0) and np.all(got[5] == 9.0)
    t = np.full_like(table, -1)                                    # no page at all: nothing seen
    p.page_table.copy_(torch.from_numpy(t))
    assert np.all(_attend(p, q[:2], [192, 7]) == 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_that_are_not_finite(dtype):
    """A key at -inf logits has weight 0; what is NaN or infinite in a seen value reaches only its own head and coordinate."""
    d = 128 if dtype == "bf16" else 64
    lens = [300, 300, 300]
    p, held, rng = _filled(lens, dtype=dtype, d=d, Hq=4, Hkv=2)
    s = p.struct
    q = synth.round_to_storage((np.abs(_values(rng, dtype, 3, 4, d)) + 0.5).astype(np.float32), dtype).astype(np.float64)   # as the GPU gets it
    # request 0: the first 64 slots of head 0 have logits of -inf (their values NaN would still count: left finite)
    k, v = (t.copy() for t in held[0])
    k[:64, 0] = -np.inf
    put(p, 0, 0, k, v)
    # request 1: a NaN and an infinity in the values of slot 17, head 1
    k1, v1 = (t.copy() for t in held[1])
    v1[17, 1, 3], v1[17, 1, 5] = np.nan, np.inf
    put(p, 1, 0, k1, v1)
    # request 2: a NaN in a key of head 0
    k2, v2 = (t.copy() for t in held[2])
    k2[299, 0, 0] = np.nan
    put(p, 2, 0, k2, v2)
    got = _attend(p, q, lens)
    want = gen.attend(q[0], k[64:, :1], v[64:, :1], d ** -0.5)[:2]
    _check(got[0, :2], want, np.abs(v).max(), dtype)
    _check(got[0, 2:], gen.attend(q[0, 2:], k[:, 1:], v[:, 1:], d ** -0.5), np.abs(v).max(), dtype)
    ok = np.ones(d, bool)
    ok[[3, 5]] = False
    want = gen.attend(q[1, 2:], k1[:, 1:], held[1][1][:, 1:], d ** -0.5)
    _check(got[1, 2:][:, ok], want[:, ok], np.abs(held[1][1]).max(), dtype)
    assert np.isnan(got[1, 2:, 3]).all() and np.isposinf(got[1, 2:, 5]).all()
    _check(got[1, :2], gen.attend(q[1, :2], k1[:, :1], v1[:, :1], d ** -0.5), np.abs(held[1][1]).max(), dtype)
    assert np.isnan(got[2, :2]).all()
    _check(got[2, 2:], gen.attend(q[2, 2:], k2[:, 1:], v2[:, 1:], d ** -0.5), np.abs(v2).max(), dtype)
    # nothing but -inf: no distribution
    k[:, 0] = -np.inf
    put(p, 0, 0, k, v)
    assert np.isnan(_attend(p, q, lens)[0, :2]).all()


@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False)])
def test_large_logits_and_a_scale_of_ones_own(dtype, q8):
    """Logits of some hundreds, far from each other and from zero: one key has all the weight, or two share it."""
    d = 128
    p = make_pages([600, 600], dtype=dtype, d=d, Hq=4, Hkv=2, q8=q8, sm_scale=1.0)
    rng = np.random.default_rng(9)
    held = []
    for r in range(2):
        k, v = (_values(rng, dtype, 600, 2, d) for _ in range(2))
        k[411] = k[33] = 4.0 if r == 0 else -4.0
        held.append(put(p, r, 0, k, v))
    q = np.full((2, 4, d), 1.0)
    got = _attend(p, q, [600, 600])
    want0 = np.repeat((held[0][1][33] + held[0][1][411]) / 2, 2, 0)
    _check(got[0], want0, np.abs(held[0][1]).max(), dtype)
    k, v = held[1]
    _check(got[1], gen.attend(q[1], k, v, 1.0), np.abs(v).max(), dtype)


def test_the_same_bits_again_on_another_stream_and_in_place():
    lens = [1000, 5, 64, 3001]
    p, held, rng = _filled(lens)
    q = _values(rng, "bf16", 4, 8, 128)
    a = _attend(p, q, lens)
    assert np.array_equal(a, _attend(p, q, lens))
    st = torch.cuda.Stream()
    qd, n, ws = to_dev(q, "bf16"), idev(lens), p.workspace(4)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        api.a3_paged_attention(p, qd, None, n, 4, qd, ws)          # out = q
    st.synchronize()
    assert np.array_equal(a, to_host(qd))


def test_captured_with_lengths_that_change():
    """A captured call follows lengths, page table and cache as they are at each replay; two graphs take turns on one workspace."""
    lens = [900, 70, 2500]
    p, held, rng = _filled(lens, Hq=4, Hkv=2)
    q = _values(rng, "bf16", 3, 4, 128)
    qd, n, ws = to_dev(q, "bf16"), idev(lens), p.workspace(3)
    outs = [torch.empty_like(qd) for _ in range(2)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    api.a3_paged_attention(p, qd, None, n, 3, outs[0], ws)
    torch.cuda.synchronize()
    for g, out in zip(graphs, outs):
        with torch.cuda.graph(g):
            api.a3_paged_attention(p, qd, None, n, 3, out, ws)
    for now in ([900, 70, 2500], [1, 0, 1], [0, 0, 0], [64, 65, 2049], [899, 70, 3]):
        n.copy_(idev(now))
        for g, out in zip(graphs, outs):
            out.fill_(5.0)
            g.replay()
            torch.cuda.synchronize()
            got = to_host(out)
            assert np.array_equal(got, _attend(p, q, now))
            _check_rows(p, held, q, got, now)


def test_a_cache_beyond_32_bits():
    """Pools of more than 4 GiB each, a request whose pages lie at both ends."""
    n_pages = (5 << 30) // (8 * 1024 * 128 * 2)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device="cuda")
    p = api.Pages(dtype="bf16", n_q_heads=16, n_kv_heads=8, head_dim=128, page_size=1024, n_pages=n_pages, page_table=table, rope_base=1e4,
                  n_pos=8)
    rng = np.random.default_rng(8)
    k, v = (_values(rng, "bf16", 2100, 8, 128) for _ in range(2))
    held = [put(p, 0, 0, k, v)]
    q = _values(rng, "bf16", 1, 16, 128)
    _check_rows(p, held, q, _attend(p, q, [2100]), [2100])


def test_two_calls_at_once():
    """Two streams over one cache, each with a workspace of its own."""
    lens = [3000, 17, 900]
    p, held, rng = _filled(lens)
    q = [_values(rng, "bf16", 3, 8, 128) for _ in range(2)]
    qd, n = [to_dev(x, "bf16") for x in q], idev(lens)
    out, ws, streams = [torch.empty_like(x) for x in qd], [p.workspace(3) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            api.a3_paged_attention(p, qd[i], None, n, 3, out[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        _check_rows(p, held, q[i], to_host(out[i]), lens)


@pytest.mark.parametrize("n_rows,Hq,Hkv", [(64, 8, 1), (65, 8, 8), (300, 32, 2), (520, 16, 16)])
def test_many_items_of_a_few_steps(n_rows, Hq, Hkv):
    """Shares that hold several items, whole and cut, on both sides of the number of shares; requests that do not exist between them."""
    rng = np.random.default_rng(n_rows)
    lens = [0, 200, 385, 1, 513]
    p, held, _ = _filled(lens, Hq=Hq, Hkv=Hkv, d=64)
    req = rng.integers(0, 5, n_rows)
    n = np.array([rng.integers(0, lens[r] + 1) for r in req])
    q = _values(rng, "bf16", n_rows, Hq, 64)
    named = np.where(rng.random(n_rows) < 0.2, 7, req)
    got = _attend(p, q, n, req=named)
    off = named == 7
    assert np.all(got[off] == 9.0)
    _check_rows(p, held, q[~off], got[~off], n[~off].tolist(), req=req[~off].tolist())
