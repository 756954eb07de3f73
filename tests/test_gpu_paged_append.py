"""Appending to a paged cache, against the float64 oracle.

Tolerances.  Turned in float32 (two products and a sum of values up to |x|: 3 * 2^-24 of the pair's norm) and rounded once:
fp32 4 * 2^-24 of the row's largest pair, bf16 half a step (2^-8 of the element) and that.  8-bit pages: codes and scales are
the oracle's, bit for bit (both sides form them in float64)."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as gen
from oracle import q8_oracle as q8
from paper_2511_17560_amd import api
from gpu_util import idev, to_dev, to_host
from paged_util import get, make_pages, parts
import a3_synth as synth

pytestmark = pytest.mark.gpu


def _values(rng, dtype, *shape):
    return synth.round_to_storage(rng.standard_normal(shape, dtype=np.float32), dtype).astype(np.float64)


def _near(got, want, dtype):
    bound = 4 * 2.0 ** -24 * np.sqrt(2) * np.abs(want).max(-1, keepdims=True)
    return np.all(np.abs(got - want) <= bound + (0 if dtype == "f32" else 2.0 ** -8 * np.abs(want)))


@pytest.mark.parametrize("q8_pages", [False, True])
@pytest.mark.parametrize("dtype,d,Hq,Hkv,page,layout", [("bf16", 128, 32, 8, 64, 1), ("bf16", 128, 28, 4, 32, 0), ("bf16", 64, 3, 3, 128, 1),
                                                        ("f32", 64, 8, 8, 64, 0), ("f32", 128, 16, 1, 32, 1)])
def test_new_tokens(dtype, d, Hq, Hkv, page, layout, q8_pages):
    """Rows of several requests in any order, slots that are not positions, first and last slot of a page; everything else stays."""
    rng = np.random.default_rng(d + Hq + page)
    lens = [1, page, page + 1, 3 * page - 1, 200]
    p = make_pages(lens, dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, page=page, q8=q8_pages, layout=layout, base=5e5, n_pos=5000, fill=3.0)
    before = [t.clone() for t in (p.k_pool, p.v_pool)]
    req, slot = np.array([4, 2, 0, 3, 1, 2]), np.array([199, page, 0, 3 * page - 2, page - 1, 0])
    pos = np.array([4999, 0, 77, 1234, 1, 4095])
    n = len(req)
    q, k, v = _values(rng, dtype, n, Hq, d), _values(rng, dtype, n, Hkv, d), _values(rng, dtype, n, Hkv, d)
    k[3] = 0.0
    qd = to_dev(q, dtype)
    api.a3_paged_append(p, to_dev(k, dtype), to_dev(v, dtype), idev(req), idev(slot), idev(pos), n, q=qd, q_out=qd)
    torch.cuda.synchronize()
    assert _near(to_host(qd), gen.turn(q, pos, 5e5, layout), dtype)
    turned = gen.turn(k, pos, 5e5, layout)
    for i in range(n):
        got_k, got_v = (t[0] for t in get(p, req[i], slot[i], slot[i] + 1))
        if q8_pages:
            for got, want in ((got_k, turned[i]), (got_v, v[i])):
                assert np.array_equal(got, q8.dequantize_q8(*q8.quantize_q8(want[None]))[0])
        else:
            assert _near(got_k, turned[i], dtype) and np.array_equal(got_v, v[i])
    # nothing but the named slots was written
    table = p.page_table.cpu().numpy()
    for pool, old in zip((p.k_pool, p.v_pool), before):
        for now, was in zip(*(parts(p, t) if q8_pages else [t] for t in (pool, old))):
            rest = torch.ones(now.shape[:3], dtype=torch.bool, device="cuda")
            for r, s in zip(req, slot):
                rest[table[r, s // page], :, s % page] = False
            assert torch.equal(now[rest], was[rest])


@pytest.mark.parametrize("q8_pages", [False, True])
@pytest.mark.parametrize("dtype,lens", [("bf16", [700, 1, 65]), ("f32", [33, 257])])
def test_a_prompt_as_it_stands(dtype, lens, q8_pages):
    """row_pos NULL: the fused caches of a batch, by the layout's own tables, not turned."""
    d = 128 if dtype == "bf16" else 64
    w = synth.custom(synth.ModelShape("p", dtype, 256, 4, 2, d, 1e4), [[n - 1] if n > 1 else [] for n in lens], [1] * len(lens))
    lay = api.Layout.from_workload(w)
    p = make_pages(lens, dtype=dtype, Hq=4, Hkv=2, d=d, q8=q8_pages)
    rng = np.random.default_rng(5)
    T = w.total_tokens
    k, v = _values(rng, dtype, T, 2, d), _values(rng, dtype, T, 2, d)
    k[1, 0, :4] = [127.0, 62.5, -63.5, 0.5]      # ties of the codes: half to even
    k[1, 0, 4:] = 0.0
    api.a3_paged_append(p, to_dev(k, dtype), to_dev(v, dtype), lay.tok_req, lay.tok_pos, None, T)
    torch.cuda.synchronize()
    for r, n in enumerate(lens):
        a = int(w.seg_start[r])
        for got, want in zip(get(p, r, 0, n), (k[a:a + n], v[a:a + n])):
            assert np.array_equal(got, q8.dequantize_q8(*q8.quantize_q8(want)) if q8_pages else want)


def test_rows_that_do_not_exist_are_skipped():
    p = make_pages([70, 70], n_pos=100, fill=3.0)
    table = p.page_table.cpu().numpy()
    bad_table = table.copy()
    bad_table[1, 1] = p.struct.n_pages           # a page outside the pool
    p.page_table.copy_(torch.from_numpy(bad_table))
    before = [t.clone() for t in (p.k_pool, p.v_pool)]
    rows = [(-1, 0, 0), (2, 0, 0), (0, -1, 0), (0, 3 * 64, 0), (0, 2 * 64, 0), (1, 64, 0), (0, 0, -1), (0, 0, 100), (2 ** 31 - 1, 0, 0), (0, 2 ** 31 - 1, 0)]
    req, slot, pos = (np.array(c) for c in zip(*rows))
    one = torch.ones((len(rows), 2, 128), dtype=torch.bfloat16, device="cuda")
    q = torch.full((len(rows), 8, 128), 2.0, dtype=torch.bfloat16, device="cuda")
    q_out = torch.full_like(q, 7.0)
    api.a3_paged_append(p, one, one, idev(req), idev(slot), idev(pos), len(rows), q=q, q_out=q_out)
    torch.cuda.synchronize()
    assert torch.equal(p.k_pool, before[0]) and torch.equal(p.v_pool, before[1]) and bool((q_out == 7.0).all())


def test_pools_beyond_32_bits():
    """A pool of more than 4 GiB: the last page's last slot."""
    n_pages = (5 << 30) // (8 * 1024 * 128 * 2)
    table = torch.tensor([[n_pages - 1, 0]], dtype=torch.int32, device="cuda")
    p = api.Pages(dtype="bf16", n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=1024, n_pages=n_pages, page_table=table, rope_base=1e4,
                  n_pos=8)
    rng = np.random.default_rng(6)
    k, v = _values(rng, "bf16", 2, 8, 128), _values(rng, "bf16", 2, 8, 128)
    api.a3_paged_append(p, to_dev(k, "bf16"), to_dev(v, "bf16"), idev([0, 0]), idev([1023, 1024]), None, 2)
    torch.cuda.synchronize()
    for i in range(2):
        for got, want in zip(get(p, 0, 1023 + i, 1024 + i), (k, v)):
            assert np.array_equal(got[0], want[i])
