"""NaN and infinities in seen slots, however the steps of a row are cut over workgroups.

A row's result is the softmax over all its slots: a NaN logit makes the row's head NaN, a NaN value its coordinate, whether the
row is whole in one workgroup or a piece of it (a single slot, at lengths of one more than a step) holds nothing but the NaN.
Tolerances of the finite outputs are those of tests/test_gpu_paged_attention.py: 1e-4 of the largest value seen, bf16 2^-8 of the
element more (the output's rounding)."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as gen
from paper_2511_17560_amd import api
from gpu_util import idev, to_dev, to_host
from paged_util import make_pages, parts, put
import a3_synth as synth

pytestmark = pytest.mark.gpu

# rows beside the one looked at: none (every step a workgroup of its own, joined by item), many (joined by workgroup; several steps a
# workgroup, so that most rows are whole in one and some are cut)
BESIDE = [0, 70, 300]


def _values(rng, dtype, *shape):
    return synth.round_to_storage(rng.standard_normal(shape, dtype=np.float32), dtype).astype(np.float64)


def _filled(n, dtype, q8, Hq=4, Hkv=2, d=128, **kw):
    rng = np.random.default_rng(n)
    p = make_pages([n, n], dtype=dtype, Hq=Hq, Hkv=Hkv, d=d, q8=q8, **kw)
    held = [put(p, r, 0, _values(rng, dtype, n, Hkv, d), _values(rng, dtype, n, Hkv, d)) for r in range(2)]
    return p, held, rng


def _attend(p, q, req, lens):
    out = torch.full(q.shape, 9.0, dtype=api.torch_dtype(p.dtype), device="cuda")
    api.a3_paged_attention(p, to_dev(q, p.dtype), idev(req), idev(lens), len(req), out, p.workspace(len(req)).fill_(255))
    torch.cuda.synchronize()
    return to_host(out)


def _near(got, want, top, dtype):
    return np.all(np.abs(got - want) <= 1e-4 * top + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0))


def _set(p, r, slot, head, what):
    """A key or a value row of one slot and head becomes NaN: the elements, or the scale of an 8-bit page."""
    page = int(p.page_table[r, slot // p.struct.page_size])
    pool, at = (p.k_pool if what == "key" else p.v_pool), slot % p.struct.page_size
    (parts(p, pool)[1] if p.q8 else pool)[page, head, at] = float("nan")


@pytest.mark.parametrize("beside", BESIDE)
@pytest.mark.parametrize("n", [65, 129, 257, 1025])
@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False), ("f32", True)])
@pytest.mark.parametrize("what", ["key", "value"])
def test_the_last_slot_alone_is_nan(what, dtype, q8, n, beside):
    """The newest token's key or value is NaN and alone in its step: its head is NaN, the other head and the other request are not."""
    p, held, rng = _filled(n, dtype, q8)
    _set(p, 0, n - 1, 1, what)
    req = np.array([0, 1] + [0] * beside)
    lens = np.array([n, n] + [n - 1] * beside)                      # (the rows beside it end before the NaN)
    q = _values(rng, dtype, len(req), 4, 128)
    got = _attend(p, q, req, lens)
    assert np.isnan(got[0, 2:]).all()
    for i in range(len(req)):
        k, v = (t[:lens[i]] for t in held[req[i]])
        want = gen.attend(q[i], k, v, 128 ** -0.5)
        heads = slice(0, 2) if i == 0 else slice(0, 4)
        assert _near(got[i, heads], want[heads], np.abs(v).max(), dtype)


@pytest.mark.parametrize("beside", BESIDE)
@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("bf16", True), ("f32", False)])
def test_a_step_of_nan_in_the_middle_of_many(dtype, q8, beside):
    """Of a row of some 20 steps one is NaN throughout, in the keys of one head."""
    p, held, rng = _filled(2500, dtype, q8)
    for slot in range(1280, 1408):
        _set(p, 0, slot, 0, "key")
    req = np.array([0] + [0] * beside)
    lens = np.array([2500] + [1280] * beside)
    q = _values(rng, dtype, len(req), 4, 128)
    got = _attend(p, q, req, lens)
    assert np.isnan(got[0, :2]).all()
    for i in range(len(req)):
        k, v = (t[:lens[i]] for t in held[0])
        heads = slice(2, 4) if i == 0 else slice(0, 4)
        assert _near(got[i, heads], gen.attend(q[i], k, v, 128 ** -0.5)[heads], np.abs(v).max(), dtype)


@pytest.mark.parametrize("beside", BESIDE)
@pytest.mark.parametrize("n", [385, 2049])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_nan_value_far_below_the_rows_maximum(dtype, n, beside):
    """The step that holds the NaN has weights that float cannot hold beside the first slots' (logits 200 apart): 0 times NaN is NaN
    in its coordinate, and what is finite adds nothing to the others.  A step of -inf logits adds nothing either."""
    p, held, rng = _filled(n, dtype, False, sm_scale=1.0)
    k, v = (t.copy() for t in held[0])
    k[:, :, :] = 0.0
    k[0, :, 0], k[1:, :, 0] = 100.0, -100.0                         # logits of +-100 with q = e_0
    k[128:256, :, 0] = -np.inf
    v[n - 1, 1, 3] = np.nan
    put(p, 0, 0, k, v)
    req, lens = np.array([0] * (1 + beside)), np.array([n] + [n - 1] * beside)
    q = np.zeros((len(req), 4, 128))
    q[:, :, 0] = 1.0
    got = _attend(p, q, req, lens)
    want = np.repeat(v[0], 2, 0)                                    # all the weight is on slot 0
    assert np.isnan(got[0, 2:, 3]).all()
    ok = np.ones(got.shape, bool)
    ok[0, 2:, 3] = False
    assert _near(got[ok], np.broadcast_to(want, got.shape)[ok], np.abs(v[0]).max(), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_nan_queries_and_rows_without_a_finite_logit(dtype):
    """A NaN query, and keys that are all at -inf logits: no distribution, NaN, in rows of one step and of several."""
    n = 300
    p, held, rng = _filled(n, dtype, False)
    k, v = held[0]
    put(p, 0, 0, np.full_like(k, -np.inf), v)
    q = synth.round_to_storage((np.abs(_values(rng, dtype, 5, 4, 128)) + 0.5).astype(np.float32), dtype).astype(np.float64)
    q[2, 1, 7] = np.nan
    got = _attend(p, q, [0, 0, 1, 1, 0], [1, n, n, n, 0])
    assert np.isnan(got[:2]).all() and np.isnan(got[2, 1]).all() and np.all(got[4] == 0.0)
    k, v = held[1]
    heads = [0, 2, 3]
    assert _near(got[2, heads], gen.attend(q[2], k, v, 128 ** -0.5)[heads], np.abs(v).max(), dtype)
    assert _near(got[3], gen.attend(q[3], k, v, 128 ** -0.5), np.abs(v).max(), dtype)
