"""Rows of the product with the vocabulary's weights that do not exist: what a padded list names is neither read nor written.

Tolerance of the others: 8 sqrt(h) 2^-24 sum |x w|, as in tests/test_gpu_logits.py."""
import numpy as np
import pytest
import torch

from paper_2511_17560_amd import api, stack
from gpu_util import idev, to_dev, to_host
import a3_synth as synth

pytestmark = pytest.mark.gpu


def _layout(dtype, h, T):
    return api.Layout.decode(dtype=dtype, n_q_heads=2, n_kv_heads=1, head_dim=128 if dtype == "bf16" else 64, hidden=h, rope_base=1e4, n_req=T)


def _values(rng, dtype, *shape):
    return synth.round_to_storage(rng.standard_normal(shape, dtype=np.float32), dtype).astype(np.float64)


@pytest.mark.parametrize("n,vocab,tb", [(1, 300, -1), (17, 513, -1), (70, 20001, -1), (150, 9000, -1)] + [(40, 700, tb) for tb in (2, 3, 4, 5, 6, 7)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_do_not_exist(dtype, n, vocab, tb, tuning):
    if tb >= 0:
        tuning("gemm_tb", tb)
    h, T = 192, 33
    rng = np.random.default_rng(vocab + n)
    lay, x, w = _layout(dtype, h, T), _values(rng, dtype, T, h), _values(rng, dtype, vocab, h)
    idx = rng.integers(0, T, n)
    gone = np.arange(n) % 3 == 0
    idx[gone] = np.resize([-1, T, 2 ** 31 - 1, -2 ** 31], gone.sum())
    logits = torch.full((n, vocab), 7.0, device="cuda")
    api.a3_lm_head(lay, to_dev(x, dtype), idev(idx), n, to_dev(w, dtype), logits)
    torch.cuda.synchronize()
    got, ok = to_host(logits), ~gone
    assert np.all(got[gone] == 7.0)
    rows = x[idx[ok]]
    assert np.all(np.abs(got[ok] - rows @ w.T) <= 8 * np.sqrt(h) * 2.0 ** -24 * (np.abs(rows) @ np.abs(w).T))


def test_a_list_of_rows_needs_all_hidden_rows():
    """The list's range is [0, total_tokens), which the kernel goes by: fewer rows behind ``hidden`` are refused."""
    lay = _layout("f32", 64, 10)
    hidden, w, logits = torch.zeros((10, 64), device="cuda"), torch.zeros((5, 64), device="cuda"), torch.zeros((2, 5), device="cuda")
    api.a3_lm_head(lay, hidden, idev([9, 0]), 2, w, logits)
    api.a3_lm_head(lay, hidden[:2], None, 2, w, logits)
    with pytest.raises(ValueError):
        api.a3_lm_head(lay, hidden[:9], idev([0, 1]), 2, w, logits)
    with pytest.raises(ValueError):
        stack.score_tokens(lay, hidden[:9], idev([0, 1]), 2, w, None, api.TokenLogprobs(2, 5, 0, 1))
    torch.cuda.synchronize()
