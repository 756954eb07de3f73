"""Alternatives of rows in which whole halves of what a thread reads are NaN: every index is valid, NaN comes last.

Indexes are compared exactly (fp32 and bf16 logits are the oracle's, ties go to the lower index).  Such rows have no distribution:
their log probabilities and entropy are NaN."""
import numpy as np
import pytest
import torch

from oracle import generate_oracle as gen
from paper_2511_17560_amd import api

pytestmark = pytest.mark.gpu


def _rows(rng, n, vocab, dtype):
    """Rows of several kinds in turn; returned as they are stored, in float64, with the tensor."""
    v = np.arange(vocab)
    per = 8 if dtype is torch.bfloat16 else 4
    x = rng.standard_normal((n, vocab)) * 3
    for i in range(n):
        kind = i % 6
        if kind == 0:
            x[i, 1::2] = np.nan
        elif kind == 1:
            x[i, ::2] = np.nan
        elif kind == 2:                                              # one thread's odd values, and two far above all others beside them
            mine = (v // per) % 256 == 7
            x[i, mine & (v % 2 == 1)] = np.nan
            x[i, 7 * per], x[i, min(7 * per + 4096, vocab - 2)] = 90.0, 80.0
        elif kind == 3:                                              # a few numbers among NaN
            keep = rng.permutation(vocab)[:20]
            row = np.full(vocab, np.nan)
            row[keep] = x[i, keep]
            x[i] = row
        elif kind == 4:                                              # the even half -inf, the odd one NaN
            x[i, 1::2] = np.nan
            x[i, ::2] = -np.inf
            x[i, 100] = 1.0
    t = torch.from_numpy(x).to(dtype).cuda()
    return t, t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,vocab", [(1030, 8200), (64, 128256), (1024, 16390), (2, 8192), (6, 171000)])
def test_halves_of_nan(n, vocab, dtype):
    rng = np.random.default_rng(vocab)
    t, x = _rows(rng, n, vocab, dtype)
    some = np.unique(np.concatenate([np.arange(min(n, 12)), rng.integers(0, n, 40), np.arange(max(n - 6, 0), n)]))
    want, lp = gen.top(x[some], 64), gen.log_probs(x[some])
    for n_top in (1, 2, 20, 64):
        out = api.TokenLogprobs(n, vocab, 0, n_top)
        out.top_idx.fill_(-7)
        out.ws.fill_(255)
        api.a3_token_logprobs(t, None, out)
        torch.cuda.synchronize()
        idx = out.top_idx.cpu().numpy()
        assert idx.min() >= 0 and idx.max() < vocab
        assert np.array_equal(idx[some], want[:, :n_top])
        got, ref = out.top_logprob.double().cpu().numpy()[some], np.take_along_axis(lp, want[:, :n_top], -1)
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        ok = np.isfinite(ref)
        assert np.all(np.abs(got[ok] - ref[ok]) <= 1e-5 * (1 + np.abs(ref[ok])))
