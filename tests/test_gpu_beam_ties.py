"""Beams whose scores are so large that a double holds no difference between the worths of their tokens: within a beam the larger logit goes
first all the same, across beams equal worths go by the beam.

Scores of -1e30 and below leave score + x - m - log Z at the score exactly, in the kernel as here; with -1e9 a double's step is 1e-7, so beams lie
1000 apart and logits differ by multiples of 1e-8."""
import numpy as np
import pytest
import torch

from paper_2511_17560_amd import api
from gpu_util import idev, to_host

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _call(x, score, n_beams, n_best, done=None, dtype="f32"):
    d = torch.from_numpy(x).to(TYPES[dtype]).cuda()
    out = api.BeamChoice(len(x) // n_beams, n_beams, x.shape[1], n_best)
    api.a3_beam_select(d, torch.tensor(score, dtype=torch.float32, device="cuda"), None if done is None else idev(done), 1, out)
    torch.cuda.synchronize()
    return out, d.double().cpu().numpy()


def _order(row, n):
    return np.lexsort((np.arange(len(row)), -row))[:n]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,n_best", [(3, 3), (300, 5), (8200, 64), (32003, 8), (128256, 16), (170000, 64)])
def test_one_worth_for_all_tokens(vocab, n_best, dtype):
    rng = np.random.default_rng(vocab)
    for score in (-1e30, 1e25, -3.4028234e38):
        x = rng.standard_normal((6, vocab)).astype(np.float32) * 2
        x[0, 0], x[0, vocab - 1] = -7.0, 9.0
        out, stored = _call(x, [score] * 6, 3, n_best, dtype=dtype)
        for g in range(2):
            want = [(g * 3 + b, t) for b in range(3) for t in _order(stored[g * 3 + b], n_best)][:n_best]
            assert out.row[g].tolist() == [r for r, _ in want] and out.token[g].tolist() == [int(t) for _, t in want]
            assert bool((out.score[g] == torch.tensor(score, dtype=torch.float32)).all())


@pytest.mark.parametrize("vocab", [300, 32003, 128256])
def test_worths_within_a_step_of_a_double(vocab):
    rng = np.random.default_rng(vocab)
    x = (rng.integers(0, 200, (4, vocab)) * 1e-8).astype(np.float32)
    out, stored = _call(x, [0.0, -1e9, -2e9, -3e9], 4, 64)
    assert out.row[0].tolist() == [0] * 64 and out.token[0].tolist() == _order(stored[0], 64).tolist()
    out, stored = _call(x, [-4e9, -1e9, -2e9, -3e9], 4, 64)
    assert out.row[0].tolist() == [1] * 64 and out.token[0].tolist() == _order(stored[1], 64).tolist()


def test_ended_beams_among_them():
    """Worths all equal: the beams in turn, an ended one with one candidate."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 2000)).astype(np.float32)
    x[0, 7:], x[2, 3:] = -np.inf, -np.inf
    out, stored = _call(x, [-1e30] * 4, 4, 14, done=[0, 1, 0, 0])
    want = [(0, t) for t in _order(stored[0], 7)] + [(1, 1)] + [(2, t) for t in _order(stored[2], 3)] + [(3, t) for t in _order(stored[3], 3)]
    assert out.row[0].tolist() == [r for r, _ in want] and out.token[0].tolist() == [int(t) for _, t in want]
    assert np.isfinite(to_host(out.score)).all()
