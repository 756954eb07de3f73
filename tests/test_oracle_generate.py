"""Pins of the oracle for generating on the fused cache: closed forms and library routines."""
import numpy as np
import pytest
import torch
from scipy.special import log_softmax
from scipy.stats import entropy as scipy_entropy

from oracle import a3_oracle as ora
from oracle import generate_oracle as gen


@pytest.mark.parametrize("layout", [0, 1])
def test_turn_is_the_rotation_of_the_fusion_path(layout):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((7, 3, 64))
    pos = np.array([0, 1, 5, 100, 4096, 99999, 3])
    assert np.abs(gen.turn(x, pos, 1e4, layout) - ora.rope_rotate(x, pos, 1e4, layout)).max() < 1e-6   # the table is float32
    assert np.array_equal(gen.turn(x, np.zeros(7), 1e4, layout), x)


def test_attend_is_the_last_row_of_causal_attention():
    rng = np.random.default_rng(2)
    n, Hq, Hkv, d = 37, 6, 2, 64
    q, k, v = rng.standard_normal((n, Hq, d)), rng.standard_normal((n, Hkv, d)), rng.standard_normal((n, Hkv, d))
    want = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(t).repeat_interleave(g, 1).transpose(0, 1) for t, g in ((q, 1), (k, 3), (v, 3))), is_causal=True)
    assert np.abs(gen.attend(q[-1], k, v, d ** -0.5) - want[:, -1].numpy()).max() < 1e-12
    assert np.array_equal(gen.attend(q[0], k[:0], v[:0], 1.0), np.zeros((Hq, d)))
    assert np.abs(gen.attend(0 * q[0], k, v, 1.0) - np.repeat(v.mean(0), 3, 0)).max() < 1e-12


def test_log_probs_entropy_and_top():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 101)) * 4
    x[1, 7:20] = -np.inf
    lp = gen.log_probs(x)
    assert np.allclose(lp, log_softmax(x, -1), atol=1e-12) and np.allclose(gen.entropy(lp), scipy_entropy(np.exp(lp), axis=-1))
    assert np.allclose(gen.entropy(gen.log_probs(np.zeros((1, 64)))), np.log(64))
    assert np.array_equal(gen.given(lp, [[3, -1], [7, 101], [0, 100], [1, 1], [2, 5]])[:2], [[lp[0, 3], -np.inf], [-np.inf, -np.inf]])
    tied = np.array([[1.0, 5.0, -np.inf, 5.0, np.nan, -0.0, 0.0]])
    assert gen.top(tied, 7).tolist() == [[1, 3, 0, 5, 6, 2, 4]]
    for bad in (np.array([[1.0, np.nan]]), np.array([[1.0, np.inf]]), np.full((1, 4), -np.inf)):
        assert np.isnan(gen.log_probs(bad)).all()
