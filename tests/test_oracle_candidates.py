"""Pins of the oracle for several candidates: closed forms, library routines, and brute force."""
import numpy as np
import torch

from oracle import candidates_oracle as cand
from oracle import generate_oracle as gen


def test_ancestors_and_their_bits():
    seen = cand.ancestors([-1, 0, 0, 1, 3])
    assert seen.astype(int).tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 1, 0, 1, 0], [1, 1, 0, 1, 1]]
    assert cand.pack(seen, 1)[:, 0].tolist() == [1, 3, 5, 11, 27]
    chain = cand.ancestors(list(range(-1, 69)))
    assert np.array_equal(chain, np.tri(70, dtype=bool))
    assert cand.pack(chain, 3)[69].view(np.uint32).tolist() == [2 ** 32 - 1, 2 ** 32 - 1, 63]


def test_a_chain_is_causal_attention():
    rng = np.random.default_rng(2)
    n, Hq, Hkv, d, before = 11, 6, 2, 64, 20
    q = rng.standard_normal((before + n, Hq, d))
    k, v = rng.standard_normal((2, before + n, Hkv, d))
    want = torch.nn.functional.scaled_dot_product_attention(
        *(torch.from_numpy(t).repeat_interleave(g, 1).transpose(0, 1) for t, g in ((q, 1), (k, 3), (v, 3))), is_causal=True)
    got = cand.tree_attend(q[before:], k, v, before, np.tri(n, dtype=bool), d ** -0.5)
    assert np.abs(got - want[:, before:].transpose(0, 1).numpy()).max() < 1e-12


def test_a_branch_is_the_text_of_its_ancestors():
    rng = np.random.default_rng(3)
    parents = [-1, 0, 0, 2, 1, 3]
    q, (k, v) = rng.standard_normal((6, 4, 64)), rng.standard_normal((2, 9, 2, 64))
    got = cand.tree_attend(q, k, v, 3, cand.ancestors(parents), 0.2)
    for j, slots in ((0, [0, 1, 2, 3]), (4, [0, 1, 2, 3, 4, 7]), (5, [0, 1, 2, 3, 5, 6, 8])):
        assert np.abs(got[j] - gen.attend(q[j], k[slots], v[slots], 0.2)).max() < 1e-13
    assert np.array_equal(cand.tree_attend(q[:1], k[:0], v[:0], 0, np.zeros((1, 0), bool), 0.2), np.zeros((1, 4, 64)))


def test_follow():
    parents, tokens = [-1, 0, 0, 2, 2, 4], [9, 5, 6, 7, 8, 3]
    assert cand.follow([6, 0, 8, 0, 3, 1], tokens, parents, 16) == [0, 2, 4, 5]
    assert cand.follow([6, 0, 8, 0, 3, 1], tokens, parents, 2) == [0, 2]
    assert cand.follow([4, 0, 8, 0, 3, 1], tokens, parents, 16) == [0]
    assert cand.follow([5, 5, 0, 0, 0, 0], [1, 5, 5, 5, 0, 0], [-1, 0, 0, 1, 9, -1], 16) == [0, 1, 3]
    assert cand.follow([], [], [], 16) == []


def test_moves_of_a_set_happen_at_once():
    cache = [np.arange(6), 10 + np.arange(6)]
    got = cand.move(cache, [[(0, 1, 1, 1, 3), (1, 1, 0, 1, 3)]])
    assert got[0].tolist() == [0, 11, 12, 13, 4, 5] and got[1].tolist() == [10, 1, 2, 3, 14, 15]
    got = cand.move(cache, [[(0, 0, 0, 0, 1), (0, 2, 0, 1, 1), (0, 5, 0, 2, 1)]])
    assert got[0].tolist() == [0, 2, 5, 3, 4, 5]


def test_beams_are_the_best_of_everything():
    rng = np.random.default_rng(5)
    x, score = rng.standard_normal((3, 50)) * 3, np.array([-1.0, -2.5, -0.3])
    total = torch.from_numpy(score)[:, None] + torch.log_softmax(torch.from_numpy(x), -1)
    value, at = total.flatten().topk(7)
    s, b, t = cand.beams(x, score, None, 0, 7)
    assert np.allclose(s, value.numpy(), atol=1e-12) and np.array_equal(b * 50 + t, at.numpy())
    s, b, t = cand.beams(x, [-1.0, 0.5, -np.inf], [0, 1, 0], 49, 60)
    assert (s[0], b[0], t[0]) == (0.5, 1, 49) and np.array_equal(np.sort(t[1:51]), np.arange(50)) and (b[1:51] == 0).all()
    assert np.isneginf(s[51:]).all() and (b[51:] == -1).all() and (t[51:] == -1).all()
    s, b, t = cand.beams(np.zeros((2, 3)), [0.0, 0.0], None, 0, 4)
    assert b.tolist() == [0, 0, 0, 1] and t.tolist() == [0, 1, 2, 0]
    x[0, 3], x[1] = np.nan, -np.inf
    assert set(cand.beams(x, score, None, 0, 5)[1].tolist()) == {2}
