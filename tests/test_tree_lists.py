"""Lists that describe no trees, or not as many, are refused when the rows of a step are made (no GPU needed)."""
import numpy as np
import pytest

from paper_2511_17560_amd import stack


@pytest.mark.parametrize("kw", [dict(lens=[5]), dict(lens=[5, 7, 9]), dict(tokens=np.zeros(4)), dict(tokens=np.zeros(6)), dict(reqs=[0]), dict(reqs=[0, 1, 2]),
                                dict(positions=[1]), dict(positions=[1, 2, 3]), dict(max_path=0), dict(max_path=65), dict(max_rows=1025)])
def test_lists_that_are_no_trees(kw):
    a = dict(lens=[5, 7], tokens=np.zeros(5), reqs=[0, 1], positions=None) | kw
    with pytest.raises(ValueError):
        stack.TreeRows([[-1, 0, 0], [-1, 0]], device="cpu", **a)
    with pytest.raises(ValueError):
        stack.TreeRows([[-1] + [0] * 1024], [5], device="cpu")


def test_one_tree_and_lists_of_more():
    """(NumPy would repeat them.)"""
    for kw in (dict(lens=[5, 7]), dict(lens=[5], reqs=[0, 1]), dict(lens=[5], positions=[1, 2])):
        with pytest.raises(ValueError):
            stack.TreeRows([[-1]], device="cpu", **kw)


def test_tokens_of_equal_trees_as_rows():
    a, b = (stack.TreeRows([[-1, 0, 0]] * 2, [5, 7], tokens, device="cpu") for tokens in (np.arange(6), np.arange(6).reshape(2, 3)))
    assert a.tokens.tolist() == b.tokens.flatten().tolist()
