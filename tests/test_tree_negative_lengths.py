"""Rows of trees behind a negative committed length stand where those behind a length of 0 do (no GPU needed)."""
import numpy as np
import pytest

from paper_2511_17560_amd import stack


@pytest.mark.parametrize("positions", [None, [3, 9]])
def test_rows_of_a_step(positions):
    trees = [[-1, 0, 1], [-1, 0]]
    a, b = (stack.TreeRows(trees, lens, positions=positions, device="cpu") for lens in ([-4, 6], [0, 6]))
    for name in ("row_slot", "row_pos", "row_req", "mask", "parent", "path_req"):
        assert np.array_equal(getattr(a, name).numpy(), getattr(b, name).numpy()), name
    assert a.row_slot.tolist() == [0, 1, 2, 6, 7]
