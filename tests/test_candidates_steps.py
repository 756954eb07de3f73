"""What steps over trees and beams refuse before anything runs (on the CPU)."""
from types import SimpleNamespace as NS

import pytest

from paper_2511_17560_amd import stack


def test_trees_of_another_number_of_rows_than_the_step():
    tree = stack.TreeRows([[-1, 0], [-1]], [5, 0], device="cpu")
    bufs = NS(x=[0] * 8, logits=None, ws_tree=object())
    for n in (2, 4):
        with pytest.raises(ValueError, match="trees of 3 rows"):
            stack.decode_stack(NS(n_req=n), NS(rms_eps=1e-5), [], None, None, [], None, None, None, bufs, tree=tree)


def test_rows_that_are_no_groups_of_beams():
    out = NS(n_best=3, n_beams=3)
    with pytest.raises(ValueError, match="no groups of 3"):
        stack.beam_stack(NS(n_req=7), NS(rms_eps=1e-5), [], None, None, None, None, None, None, None, None, None, None, None, 4, out)
