"""A group whose committed length is negative counts as one of 0 wherever it is read: attention, the accepted path's slots, and the rows of a step."""
import numpy as np
import pytest
import torch

from paper_2511_17560_amd import api
from gpu_util import idev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[-1, 5, -2 ** 31], [0, 5, 0]])
def test_slots_of_accepted_paths(lens):
    picked, parents, tokens = [7, 8, 1, 4, 9, 6, 6, 2], [-1, 0, 0, -1, 0, -1, 0, 1], [3, 5, 7, 3, 4, 3, 1, 6]
    out = api.TreeAccepted(3, 8, 4)
    for t in (out.src_slot, out.dst_slot):
        t.fill_(-77)
    out.picked.copy_(idev(picked))
    api.a3_tree_accept(None, idev(tokens), idev(parents), idev([0, 3, 5, 8]), idev(lens), 8, 3, out)
    torch.cuda.synchronize()
    assert out.path.tolist() == [[0, 2, -1, -1], [0, 1, -1, -1], [0, -1, -1, -1]]
    assert out.src_slot.tolist() == [[0, 2, -1, -1], [5, 6, -1, -1], [0, -1, -1, -1]]
    assert out.dst_slot.tolist() == [[0, 1, -1, -1], [5, 6, -1, -1], [0, -1, -1, -1]]
