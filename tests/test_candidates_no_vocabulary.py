"""Steps over candidates need logits: without the vocabulary's weights they are refused, and nothing runs (no GPU needed)."""
from types import SimpleNamespace as NS

import pytest
import torch

from paper_2511_17560_amd import api, stack


@pytest.fixture
def ran(monkeypatch):
    names = []
    for module, name in ((stack, "decode_stack"), (api, "a3_tree_accept"), (api, "a3_beam_select"), (api, "a3_paged_move")):
        monkeypatch.setattr(module, name, lambda *a, name=name, **k: names.append(name) or dict(logits=None))
    return names


def test_a_verification_step(ran):
    """(It would follow the picks of the step before.)"""
    tree = stack.TreeRows([[-1, 0], [-1]], [5, 0], max_path=4, device="cpu")
    out = NS(max_path=4, picked=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="logits"):
        stack.verify_stack(NS(n_req=3), None, [], None, torch.zeros(3, 4), NS(pages=[]), tree, None, None, out)
    assert ran == []


def test_a_step_of_beams(ran):
    with pytest.raises(ValueError, match="logits"):
        stack.beam_stack(NS(n_req=4), None, [], None, torch.zeros(4, 4), NS(pages=[]), None, None, None, None, None, None, None, None, 4, NS(n_best=2, n_beams=2))
    assert ran == []
