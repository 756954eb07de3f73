"""Steps of beams without run lengths move one slot a beam, as the moves without lengths do (no GPU needed: the calls are recorded)."""
from types import SimpleNamespace as NS

import torch

from paper_2511_17560_amd import api, stack


def test_no_lengths(monkeypatch):
    got = []
    monkeypatch.setattr(api, "a3_beam_select", lambda *a, **k: None)
    monkeypatch.setattr(api, "a3_paged_move", lambda layers, src_req, src_slot, dst_req, dst_slot, n_slots, *a, **k: got.append(n_slots))
    monkeypatch.setattr(api, "torch_stream", lambda stream: None)
    monkeypatch.setattr(stack, "decode_stack", lambda *a, **k: dict(logits=torch.zeros(4, 50)))
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    out = api.BeamChoice(2, 2, 50, 2, device="cpu")
    bufs = NS(rows=i32(4), source=i32(4), runs=i32(4))
    stack.beam_stack(NS(n_req=4), None, [], None, torch.zeros(4, 4), NS(pages=[]), i32(4), i32(4), i32(4), bufs, torch.zeros(50, 4), torch.zeros(4), i32(4), None, 1, out)
    assert got == [None]
