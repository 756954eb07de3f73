"""Steps of beams whose runs differ in length: every target takes over as many slots as its source has (on the CPU: what the move gets)."""
from types import SimpleNamespace as NS

import torch

from paper_2511_17560_amd import api, stack


def test_runs_are_as_long_as_their_sources(monkeypatch):
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)
    n, rows = 6, i32(2, 0, 0, 5, -1, 4)                                  # (a group with fewer continuations than beams)
    got = {}

    def select(logits, score, done, end_token, out, stream=None):
        out.row.view(-1)[:n] = rows

    def move(layers, src_req, src_slot, dst_req, dst_slot, n_slots, max_slots, n_sets, set_size, stream=None):
        got.update(src=src_req.flatten()[:n].tolist(), run=n_slots.flatten().tolist())

    monkeypatch.setattr(api, "a3_beam_select", select)
    monkeypatch.setattr(api, "a3_paged_move", move)
    monkeypatch.setattr(api, "torch_stream", lambda stream: None)
    monkeypatch.setattr(stack, "decode_stack", lambda *a, **k: dict(logits=torch.zeros(n, 50)))
    monkeypatch.setattr(api, "lib", lambda: NS(a3_beam_select_ws_bytes=lambda *a: 256))
    new = lambda: torch.zeros(2, 3, dtype=torch.int32)
    out = NS(n_beams=3, n_best=3, row=new(), token=new(), score=torch.zeros(2, 3), ws=torch.zeros(256, dtype=torch.uint8))
    bufs = NS(rows=torch.arange(n, dtype=torch.int32), source=torch.zeros(n, dtype=torch.int32), runs=torch.zeros(n, dtype=torch.int32))
    slots = torch.zeros(n, dtype=torch.int32)
    stack.beam_stack(NS(n_req=n), None, [], None, torch.zeros(n, 4), NS(pages=[]), slots, slots, slots, bufs, torch.zeros(50, 4), torch.zeros(n), slots,
                     i32(7, 8, 9, 10, 11, 12), 20, out)
    want = [9, 7, 7, 12, None, 11]                                       # (nothing moves where the row is -1)
    assert got["src"] == rows.tolist() and len(got["run"]) == n
    assert all(w is None or r == w for r, w in zip(got["run"], want))
