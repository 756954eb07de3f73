"""Steps over trees and beams whose outputs, buffers or lists do not fit are refused before any call is made, so that nothing of the caches or
the residual stream has changed (no GPU needed: the calls are recorded, not made)."""
import numpy as np
import pytest
import torch

import a3_synth as synth
from paper_2511_17560_amd import api, stack

SHAPE, VOCAB = synth.ModelShape("early", "bf16", 512, 8, 2, 128, 5e5, synth.ROPE_HALF, ffn=768), 300
CALLS = ("a3_rms_norm", "a3_selected_qkv_proj", "a3_paged_append", "a3_paged_attention", "a3_tree_attention", "a3_block_tail", "a3_lm_head",
         "a3_tree_accept", "a3_beam_select", "a3_paged_move")


@pytest.fixture
def ran(monkeypatch):
    names = []
    for name in CALLS:
        monkeypatch.setattr(api, name, lambda *a, name=name, **k: names.append(name))
    monkeypatch.setattr(api, "torch_stream", lambda stream: None)
    return names


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


class Step:
    """What a step takes, all of it fitting."""

    def __init__(self, n, **bufs):
        self.n = n
        self.layout = api.Layout.decode(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=512, rope_base=5e5, n_req=n, device="cpu", prepare=False)
        p = api.Pages(page_table=_i32(n, 4), rope_cs=torch.empty((50, 64, 2)), dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=32,
                      n_pages=8, rope_base=5e5, n_pos=50)
        self.pages = [p, p.sibling()]
        self.layers = [dict(g_in=None, wq=None, wk=None, wv=None, wo=None, g_post=None, w_gate=torch.zeros((SHAPE.ffn, 4)), w_up=None, w_down=None)] * 2
        self.resid, self.w = torch.zeros((n, 512), dtype=torch.bfloat16), torch.zeros((VOCAB, 512), dtype=torch.bfloat16)
        self.bufs = self.buffers(**bufs)

    def buffers(self, vocab=VOCAB, tree=(2, 3), n=None):
        layout = self.layout
        if n is not None:
            layout = api.Layout.decode(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=512, rope_base=5e5, n_req=n, device="cpu", prepare=False)
        return stack.DecodeBuffers(layout, SHAPE, SHAPE.ffn, self.pages, vocab, tree=tree)


def _verify(s, **over):
    a = dict(resid=s.resid, bufs=s.bufs, tree=stack.TreeRows([[-1, 0, 0], [-1, 0]], [5, 7], np.zeros(5), max_path=4, device="cpu"),
             out=api.TreeAccepted(2, 5, 4, VOCAB, device="cpu")) | over
    return stack.verify_stack(s.layout, SHAPE, s.layers, None, a["resid"], api.PageLayers(s.pages), a["tree"], a["bufs"], s.w, a["out"])


def _beam(s, **over):
    a = dict(resid=s.resid, bufs=s.bufs, slot=_i32(6), pos=_i32(6), length=_i32(6), score=torch.zeros(6), first=_i32(6), run=_i32(6), most=9, done=_i32(6),
             end=3, out=api.BeamChoice(2, 3, VOCAB, 3, device="cpu")) | over
    a["out"].row.zero_()
    return stack.beam_stack(s.layout, SHAPE, s.layers, None, a["resid"], api.PageLayers(s.pages), a["slot"], a["pos"], a["length"], a["bufs"], s.w,
                            a["score"], a["first"], a["run"], a["most"], a["out"], done=a["done"], end_token=a["end"])


def test_steps_that_fit(ran):
    _verify(Step(5))
    assert ran[0] == "a3_rms_norm" and ran[-2:] == ["a3_tree_accept", "a3_paged_move"] and ran.count("a3_tree_attention") == 2
    del ran[:]
    _beam(Step(6))
    assert ran[0] == "a3_rms_norm" and ran[-2:] == ["a3_beam_select", "a3_paged_move"]
    for over in (dict(done=None), dict(run=None), dict(out=api.BeamChoice(9, 3, VOCAB, 3, device="cpu"))):
        _beam(Step(6), **over)


@pytest.mark.parametrize("out", [(1, 5, VOCAB), (2, 4, VOCAB), (2, 5, 0), (2, 5, 1)])
def test_accepted_paths_of_other_sizes(ran, out):
    """Fewer trees, fewer rows, no vocabulary (hence no workspace), or the rows' workspace of a smaller vocabulary."""
    groups, rows, vocab = out
    accepted = api.TreeAccepted(groups, rows, 4, vocab, device="cpu")
    if vocab == 1:
        accepted.ws = accepted.ws[:16]
    if vocab == 0:
        accepted.ws = accepted.ws[:0]
    with pytest.raises(ValueError):
        _verify(Step(5), out=accepted)
    assert ran == []


@pytest.mark.parametrize("tree", [None, (1, 1)])
def test_buffers_for_smaller_trees(ran, tree):
    s = Step(5, tree=tree)
    if tree:
        assert s.bufs.ws_tree.numel() < api.a3_tree_attention_ws_bytes(s.pages[0], 2, 3)
    with pytest.raises(ValueError):
        _verify(s)
    assert ran == []


@pytest.mark.parametrize("what", ["rows", "type", "strided"])
def test_hidden_states_that_do_not_fit(ran, what):
    for step, n in ((_verify, 5), (_beam, 6)):
        x = dict(rows=torch.zeros((n - 1, 512), dtype=torch.bfloat16), type=torch.zeros((n, 512)), strided=torch.zeros((n, 1024), dtype=torch.bfloat16)[:, ::2])
        with pytest.raises(ValueError):
            step(Step(n), resid=x[what])
    assert ran == []


@pytest.mark.parametrize("over", [dict(score=torch.zeros(5)), dict(score=torch.zeros(6, dtype=torch.float64)), dict(score=torch.zeros(12)[::2]), dict(score=None),
                                  dict(done=_i32(5)), dict(done=torch.zeros(6, dtype=torch.bool)), dict(first=_i32(5)), dict(first=None), dict(run=_i32(5)),
                                  dict(run=torch.zeros(6, dtype=torch.int64)), dict(run=_i32(12)[::2]), dict(slot=_i32(5)), dict(pos=_i32(5)), dict(length=_i32(5)),
                                  dict(length=None), dict(most=-1), dict(end=-1), dict(out=(1, 3, VOCAB, 3)), dict(out=(2, 3, 1, 3))])
def test_beams_that_do_not_fit(ran, over):
    if "out" in over:
        choice = api.BeamChoice(*over["out"], device="cpu")
        if over["out"][2] == 1:
            choice.ws = choice.ws[:64]
        over = dict(out=choice)
    with pytest.raises(ValueError):
        _beam(Step(6), **over)
    assert ran == []


@pytest.mark.parametrize("what", ["width", "type", "strided", "flat"])
def test_vocabularies_that_do_not_fit(ran, what):
    for step, n in ((_verify, 5), (_beam, 6)):
        s = Step(n)
        s.w = dict(width=torch.zeros((VOCAB, 256), dtype=torch.bfloat16), type=s.w.float(), strided=torch.zeros((VOCAB, 1024), dtype=torch.bfloat16)[:, ::2],
                   flat=torch.zeros((VOCAB,), dtype=torch.bfloat16))[what]
        with pytest.raises(ValueError):
            step(s)
    assert ran == []


def test_more_beams_than_there_can_be(ran):
    out = api.BeamChoice(1, 65, VOCAB, 65, device="cpu")
    s = Step(65)
    with pytest.raises(ValueError):
        _beam(s, out=out, **{k: _i32(65) for k in ("slot", "pos", "length", "first", "run", "done")}, score=torch.zeros(65))
    assert ran == []


def test_buffers_of_a_smaller_block(ran):
    s = Step(6)
    s.bufs.ws_tail = s.bufs.ws_tail[:16]
    with pytest.raises(ValueError):
        _beam(s)
    s = Step(6)
    s.bufs.ws_attn = s.bufs.ws_attn[:16]
    with pytest.raises(ValueError):
        _beam(s)
    assert ran == []
