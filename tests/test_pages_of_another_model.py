"""Pages whose type, heads, rotation or scale are not the layout's are refused before anything runs (no GPU needed: nothing does)."""
import numpy as np
import pytest
import torch

import a3_synth as synth
from paper_2511_17560_amd import api, stack

SHAPE = synth.ModelShape("fit", "bf16", 512, 8, 2, 128, 5e5, synth.ROPE_HALF, ffn=768)


def _pages(n_pos=50, own_rope=True, **over):
    kw = dict(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=32, n_pages=8, rope_base=5e5, rope_layout=1, sm_scale=0.0) | over
    p = api.Pages(page_table=torch.zeros((2, 4), dtype=torch.int32), n_pos=n_pos, rope_cs=torch.empty((n_pos, kw["head_dim"] // 2, 2)), **kw)
    p.own_rope = own_rope
    return [p, p.sibling()]


def _layout(**kw):
    w = synth.custom(SHAPE, [[20], [30]], [4, 4], seed=1)
    return w, api.Layout.from_workload(w, device="cpu", prepare=False, **kw)


def _calls(layout, w, pages):
    """Every call that takes pages of a prompt; without a GPU the first kernel call raises something else than ValueError."""
    layers = [dict(w_gate=torch.zeros((SHAPE.ffn, SHAPE.hidden)), g_in=None)] * 2
    x = torch.zeros((w.total_tokens, SHAPE.hidden), dtype=torch.bfloat16)
    yield lambda: stack.prefill_stack(layout, SHAPE, layers, None, x, pages=pages)
    yield lambda: stack.fuse_stack(layout, SHAPE, layers, None, x, [], [], np.zeros(3, dtype=np.int32), np.arange(8), pages=pages)


@pytest.mark.parametrize("over", [dict(rope_layout=0), dict(rope_base=1e4), dict(sm_scale=0.1), dict(dtype="f32"), dict(n_q_heads=16), dict(n_kv_heads=4),
                                  dict(head_dim=64), dict(rope_layout=0, own_rope=False)])
def test_a_prompts_pages(over):
    w, layout = _layout()
    for call in _calls(layout, w, _pages(**over)):
        with pytest.raises(ValueError, match="pages: their"):
            call()


def test_one_layer_of_another_model():
    w, layout = _layout()
    for call in _calls(layout, w, [_pages()[0], _pages(rope_layout=0)[0]]):
        with pytest.raises(ValueError, match="rope_layout"):
            call()


@pytest.mark.parametrize("over,layout_kw", [(dict(), {}), (dict(sm_scale=128 ** -0.5), {}), (dict(), dict(sm_scale=128 ** -0.5)),
                                            (dict(sm_scale=0.3), dict(sm_scale=0.3)), (dict(rope_base=1e4, own_rope=False), {}),
                                            (dict(n_pos=0, rope_layout=0, rope_base=1e4), {})])
def test_pages_that_are_taken(over, layout_kw):
    """The layout's numbers however they are said; a table of the caller's own goes by what is in it; pages that turn nothing have no rotation."""
    w, layout = _layout(**layout_kw)
    stack._fit(_pages(**over), 2, 2, layout.max_len, layout, prompt=True)


@pytest.mark.parametrize("over,taken", [(dict(), True), (dict(rope_layout=0, rope_base=1e4, sm_scale=0.2), True), (dict(dtype="f32"), False),
                                        (dict(n_q_heads=4), False), (dict(n_kv_heads=8), False), (dict(head_dim=64), False)])
def test_a_steps_pages(over, taken):
    """A decoding step's layout has no rotation and no scale: those are the pages' alone."""
    layout = api.Layout.decode(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=512, rope_base=5e5, n_req=2, device="cpu", prepare=False)
    bufs = object.__new__(stack.DecodeBuffers)
    bufs.x, bufs.logits = torch.zeros((2, 512), dtype=torch.bfloat16), None
    i32 = torch.zeros(2, dtype=torch.int32)
    call = lambda: stack.decode_stack(layout, SHAPE, [dict(g_in=None)] * 2, None, bufs.x, _pages(**over), i32, i32, i32, bufs)
    if taken:
        stack._fit(_pages(**over), 2, 2, 0, layout, prompt=False)
    else:
        with pytest.raises(ValueError, match="pages: their"):
            call()


def test_siblings_keep_whose_table_it_is():
    assert [p.own_rope for p in _pages()] == [True, True] and [p.own_rope for p in _pages(own_rope=False)] == [False, False]
