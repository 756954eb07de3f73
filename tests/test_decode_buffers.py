"""A decoding step whose buffers do not hold its logits is refused before the cache and the residual stream are written (no GPU
needed: nothing runs)."""
import pytest
import torch

import a3_synth as synth
from paper_2511_17560_amd import api, stack

SHAPE = synth.ModelShape("buffers", "bf16", 512, 8, 2, 128, 5e5, synth.ROPE_HALF, ffn=768)


@pytest.mark.parametrize("logits,vocab", [((2, 300), 299), ((2, 300), 301), (None, 300), ((1, 300), 300)])
def test_logits_of_another_vocabulary(logits, vocab):
    layout = api.Layout.decode(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, hidden=512, rope_base=5e5, n_req=2, device="cpu", prepare=False)
    pages = [api.Pages(page_table=torch.zeros((2, 4), dtype=torch.int32), rope_cs=torch.empty((50, 64, 2)), dtype="bf16", n_q_heads=8, n_kv_heads=2,
                       head_dim=128, page_size=32, n_pages=8, rope_base=5e5, n_pos=50)] * 2
    bufs = object.__new__(stack.DecodeBuffers)
    bufs.x, bufs.logits = torch.zeros((len(torch.empty(logits)) if logits else 2, 512), dtype=torch.bfloat16), torch.empty(logits) if logits else None
    i32, w = torch.zeros(2, dtype=torch.int32), torch.zeros((vocab, 512), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="buffers of"):
        stack.decode_stack(layout, SHAPE, [dict(g_in=None)] * 2, None, bufs.x, pages, i32, i32, i32, bufs, w_vocab=w)
