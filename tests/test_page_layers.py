"""Layers whose pages are laid out in different ways are refused when they are put together, not by a step's last call (no GPU needed)."""
import pytest
import torch

from paper_2511_17560_amd import api


@pytest.mark.parametrize("over", [dict(dtype="f32"), dict(q8=True), dict(n_q_heads=4), dict(n_kv_heads=4), dict(head_dim=64), dict(page_size=64), dict(n_pages=9)])
def test_layers_that_are_not_laid_out_alike(over):
    kw = dict(page_table=torch.zeros((2, 4), dtype=torch.int32), dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=32, n_pages=8, rope_base=5e5, n_pos=50)
    make = lambda **kw: api.Pages(rope_cs=torch.empty((50, kw["head_dim"] // 2, 2)), **kw)
    first = make(**kw)
    api.PageLayers([first, first.sibling()])
    with pytest.raises(ValueError, match="layer 1"):
        api.PageLayers([first, make(**(kw | over))])
