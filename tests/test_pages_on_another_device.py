"""A position table is filled only where the kernel can write it (no GPU needed: CPU tensors never reach the library)."""
import pytest
import torch

from paper_2511_17560_amd import api

KW = dict(dtype="bf16", n_q_heads=8, n_kv_heads=2, head_dim=128, page_size=32, n_pages=8, rope_base=5e5, n_pos=50)


def test_pages_made_on_the_cpu_are_refused():
    with pytest.raises(ValueError, match="cpu"):
        api.Pages(page_table=torch.zeros((2, 4), dtype=torch.int32), stream=0, **KW)


def test_a_table_on_the_cpu_is_not_filled():
    table = torch.full((50, 64, 2), 7.0)
    p = api.Pages(page_table=torch.zeros((2, 4), dtype=torch.int32), rope_cs=table, **KW)
    with pytest.raises(ValueError, match="cpu"):
        api.a3_pages_prepare(p, stream=0)
    assert bool((table == 7.0).all())
