"""Limits of the rotary tables and the paged cache: the boundary of each, from both sides, before anything reaches a device."""
import torch

from paper_2512_12131_amd import binding as B


def test_a_workspace_query_takes_every_table_that_the_call_takes():
    """Of a table of one row the row stride says nothing: a column that is turned has any."""
    cache = torch.zeros((40, 16, 2, 128), dtype=torch.bfloat16)
    size = B.lr_attention_paged_workspace_bytes(cache, torch.zeros((1, 30), dtype=torch.int32), 1, 4)
    turned = torch.zeros((30, 1), dtype=torch.int32).t()
    assert turned.is_contiguous() and turned.stride(0) == 1
    assert size > 0 and B.lr_attention_paged_workspace_bytes(cache, turned, 1, 4) == size
