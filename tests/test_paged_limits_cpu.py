"""Limits of the rotary tables and the paged cache: the boundary of each, from both sides, before anything reaches a device."""
import torch

from paper_2512_12131_amd import binding as B
from test_paged_cpu import EINVAL, EUNSUPPORTED, _append, _cache, _paged


def test_a_workspace_query_takes_every_table_that_the_call_takes():
    """Of a table of one row the row stride says nothing: a column that is turned has any."""
    cache = torch.zeros((40, 16, 2, 128), dtype=torch.bfloat16)
    size = B.lr_attention_paged_workspace_bytes(cache, torch.zeros((1, 30), dtype=torch.int32), 1, 4)
    turned = torch.zeros((30, 1), dtype=torch.int32).t()
    assert turned.is_contiguous() and turned.stride(0) == 1
    assert size > 0 and B.lr_attention_paged_workspace_bytes(cache, turned, 1, 4) == size


def test_keys_of_a_sequence():
    """Up to 2^31 - 2048: tiles and the windows of page numbers that are looked up ahead are counted in 31 bits."""
    cache = lambda keys: _cache(page_size=8, max_pages=keys // 8, table_ld=keys // 8, page_stride=8 * 256, n_pages=1, batch=1)
    most = (1 << 31) - 2048
    query = lambda keys: B.lib().lr_attention_paged_workspace_bytes(cache(keys), 4, 4)
    assert query(most) > 0 and _paged(cache(most), T=0) == 0 and _append(cache(most), T=0) == 0
    for keys in (most + 8, (1 << 31) - 64, (1 << 31) - 8):
        assert query(keys) == 0 and _paged(cache(keys), T=0) == EUNSUPPORTED and _append(cache(keys), T=0) == EUNSUPPORTED, keys


def test_a_batch_of_no_sequences_needs_no_lists():
    """Empty tensors have null pointers; the one boundary of cu_q is there."""
    none = lambda **over: _cache(batch=0, page_table=None, kv_len=None, **over)
    assert _append(none()) == 0 and _paged(none()) == 0
    assert _append(none(k=None)) == EINVAL and _paged(none(cu_q=None)) == EINVAL
    assert _append(_cache(page_table=None)) == EINVAL and _paged(_cache(kv_len=None)) == EINVAL
