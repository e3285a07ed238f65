"""Limits of the rotary tables and the paged cache: the boundary of each, from both sides, before anything reaches a device."""
import pytest
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


def test_angles_of_the_tables():
    """Up to 2^31, whatever the base and the scaling make of the positions.  Accepted calls get as far as the missing output."""
    def f(*, n=4, rot=8, first=0, base=1e4, factor=1.0, context=0.0, low=1.0, high=32.0):
        return B.lib().lr_rope_table(None, None, n, rot, first, base, factor, context, low, high, 1.0, None)
    far = 1 << 31
    # frequencies 1, 1000^(1/4) .. 1000^(3/4) = 177.8; 1e4^(-3/4) = 0.001 of which is divided by the factor
    for args in ({}, dict(first=far - 4), dict(first=far - 4, factor=32.0), dict(base=1e-3, first=int(far / 1000 ** 0.75) - 1000), dict(factor=0.5, first=far // 2 - 3),
                 dict(factor=1e-6, context=4096.0, n=1000), dict(factor=1e-9, n=1), dict(rot=8192, base=0.5, first=far // 2 - 4), dict(base=1e300)):
        assert f(**args) == EINVAL, args
    for args in (dict(base=1e-3, first=int(far / 1000 ** 0.75) + 1000), dict(factor=0.5, first=far // 2), dict(factor=1e-6, context=4096.0, first=far // 100),
                 dict(factor=1e-9), dict(factor=1e-300), dict(rot=8192, base=0.5, first=far // 2 + far // 1000), dict(base=1e-300)):
        assert f(**args) == EUNSUPPORTED, args
    assert f(n=0, factor=1e-300) == 0


def test_scales_of_the_attention():
    """The exponent's factor, scale * log2(e), is finite in 32 bits."""
    for scale in (2.4e38, 3.4e38):
        assert _paged(scale=scale, T=0) == EINVAL, scale
    for scale in (2.3e38, 1.0, 1e-37):
        assert _paged(scale=scale, T=0) == 0, scale


def test_caches_of_one_page_or_head():
    """Strides of dimensions of one say nothing: turned ones have any, and keys and values need not have the same."""
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    page = bf(16, 2, 128, 1).permute(3, 0, 1, 2)                   # [1, 16, 2, 128]
    head = bf(6, 16, 128, 1).permute(0, 1, 3, 2)                   # [6, 16, 1, 128]
    other = bf(6, 1, 16, 128).transpose(1, 2)
    assert page.is_contiguous() and page.stride(0) == 1 and head.stride(2) == 1 and other.stride(2) == 2048 and head.shape == other.shape
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    for k, v in ((page, page), (page, bf(1, 16, 2, 128)), (head, head), (head, other), (other, head)):
        heads = k.shape[2]
        assert B.lr_attention_paged_workspace_bytes(k, i32(1, 30), 1, 4) > 0
        with pytest.raises(B.LrError, match="current GPU"):        # as far as a CPU tensor gets
            B.lr_attention_paged_fwd(bf(1, 512), k, v, i32(1, 30), i32(2), i32(1), 4)
        with pytest.raises(B.LrError, match="current GPU"):
            B.lr_kv_append(bf(1, heads * 128), bf(1, heads * 128), k, v, i32(1, 30), i32(2), i32(1))
