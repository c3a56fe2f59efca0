"""Tensors whose rows or pages lie on one another (expanded ones): a distance of 0 is the library's word for dense, so they are refused before
it would read past them.  And a scale that is
too large.  Needs no GPU."""
import ctypes
import types

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession, PagedCache


def test_pages_on_one_another_are_no_cache():
    page = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        PagedCache(page.expand(8, -1, -1, -1), torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16).expand(8, -1, -1, -1))
    near = torch.zeros(4096, dtype=torch.bfloat16).as_strided((3, 2, 16, 64), (1024, 1024, 64, 1))
    with pytest.raises(ValueError):
        PagedCache(near, near.clone().as_strided((3, 2, 16, 64), (1024, 1024, 64, 1)))
    PagedCache(page, page.clone())


def test_a_table_whose_rows_lie_on_one_another():
    s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0, stream=types.SimpleNamespace(cuda_stream=0))
    cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    q, lens = torch.zeros(5, 4, 64, dtype=torch.bfloat16), torch.ones(5, dtype=torch.int32)
    one = torch.zeros(1, 3, dtype=torch.int32)
    for table in (one.expand(5, 3), torch.zeros(7, dtype=torch.int32).as_strided((5, 3), (1, 1))):
        with pytest.raises(ValueError, match="table"):
            s.paged(cache, q, table, lens, out=torch.zeros_like(q))


def test_a_scale_that_is_infinite_times_log2_e():
    p = (ctypes.c_void_p * 1)(1 << 20)
    args = cf.cf_join(1, cf.CF_F32, 0, p, p, cf.cf_rows(2 << 20, 512, 128), None)          # no tokens: nothing to do
    cf.cf_attn_join(cf.cf_attn_desc(cf.CF_BF16, 4, 2, 128, 1.9e38), args)
    with pytest.raises(cf.CFError) as e:
        cf.cf_attn_join(cf.cf_attn_desc(cf.CF_BF16, 4, 2, 128, 3.0e38), args)
    assert e.value.status == cf.CF_ERR_INVALID_ARG
