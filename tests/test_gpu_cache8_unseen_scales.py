"""Pages that a head does not attend to: whatever lies there, scales that are infinite or NaN among them, its output and log-sum-exp are the same bits."""
import math

import pytest
import torch

from paper_2507_17511_amd.attention import AttentionSession, PagedCache8
from test_gpu_cache8 import BF, DEV, HF, filled, gen, ints, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [math.inf, -math.inf, math.nan, 2.0 ** 127, 0.0])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 32), (128, 64), (256, 128), (256, 16)])
def test_lists_with_entries_outside(dtype, dim, page, scale):
    """An entry outside of the context is none: not the first page, nor the last one, which lie nearest to it."""
    hq, hk, held = 6, 2, 9
    cache = filled(71, held + 1, hk, page, dim)
    s, q = AttentionSession(hq, hk, dim, dtype=dtype), randn(gen(72), 3, hq, dim, dtype=dtype)
    table = ints([list(range(held))] * 3)
    lens = ints([held * page, held * page - 5, 3 * page])
    some = [[-1, 2, 4, -7, 10 ** 9, 1, held, -2 ** 31], [3, -1, -1, -1, 5, 10 ** 9, 2, 1], [1, 7, 1, -1, -3, 9, -1, -1]]
    lists = ints([[row] * hk for row in some])
    rows = q.shape[:2]
    got = []
    for odd in (False, True):
        c = PagedCache8(*[x.clone() for x in cache.written])
        if odd:
            unseen = [0, held - 1]          # of the first two contexts, whose pages the third one's are
            for x in (c.k_scale, c.v_scale):
                x[unseen] = scale
            for x in (c.k, c.v):
                x.view(torch.uint8)[unseen] = 0x7f
        out, lse = torch.full_like(q, 7.0), torch.full(rows, 7.0, device=DEV)
        s.paged8(c, q, table, lens, blocks=lists, out=out, lse=lse)
        torch.cuda.synchronize()
        got.append((out, lse))
    assert bool(got[0][0].isfinite().all()) and bool(got[0][1].isfinite().all())
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_pages_past_the_end_of_a_context_and_of_others(dtype, page):
    """Entries of the table behind a context's pages, other contexts' pages, other heads' scales."""
    hq, hk, dim = 4, 2, 128
    cache = filled(73, 12, hk, page, dim)
    s, q = AttentionSession(hq, hk, dim, dtype=dtype), randn(gen(74), 2, hq, dim, dtype=dtype)
    table, lens = ints([[0, 1, 2, 9, 9, 9], [3, 4, 5, 6, 10, 11]]), ints([2 * page + 1, 4 * page])
    plain = s.paged8(cache, q, table, lens)
    odd = PagedCache8(*[x.clone() for x in cache.written])
    for x in (odd.k_scale, odd.v_scale):
        x[7:] = math.nan
        x[1, 1] = math.inf                  # the first context's, of the second head of keys
    got = s.paged8(odd, q, table, lens)
    torch.cuda.synchronize()
    assert torch.equal(got[1], plain[1]) and torch.equal(got[0, :2], plain[0, :2]) and not bool(got[0, 2:].isfinite().any())
