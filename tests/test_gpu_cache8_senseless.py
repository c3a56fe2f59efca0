"""Numbers on the device that cannot be refused: page numbers and lengths outside of the cache, scales that are no powers of two; and plans for the cache in 16 bits."""
import math

import pytest
import torch

import cache8_reference as ref
from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache, PagedCache8, PageTables
from test_gpu_cache8 import BF, DEV, HF, filled, gen, ints, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,dim,dtype", [(16, 64, BF), (32, 256, HF), (64, 128, BF), (128, 128, HF)])
def test_pages_and_lengths_outside_are_taken_as_the_nearest(page, dim, dtype):
    pages, cols, hq, hk = 9, 6, 4, 2
    cache = filled(101, pages, hk, page, dim, True)
    rows = [[3, -1, 10 ** 9, 8, 0, -2 ** 31], [2 ** 31 - 1, 1, 2, 3, 4, 5], [1, 2, 3, 4, 5, 6], [7, 7, 7, 0, 0, 0], [9, 9, 9, 9, 9, 9]]
    lens = [6 * page, 2 * page + 3, 10 ** 9, -7, 2 ** 31 - 1]
    near = [[min(max(p, 0), pages - 1) for p in row] for row in rows]
    within = [min(max(n, 0), cols * page) for n in lens]
    q = randn(gen(102), 5, hq, dim, dtype=dtype)
    for bytes_ in (64 << 20, 0):
        s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=bytes_)
        for longest in (0, 5, 2 ** 40):
            out, lse = torch.empty_like(q), torch.empty(5, hq, device=DEV)
            s.paged8(cache, q, ints(rows), ints(lens), out=out, lse=lse, max_len=longest)
            torch.cuda.synchronize()
            k, v = ref.Cache(cache.k, cache.k_scale), ref.Cache(cache.v, cache.v_scale)
            o, l, to, tl = ref.attention(q, k, v, near, within, 1 / math.sqrt(dim))
            check("out", out, o, to)
            check("lse", lse, l, tl)
    s = AttentionSession(hq, hk, dim, dtype=dtype)
    assert s.select(cache, q, ints(rows), ints(lens), 3, first=0, recent=0).tolist() == ref.select(q, cache.bounds, near, within, page, 3, 0, 0)
    lists = torch.tensor([[[0, 5, -1]] * hk] * 5, dtype=torch.int32, device=DEV)
    lists[1, :, 1], lists[2, 0] = 2 ** 31 - 1, torch.tensor([-2 ** 31, 5, 4], dtype=torch.int32)
    out = s.paged8(cache, q, ints(rows), ints(lens), blocks=lists)
    torch.cuda.synchronize()
    o, _, to, _ = ref.attention(q, k, v, near, within, 1 / math.sqrt(dim), lists.tolist())
    check("listed", out, o, to)


def test_of_other_scales_the_exponent_counts():
    """3 is taken as 2, -0.6 as 0.5; an append on a page with one lets it grow, or keeps its exponent within the range."""
    cache = filled(103, 3, 1, 16, 64, True, spread=0.0)
    plain = PagedCache8(*[x.clone() for x in cache.written])
    cache.k_scale[:, 0], plain.k_scale[:, 0] = torch.tensor([3.0, -0.6, 1.99], device=DEV), torch.tensor([2.0, 0.5, 1.0], device=DEV)
    cache.v_scale[:, 0], plain.v_scale[:, 0] = torch.tensor([1.5, 5.0, 0.26], device=DEV), torch.tensor([1.0, 4.0, 0.25], device=DEV)
    s, q, x = AttentionSession(1, 1, 64), randn(gen(104), 1, 1, 64), randn(gen(105), 1, 1, 64, scale=3000.0)
    a, b = (s.paged8(c, q, ints([[0, 1, 2]]), ints([48])) for c in (cache, plain))
    assert torch.equal(a, b)
    for c in (cache, plain):
        s.append8(c, x, x, ints([16 + 5], torch.int64))
    torch.cuda.synchronize()
    assert torch.equal(cache.k.view(torch.uint8), plain.k.view(torch.uint8)) and torch.equal(cache.k_scale[1], plain.k_scale[1]) and torch.equal(cache.bounds, plain.bounds)
    for odd, least in ((0.0, -100), (2.0 ** -140, -100), (math.inf, 119), (math.nan, 119), (2.0 ** 125, 119)):
        cache.k_scale[1, 0] = odd
        s.append8(cache, x * 0, x * 0, ints([16 + 7], torch.int64))
        torch.cuda.synchronize()
        assert cache.k_scale[1, 0].item() == 2.0 ** least
    assert not bool(cache.k[1, 0, 7].float().any())


def test_plans_for_the_cache_in_16_bits():
    """Slots, positions, tables and starts of a plan are what append, prompt and paged take."""
    g, page, hq, hk, dim = gen(106), 256, 4, 2, 64
    tables, cache = PageTables.empty(3, 4, 9, page), PagedCache.empty(9, hk, dim, page)
    s, keys = AttentionSession(hq, hk, dim), [[], [], []]
    for news in ([300, 1, 700], [1, 1, 1], [5, 0, 200]):
        rows = sum(news) + 3
        plan = s.plan(tables, ints(news), rows)
        q, k, v = randn(g, rows, hq, dim), randn(g, rows, hk, dim), randn(g, rows, hk, dim)
        s.append(cache, k, v, plan.slots)
        at = plan.cu.tolist()
        for b in range(3):
            keys[b] += [(k[t], v[t]) for t in range(at[b], at[b + 1])]
        if news[0] == 300:
            out = s.prompt(q, k, v, plan.cu)
            for b in range(3):
                span = slice(at[b], at[b + 1])
                o, _, to, _ = attend(q[span, 1], k[span, 0], v[span, 0], list(range(1, news[b] + 1)), 1 / 8)
                check("prompt", out[span, 1], o, to)
        one = randn(g, 3, hq, dim)
        out = s.paged(cache, one, tables.table, tables.lens)
        torch.cuda.synchronize()
        assert tables.lens.tolist() == [len(x) for x in keys] and plan.refused.item() == 0
        for b in range(3):
            for h in range(hq):
                kk, vv = (torch.stack([x[i][h // 2] for x in keys[b]]) for i in (0, 1))
                o, _, to, _ = attend(one[b, h:h + 1], kk, vv, [len(kk)], 1 / 8)
                check("paged", out[b, h:h + 1], o, to)
