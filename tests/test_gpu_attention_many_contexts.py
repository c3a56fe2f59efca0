"""More contexts than a workgroup lists, one of them long: they are split as fewer are, and all of them come out right."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim,hq,hk", [(BF, 128, 2, 1), (HF, 64, 3, 3), (BF, 256, 4, 2)])
@pytest.mark.parametrize("n", [2048, 2049, 4500])
def test_one_long_context_among_many(dtype, dim, hq, hk, n):
    g = gen(151)
    page, pages = 64, 400
    cache = PagedCache(randn(g, pages, hk, page, dim, dtype=dtype), randn(g, pages, hk, page, dim, dtype=dtype))
    table = torch.stack([torch.randperm(pages, generator=g, device=DEV)[:260] for _ in range(8)]).repeat(n // 8 + 1, 1)[:n].to(torch.int32).contiguous()
    lens = torch.randint(0, 40, (n,), generator=g, device=DEV, dtype=torch.int32)
    long = [0, 5, 1024, 2047, n - 1]
    for i, b in enumerate(long):
        lens[b] = 16600 - 3000 * i
    q = randn(g, n, hq, dim, dtype=dtype)
    s = AttentionSession(hq, hk, dim, dtype=dtype)
    parts = s.workspace[cf.CF_ATTN_COUNTER_BYTES:]
    parts.fill_(255)                    # NaN
    out, lse = torch.full(q.shape, 7.0, dtype=dtype, device=DEV), torch.full(q.shape[:2], 7.0, device=DEV)
    s.paged(cache, q, table, lens, out=out, lse=lse, max_len=16384)
    whole = out.clone()
    s.paged(cache, q, table, lens, out=out, lse=lse)
    rows = -(-n // -(-n // 2048)) * hq
    assert bool((parts[:4 * rows * dim] != 255).any()) and not bool(s.workspace[:cf.CF_ATTN_COUNTER_BYTES].any())
    assert torch.equal(out, s.paged(cache, q, table, lens))
    others = [b for b in range(n) if b not in long]
    assert torch.equal(whole[others], out[others])
    for b in long + list(range(6, n, 97)):
        used, length = table[b].long(), int(lens[b])
        k, v = (x[used].transpose(1, 2).reshape(-1, hk, dim)[:length] for x in (cache.k, cache.v))
        for h in range(hk):
            heads = slice(h * (hq // hk), (h + 1) * (hq // hk))
            o, l, to, tl = attend(q[b, heads], k[:, h], v[:, h], [length] * (hq // hk), 1 / math.sqrt(dim))
            check(f"out of {b}", out[b, heads], o, to)
            check(f"lse of {b}", lse[b, heads], l, tl)
