"""One new token over a paged cache where the parts of many contexts are listed, where there are more contexts than are split, and where the
last key's value is infinite; what the calls leave in the workspace."""
import math

import pytest
import torch

from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, gen, randn, run_paged

pytestmark = pytest.mark.gpu


def ragged(n, seed, edges):
    """`n` lengths: none, one, and the given ones among short ones."""
    short = torch.randint(0, 90, (n,), generator=torch.Generator().manual_seed(seed)).tolist()
    short[:2] = 0, 1
    for i, x in enumerate(edges):
        short[3 + i * (n // len(edges))] = x
    return short


@pytest.mark.parametrize("dtype,dim,hq,hk,n", [(BF, 64, 4, 4, 90), (HF, 128, 20, 4, 90), (BF, 256, 34, 2, 90), (HF, 64, 3, 1, 400), (BF, 128, 4, 1, 400)])
def test_parts_of_many_contexts(dtype, dim, hq, hk, n):
    edges = [8192, 2048, 2049, 4096, 127, 6000]
    run_paged(61, dtype, hq, hk, dim, ragged(n, 1, edges), 64, max_len=8192)


def test_more_contexts_than_are_split():
    lens = [0, 1, 33] * 700 + [700]
    run_paged(62, BF, 2, 1, 64, lens, 16, max_len=100000)


def test_the_workspace_is_left_as_it_was_found():
    g = gen(63)
    hq, hk, d, page = 8, 2, 128, 64
    s = AttentionSession(hq, hk, d)
    cache = PagedCache(randn(g, 300, hk, page, d), randn(g, 300, hk, page, d))
    kept = {}
    for again in range(3):
        for n, longest in ((1, 901), (3, 4000), (160, 16384), (7, 130), (40, 1000)):
            table = torch.randint(0, 300, (n, longest // page + 1), generator=torch.Generator(device=DEV).manual_seed(n), device=DEV, dtype=torch.int32)
            lens = torch.full((n,), longest, dtype=torch.int32, device=DEV)
            lens[n // 2] = 1
            q = randn(gen(n), n, hq, d)
            out = s.paged(cache, q, table, lens, max_len=longest)
            counters = s.workspace[:256 * 1024]
            assert not bool(counters.any()), (n, longest)
            assert torch.equal(out, kept.setdefault((n, longest), out))


@pytest.mark.parametrize("bad", [math.inf, -math.inf])
@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128), (BF, 256)])
@pytest.mark.parametrize("n", [1, 2, 15, 17, 33, 40, 300, 1025, 3001])
def test_an_infinite_value_of_the_last_key(bad, dtype, dim, n):
    """Its weight is positive: the outputs are infinite where it is, and finite elsewhere, whatever is read in place of keys past it."""
    g = gen(64)
    hq, hk, page = 4, 2, 16
    pages = -(-n // page)
    cache = PagedCache(randn(g, pages, hk, page, dim, dtype=dtype), randn(g, pages, hk, page, dim, dtype=dtype))
    cache.v[-1, :, (n - 1) % page, ::3] = bad
    q = randn(g, 1, hq, dim, dtype=dtype) * 0.25
    out = AttentionSession(hq, hk, dim, dtype=dtype).paged(cache, q, torch.arange(pages, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV))
    assert bool((out[..., ::3] == bad).all())
    k, v = (x.transpose(1, 2).reshape(-1, hk, dim)[:n] for x in (cache.k, cache.v))
    finite = torch.arange(dim) % 3 != 0
    for h in range(hq):
        o, _, to, _ = attend(q[:, h], k[:, h // 2], torch.where(torch.isinf(v), torch.zeros_like(v), v)[:, h // 2], [n], 1 / math.sqrt(dim))
        check("out", out[:, h, finite], o[:, finite], to[:, finite])
