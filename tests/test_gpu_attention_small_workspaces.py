"""Workspaces that hold two parts, where more would be made: coarser parts, the last of which takes the rest.  That both are there is seen in the workspace: it is NaN
before the call.  And parts that are listed though there are few of them, as contexts that may differ could fill 128 MB."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, expect_prompt, gen, randn, run_paged, starts

pytestmark = pytest.mark.gpu


def session(rows, hq, hk, dim, dtype):
    """With a workspace for two parts of `rows` rows of heads, and what shows which of them were written."""
    size = -(-(cf.CF_ATTN_COUNTER_BYTES + 2 * rows * (dim + 1) * 4) // 256) * 256
    s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=size)
    parts = s.workspace[cf.CF_ATTN_COUNTER_BYTES:][:2 * rows * dim * 4].view(torch.float32).view(2, rows, dim)
    s.workspace[cf.CF_ATTN_COUNTER_BYTES:].fill_(255)
    torch.cuda.synchronize()

    def written():
        torch.cuda.synchronize()
        assert not bool(s.workspace[:cf.CF_ATTN_COUNTER_BYTES].any())
        return [bool((~torch.isnan(p)).any()) for p in parts]
    return s, written


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens_q,lens_k,max_k", [([40], [5000], 0), ([3, 20], [3000, 700], 3000), ([33, 1, 50], [10, 1, 4100], 0), ([20], [4000], 1000)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt(dtype, dim, lens_q, lens_k, max_k, causal):
    hq, hk, tq, tk = 4, 2, sum(lens_q), sum(lens_k)
    g = gen(191)
    q, k, v = randn(g, tq, hq, dim, dtype=dtype), randn(g, tk, hk, dim, dtype=dtype), randn(g, tk, hk, dim, dtype=dtype)
    s, written = session(tq * hq, hq, hk, dim, dtype)
    lse = torch.empty(tq, hq, device=DEV)
    out = s.prompt(q, k, v, starts(lens_q), starts(lens_k), causal=causal, lse=lse, max_k=max_k)
    assert written() == [True, True]
    res, tol = expect_prompt(q, k, v, lens_q, lens_k, causal, 1 / math.sqrt(dim))
    check("out", out, res[0], tol[0])
    check("lse", lse, res[1], tol[1])
    assert torch.equal(out, s.prompt(q, k, v, starts(lens_q), starts(lens_k), causal=causal, max_k=max_k))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(8, 2), (17, 1)])
@pytest.mark.parametrize("lens,max_len", [([5000], 0), ([4097, 1, 600, 0], 4097), ([3000, 2500], 700), ([3500], 6000), ([0, 1, 8192, 70, 6000] + [33] * 200, 8192)])
def test_paged(dtype, dim, hq, hk, lens, max_len):
    """The last of them is listed: over 1024 workgroups with 205 sequences."""
    page, n = 32, len(lens)
    g = gen(192)
    pages, cols = 300, max(-(-max(lens) // page), -(-max_len // page))
    cache = PagedCache(randn(g, pages, hk, page, dim, dtype=dtype), randn(g, pages, hk, page, dim, dtype=dtype))
    table = torch.randint(0, pages, (n, cols), generator=g, device=DEV, dtype=torch.int32)
    ln = torch.tensor(lens, dtype=torch.int32, device=DEV)
    q = randn(g, n, hq, dim, dtype=dtype)
    s, written = session(n * hq, hq, hk, dim, dtype)
    lse = torch.empty(n, hq, device=DEV)
    out = s.paged(cache, q, table, ln, lse=lse, max_len=max_len)
    assert written() == [True, True]
    for b in [b for b in range(n) if b < 8 or b % 50 == 0]:
        used = table[b].long()
        k, v = (x[used].transpose(1, 2).reshape(-1, hk, dim)[:lens[b]] for x in (cache.k, cache.v))
        for h in range(hk):
            rows = slice(h * (hq // hk), (h + 1) * (hq // hk))
            o, l, to, tl = attend(q[b, rows], k[:, h], v[:, h], [lens[b]] * (hq // hk), 1 / math.sqrt(dim))
            check(f"out of {b}", out[b, rows], o, to)
            check(f"lse of {b}", lse[b, rows], l, tl)
    assert torch.equal(out, s.paged(cache, q, table, ln, max_len=max_len))


@pytest.mark.parametrize("dtype,dim,hq,hk,lens,max_len", [(BF, 128, 8, 4, [16384, 300, 1, 5000], 16384), (HF, 64, 24, 8, [40, 22000, 0], 22000), (BF, 256, 40, 2, [12000, 3, 8191], 12000)])
def test_few_listed_parts(dtype, dim, hq, hk, lens, max_len):
    """units x max_len x head_dim x 4 passes 2^27, and there are at most 1024 parts."""
    assert max(lens) == max_len
    units = len(lens) * hk * -(-(hq // hk) // 16)
    assert units * max_len * dim * 4 >= 1 << 27 and units * 32 <= 1024
    run_paged(193, dtype, hq, hk, dim, lens, 64, max_len=max_len)
