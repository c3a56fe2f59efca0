"""fp16 keys that weigh little each and much together, behind a first key that leads by `ahead` and whose value is nearly zero: what most models'
first token is to the rest.  Their weights, relative to the largest, are below what fp16 holds in full (2^-14) or at all (2^-25).

Tolerances.  u = 2^-11.  A weight is rounded by a relative u, or below 2^-14 by 2^-25 as it is stored: relative to 2^-6 of the largest of its 64 keys (a tile) that were
there first, or so that they sum up to 2^-11 at least.  So the 64 keys that the leading one shares a tile with are off by 64 2^-25 / 2^6 = 2^-25 max|v| at most.  Other
keys' weights, which differ from one another here, are rounded up as often as down: 2^-15 of their share of the weights times max|v| are 2^-7 of what 64 weights of 2^-17 could
be off by all one way, a tile's average over some hundred tiles and more, and 2^-5 for a handful, where attention_reference's relative roundings, 2^-11 each, cover
them.  That is 2^-9 of what the lost weights summed up to."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from attention_reference import U, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, gen, randn, starts

pytestmark = pytest.mark.gpu


def inputs(dim, hq, hk, tq, tk, ahead, dtype, at=0, size=1.0):
    """The key `at` has a score `ahead` (natural) above the others', which are within 1 or so of one another; every value but its own is near 1."""
    g = gen(121)
    q, k = randn(g, tq, hq, dim, dtype=dtype) * 0.2, randn(g, tk, hk, dim, dtype=dtype) * 0.5
    q[..., 0], k[..., 0] = 4.0, 0.0
    k[at, :, 0] = ahead * math.sqrt(dim) / 4.0
    v = (1.0 + 0.1 * torch.randn(tk, hk, dim, generator=g, device=DEV)) * size
    v[at] = 2.0 ** -20
    return q, k, v.to(dtype)


def expect(q, k, v, seen, at):
    """q [R, D], k and v [K, D] -> outputs, log-sum-exps and their tolerances, in 64 bits."""
    dt, dim = q.dtype, q.shape[1]
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    s = q @ k.t() / math.sqrt(dim)
    s[torch.arange(k.shape[0])[None] >= torch.tensor(seen)[:, None]] = -math.inf
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    out, spread = p @ v, p @ v.abs()
    rest = 1.0 - p[:, at] if 0 <= at < k.shape[0] else torch.ones(len(seen), dtype=torch.float64)
    off = (2.0 ** -23 * dim / math.sqrt(dim) * (q.abs() @ k.abs().t())).amax(1)
    largest = v.abs().max()
    tol = 1.05 * (U[dt] * (spread + out.abs()) + (2 * off[:, None] + 2.0 ** -20) * spread)
    if dt == HF:
        tol = tol + (1.05 * (2.0 ** -25 + 2.0 ** -15 * rest) * largest)[:, None] + 2.0 ** -25        # an output below 2^-14 is rounded by 2^-25
    return out, lse, tol, 1.05 * off + 2.0 ** -20 * (1 + lse.abs())


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,ahead", [(HF, 8.0), (HF, 14.0), (HF, 17.5), (HF, 21.0), (BF, 17.5)])
@pytest.mark.parametrize("hq,hk,tq,tk,causal,workspace", [(2, 1, 150, 4096, False, 0), (4, 2, 700, 700, True, 0), (1, 1, 9, 30000, True, cf.CF_ATTN_WORKSPACE_BYTES), (1, 1, 33, 16384, False, 0)])
def test_prompt(dim, dtype, ahead, hq, hk, tq, tk, causal, workspace):
    q, k, v = inputs(dim, hq, hk, tq, tk, ahead, dtype, size=64.0)
    lse = torch.empty(tq, hq, device=DEV)
    out = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace).prompt(q, k, v, starts([tq]), starts([tk]), causal=causal, lse=lse)
    seen = [i + 1 + tk - tq if causal else tk for i in range(tq)]
    for h in range(hq):
        o, l, to, tl = expect(q[:, h], k[:, h // (hq // hk)], v[:, h // (hq // hk)], seen, 0)
        check("out", out[:, h], o, to)
        check("lse", lse[:, h], l, tl)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("at", [1000, 1999])
def test_prompt_the_leading_key_comes_later(dim, at):
    """The maximum rises by 25 powers of two in the middle, or at the end."""
    q, k, v = inputs(dim, 2, 1, 40, 2000, 17.5, HF, at=at, size=64.0)
    out = AttentionSession(2, 1, dim, dtype=HF, workspace_bytes=0).prompt(q, k, v, starts([40]), starts([2000]), causal=False)
    for h in range(2):
        o, _, to, _ = expect(q[:, h], k[:, 0], v[:, 0], [2000] * 40, at)
        check("out", out[:, h], o, to)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompt_leads_come_and_go(dim):
    """Keys 17.5 ahead every 500 keys, with values near zero."""
    q, k, v = inputs(dim, 2, 1, 40, 3000, 17.5, HF, size=64.0)
    k[::500], v[::500] = k[:1].clone(), 2.0 ** -20
    out = AttentionSession(2, 1, dim, dtype=HF, workspace_bytes=0).prompt(q, k, v, starts([40]), starts([3000]), causal=False)
    for h in range(2):
        o, _, to, _ = expect(q[:, h], k[:, 0], v[:, 0], [3000] * 40, -1)
        p = torch.softmax(q[:, h].double().cpu() @ k[:, 0].double().cpu().t() / math.sqrt(dim), 1)
        rest = 1.0 - p[:, ::500].sum(1)
        to = to - (1.05 * 2.0 ** -15 * (1.0 - rest) * v.double().abs().max().cpu())[:, None]        # of `rest` alone
        check("out", out[:, h], o, to)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype,ahead", [(HF, 8.0), (HF, 14.0), (HF, 17.5), (HF, 21.0), (BF, 17.5)])
@pytest.mark.parametrize("seqs,n,hq,workspace", [(2, 4096, 4, 0), (1, 30000, 4, cf.CF_ATTN_WORKSPACE_BYTES), (90, 3000, 20, cf.CF_ATTN_WORKSPACE_BYTES)])
def test_paged(dim, dtype, ahead, seqs, n, hq, workspace):
    """All sequences on the same pages, with lengths of their own."""
    page, hk = 16, 1
    pages = -(-n // page)
    q, k, v = inputs(dim, hq, hk, seqs, pages * page, ahead, dtype, size=64.0)
    cache = PagedCache(*(x.view(pages, page, hk, dim).transpose(1, 2).contiguous() for x in (k, v)))
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(seqs, 1)
    lens = [n - 7 * b for b in range(seqs)]
    lse = torch.empty(seqs, hq, device=DEV)
    out = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace).paged(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), lse=lse)
    for h in range(hq):
        o, l, to, tl = expect(q[:, h], k[:n, 0], v[:n, 0], lens, 0)
        check("out", out[:, h], o, to)
        check("lse", lse[:, h], l, tl)
