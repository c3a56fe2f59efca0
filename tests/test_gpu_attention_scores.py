"""Scores so large that the step between neighbouring fp32 numbers there is larger than 1: the row's output is the value of its largest score.

A score of D products in fp32 is off by at most D 2^-23 sum|q k| scale.  Where the largest is ahead of the next by twice that and
200 more, every other weight is below e^-200, which fp32 does not hold, and the output is that key's value: its weight is rounded once to 16 bits and
the output once, u each.  Rows with a closer race give something between the smallest and the largest value, but for the rounding."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from attention_reference import U
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, gen, randn, starts

pytestmark = pytest.mark.gpu

SIZES = [(BF, 2.0 ** 9, 1.0), (BF, 2.0 ** 12, 1.0), (BF, 2.0 ** 14, 1.0), (BF, 2.0 ** 15, 1.0), (BF, 2.0 ** 17, 1.0), (BF, 2.0 ** 30, 1.0), (BF, 2.0 ** 55, 1.0),
         (HF, 2.0 ** 11, 1.0), (HF, 2.0 ** 11, 1000.0), (HF, 2.0 ** 8, 1e30)]


def inputs(seed, dtype, size, below, tq, tk, hq, hk, dim):
    g = gen(seed)
    q, k, v = randn(g, tq, hq, dim, dtype=dtype) * size, randn(g, tk, hk, dim, dtype=dtype) * size, randn(g, tk, hk, dim, dtype=dtype)
    return (q.abs(), -k.abs(), v) if below else (q, k, v)


def check_row_heads(q, k, v, seen, scale, out, lse):
    """q, out [R, D], lse [R], k, v [K, D]; row r sees the first seen[r] keys.  -> how many rows have a clear winner."""
    q, k, v64 = q.double().cpu(), k.double().cpu(), v.double().cpu()
    score, size = (q @ k.t()) * scale, (q.abs() @ k.abs().t()) * scale
    hidden = torch.arange(k.shape[0])[None] >= torch.tensor(seen)[:, None]
    score[hidden], size[hidden] = -math.inf, 0.0
    off = q.shape[1] * 2.0 ** -23 * size.amax(1)
    first, at = score.max(1)
    rest = score.clone()
    rest[torch.arange(len(seen)), at] = -math.inf
    clear = first - rest.amax(1) > 2 * off + 200
    off_by = (out.double().cpu() - v64[at]).abs()[clear]
    assert bool((off_by <= 1.05 * 2 * U[v.dtype] * v64[at[clear]].abs() + 2.0 ** -25).all())
    assert bool(((lse.double().cpu() - first).abs()[clear] <= (off + 2.0 ** -20 * first.abs())[clear]).all())
    top = v64.abs().max() * (1 + 4 * U[v.dtype])
    assert bool((out.double().cpu().abs() <= top).all())
    return int(clear.sum())


@pytest.mark.parametrize("dtype,size,scale", SIZES)
@pytest.mark.parametrize("below", [False, True])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("causal", [False, True])
def test_prompt(dtype, size, scale, below, dim, causal):
    hq, hk, tq, tk = 4, 2, 150, 400
    q, k, v = inputs(81, dtype, size, below, tq, tk, hq, hk, dim)
    out, lse = torch.empty_like(q), torch.empty(tq, hq, device=DEV)
    AttentionSession(hq, hk, dim, dtype=dtype, scale=scale).prompt(q, k, v, starts([tq]), starts([tk]), causal=causal, out=out, lse=lse)
    seen = [i + 1 + tk - tq if causal else tk for i in range(tq)]
    clear = sum(check_row_heads(q[:, h], k[:, h // 2], v[:, h // 2], seen, scale, out[:, h], lse[:, h]) for h in range(hq))
    assert clear > tq * hq * 0.9


@pytest.mark.parametrize("dtype,size,scale", SIZES)
@pytest.mark.parametrize("below", [False, True])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("n,workspace", [(333, 0), (3000, cf.CF_ATTN_WORKSPACE_BYTES)])
def test_paged(dtype, size, scale, below, dim, n, workspace):
    hq, hk, page, seqs = 4, 2, 32, 3
    pages = -(-n // page)
    q, k, v = inputs(82, dtype, size, below, seqs, pages * page, hq, hk, dim)
    cache = PagedCache(*(x.view(pages, page, hk, dim).transpose(1, 2).contiguous() for x in (k, v)))
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(seqs, 1)
    lens = [n, n - 1, n // 2]
    out, lse = torch.empty_like(q), torch.empty(seqs, hq, device=DEV)
    AttentionSession(hq, hk, dim, dtype=dtype, scale=scale, workspace_bytes=workspace).paged(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), out=out, lse=lse)
    clear = sum(check_row_heads(q[:, h], k[:n, h // 2], v[:n, h // 2], lens, scale, out[:, h], lse[:, h]) for h in range(hq))
    assert clear > 0.9 * seqs * hq or (n == 3000 and clear > 0.5 * seqs * hq)


def test_rows_of_useless_scores_end():
    """Infinities, NaN, and scores past the largest fp32: what comes out is as useless, but it comes, and other rows are not touched by it."""
    hq, hk, d, n = 4, 2, 128, 700
    q, k, v = inputs(83, BF, 1.0, False, n, n, hq, hk, d)
    s = AttentionSession(hq, hk, d)
    want = s.prompt(q, k, v, starts([n]), starts([n]), causal=False)
    bad = q.clone()
    for i, x in enumerate([math.inf, -math.inf, math.nan, 3.0e38, -3.0e38, 1.0e20]):
        bad[20 * i] = x
        bad[20 * i + 300, :, ::2] = x
    got = s.prompt(bad, k, v, starts([n]), starts([n]), causal=False)
    same = torch.ones(n, dtype=torch.bool, device=DEV)
    same[[20 * i for i in range(6)] + [20 * i + 300 for i in range(6)]] = False
    off = (got.double() - want.double()).abs()[same]        # each is within its tolerance of the formula's, which is below 2 u of the largest value
    assert bool((off <= 4 * U[BF] * float(v.abs().max())).all())
    for x in (math.inf, math.nan, 1.0e20):
        bad_k = k.clone()
        bad_k[650:] = x
        s.prompt(q, bad_k, v, starts([n]), starts([n]), causal=True)
    torch.cuda.synchronize()
