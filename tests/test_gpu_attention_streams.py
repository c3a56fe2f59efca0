"""Sessions on a stream of their own next to a busy one: the workspace is zero before its first call, and an output that a call
allocates is not memory that the other stream is still writing."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import DEV, gen, randn

pytestmark = pytest.mark.gpu

HQ, HK, D, PAGE, N = 8, 2, 128, 16, 3000


def problem():
    g = gen(91)
    pages = -(-N // PAGE)
    cache = PagedCache(randn(g, pages, HK, PAGE, D), randn(g, pages, HK, PAGE, D))
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    q = randn(g, 1, HQ, D)
    torch.cuda.synchronize()
    return cache, q, table, torch.tensor([N], dtype=torch.int32, device=DEV)


def busy(work):
    """Some 20 ms on the current stream."""
    for _ in range(40):
        torch.mm(work, work)


def check_out(cache, q, out):
    k, v = (x.transpose(1, 2).reshape(-1, HK, D)[:N] for x in (cache.k, cache.v))
    for h in range(HQ):
        o, _, to, _ = attend(q[:, h], k[:, h // 4], v[:, h // 4], [N], 1 / math.sqrt(D))
        check("out", out[:, h], o, to)


def test_the_workspace_is_zero_for_the_first_call_on_another_stream():
    cache, q, table, lens = problem()
    work, side = torch.randn(6144, 6144, device=DEV).bfloat16(), torch.cuda.Stream()
    old = torch.full((cf.CF_ATTN_WORKSPACE_BYTES,), 255, dtype=torch.uint8, device=DEV)
    torch.mm(work, work)
    torch.cuda.synchronize()
    busy(work)
    del old
    s = AttentionSession(HQ, HK, D)
    with torch.cuda.stream(side):
        out = s.paged(cache, q, table, lens)
    torch.cuda.synchronize()
    check_out(cache, q, out)


def test_an_output_is_not_memory_that_another_stream_writes():
    cache, q, table, lens = problem()
    work, side = torch.randn(6144, 6144, device=DEV).bfloat16(), torch.cuda.Stream()
    s = AttentionSession(HQ, HK, D, stream=side)
    old = torch.empty_like(q)
    torch.mm(work, work)
    torch.cuda.synchronize()
    busy(work)
    old.fill_(7.0)
    del old
    out = s.paged(cache, q, table, lens)
    torch.cuda.synchronize()
    check_out(cache, q, out)
