"""A HIP call of someone else's that failed before, and that nobody asked about: it is no failure of an attention call."""
import ctypes

import pytest
import torch

from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import DEV, gen, randn, starts

pytestmark = pytest.mark.gpu


def test_an_error_that_was_there_is_not_the_calls_own():
    g = gen(181)
    q, k, v = randn(g, 20, 4, 64), randn(g, 20, 2, 64), randn(g, 20, 2, 64)
    cache = PagedCache(randn(g, 8, 2, 16, 64), randn(g, 8, 2, 16, 64))
    table, lens = torch.arange(8, dtype=torch.int32, device=DEV).repeat(20, 1), torch.full((20,), 100, dtype=torch.int32, device=DEV)
    s = AttentionSession(4, 2, 64)
    cu, slots, out, lse = starts([20]), torch.arange(20, device=DEV), torch.empty_like(q), torch.zeros(20, 4, device=DEV)
    hip = ctypes.CDLL("libamdhip64.so")
    calls = [lambda: s.prompt(q, k, v, cu, out=out), lambda: s.paged(cache, q, table, lens, out=out), lambda: s.append(cache, k, v, slots, q=q, q_out=out),
             lambda: s.join([q, q], [lse, lse], out=out)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    try:
        for call in calls:
            assert hip.hipSetDevice(1000) != 0          # refused by the runtime, which remembers it
            call()
    finally:
        hip.hipGetLastError()
    torch.cuda.synchronize()
