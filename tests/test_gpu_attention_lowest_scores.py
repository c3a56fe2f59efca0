"""Finite scores next to the lowest number that fp32 holds: they are scores, not masks."""
import math

import pytest
import torch

from attention_reference import U
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, gen, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("n,at", [(1, 0), (40, 17), (700, 333)])
def test_scores_of_minus_3e38(dim, n, at):
    """All scores are -2.2e38 (-3.2e38 times log2 e), but one of -2.1e38: its value is the output, rounded once as a weight and once as an output."""
    g = gen(171)
    q, k, v = torch.zeros(3, 2, dim, dtype=BF, device=DEV), torch.zeros(n, 1, dim, dtype=BF, device=DEV), randn(g, n, 1, dim)
    q[..., 0], k[..., 0] = 2.0 ** 63, -1.3046875 * 2.0 ** 64
    k[at, :, 0] = -1.2421875 * 2.0 ** 64
    assert float(q[0, 0, 0]) * float(k[at, 0, 0]) * math.log2(math.e) < -3.0e38
    lse = torch.empty(3, 2, device=DEV)
    out = AttentionSession(2, 1, dim, scale=1.0).prompt(q, k, v, starts([3]), starts([n]), causal=False, lse=lse)
    cache = PagedCache(*(torch.nn.functional.pad(x.transpose(0, 1), (0, 0, 0, 1024 - n)).view(1, 1, 1024, dim).contiguous() for x in (k, v)))
    lse_paged = torch.empty(3, 2, device=DEV)
    paged = AttentionSession(2, 1, dim, scale=1.0).paged(cache, q, torch.zeros(3, 1, dtype=torch.int32, device=DEV), torch.full((3,), n, dtype=torch.int32, device=DEV), lse=lse_paged)
    want = v[at, 0].double()
    for o, l in ((out, lse), (paged, lse_paged)):
        assert bool(((o.double() - want).abs() <= 1.05 * 2 * U[BF] * want.abs()).all())
        assert bool(((l.double() / (-1.2421875 * 2.0 ** 127) - 1).abs() <= 2.0 ** -20).all())
