"""Operands that lie between one another head by head: queries rotated in place between the keys and values of their heads, and an output there, too."""
import math

import pytest
import torch

from attention_reference import check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from test_gpu_attention import BF, DEV, HF, expect_prompt, gen, randn, rotated, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128), (BF, 256)])
@pytest.mark.parametrize("heads_first", [False, True])
def test_heads_of_queries_keys_values_and_outputs_side_by_side(dtype, dim, heads_first):
    g = gen(161)
    n, heads, page = 75, 3, 16
    x = randn(g, *((heads, n) if heads_first else (n, heads)), 4, dim, dtype=dtype)
    q, k, v, out = ((x.transpose(0, 1) if heads_first else x)[:, :, i] for i in range(4))
    before = x.clone()
    cache = PagedCache.empty(6, heads, dim, page_size=page, dtype=dtype)
    cos, sin = torch.rand(80, dim // 2, generator=g, device=DEV), torch.rand(80, dim // 2, generator=g, device=DEV)
    pos, slots = torch.arange(n, dtype=torch.int32, device=DEV), torch.arange(n, device=DEV)
    want = rotated(q.clone(), cos[:n][:, None], sin[:n][:, None], False)
    s = AttentionSession(heads, heads, dim, dtype=dtype)
    assert s.append(cache, k, v, slots, pos, cos, sin, q=q, q_out=q) is q
    assert torch.equal(q, want)
    for i in (1, 2, 3):
        assert torch.equal(x[:, :, i], before[:, :, i])
    s.prompt(q, k, v, starts([n]), out=out)
    res, tol = expect_prompt(q, k, v, [n], [n], True, 1 / math.sqrt(dim))
    check("out", out, res[0], tol[0])
    for i in (1, 2):
        assert torch.equal(x[:, :, i], before[:, :, i])
