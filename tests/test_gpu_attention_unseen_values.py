"""Infinite and NaN values at keys that a row does not see leave the row as it is, to the last bit; so do those places of a value that are finite, for rows
that see it."""
import math

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession
from test_gpu_attention import BF, DEV, HF, gen, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("hq,hk,tq,tk,workspace", [(6, 2, 140, 140, 0), (2, 1, 50, 1000, 0), (2, 1, 90, 700, 0), (1, 1, 40, 3000, cf.CF_ATTN_WORKSPACE_BYTES), (3, 3, 300, 200, 0)])
@pytest.mark.parametrize("back", [1, 8, 40])
def test_causal_rows(bad, dtype, dim, hq, hk, tq, tk, workspace, back):
    g = gen(131)
    q, k, v = randn(g, tq, hq, dim, dtype=dtype), randn(g, tk, hk, dim, dtype=dtype), randn(g, tk, hk, dim, dtype=dtype)
    spoiled = v.clone()
    spoiled[tk - back, :, ::5] = bad
    s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace)
    lse, want_lse = torch.empty(tq, hq, device=DEV), torch.empty(tq, hq, device=DEV)
    want = s.prompt(q, k, v, starts([tq]), starts([tk]), lse=want_lse)
    got = s.prompt(q, k, spoiled, starts([tq]), starts([tk]), lse=lse)
    sees = torch.arange(tq, device=DEV) + 1 + tk - tq > tk - back
    odd = torch.arange(dim, device=DEV) % 5 == 0
    assert torch.equal(got[~sees], want[~sees])
    assert torch.equal(got[..., ~odd], want[..., ~odd])
    assert torch.equal(lse, want_lse)
    there = got[sees][..., odd]
    assert bool((torch.isnan(there) if math.isnan(bad) else there == bad).all())


@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 64), (BF, 128), (HF, 128), (BF, 256), (HF, 256)])
def test_the_next_sequence(dtype, dim):
    """Keys past a sequence, and past a part of a split one, are another's."""
    g = gen(132)
    lens = [100, 37, 200, 64, 33]
    n = sum(lens)
    q, k, v = randn(g, n, 4, dim, dtype=dtype), randn(g, n, 2, dim, dtype=dtype), randn(g, n, 2, dim, dtype=dtype)
    s = AttentionSession(4, 2, dim, dtype=dtype)
    for causal in (False, True):
        want = s.prompt(q, k, v, starts(lens), causal=causal)
        for b in range(len(lens)):
            rows = slice(sum(lens[:b]), sum(lens[:b + 1]))
            spoiled_k, spoiled_v = k.clone(), v.clone()
            spoiled_k[rows], spoiled_v[rows] = math.nan, math.inf
            got = s.prompt(q, spoiled_k, spoiled_v, starts(lens), causal=causal)
            others = torch.ones(n, dtype=torch.bool, device=DEV)
            others[rows] = False
            assert torch.equal(got[others], want[others])


@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128), (BF, 256)])
def test_many_odd_values_behind_a_long_edge(dtype, dim):
    """Every value from some key on is NaN, for all rows before it: as many tiles with an edge in them as rows have."""
    g = gen(133)
    n = 1500
    q, k, v = randn(g, n, 2, dim, dtype=dtype), randn(g, n, 2, dim, dtype=dtype), randn(g, n, 2, dim, dtype=dtype)
    s = AttentionSession(2, 2, dim, dtype=dtype)
    want = s.prompt(q, k, v, starts([n]))
    for first in (1, 63, 64, 700, 1025, 1499):
        spoiled = v.clone()
        spoiled[first:] = math.nan
        got = s.prompt(q, k, spoiled, starts([n]))
        assert torch.equal(got[:first], want[:first]) and bool(torch.isnan(got[first:].float()).all())
