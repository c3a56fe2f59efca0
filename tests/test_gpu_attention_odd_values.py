"""Values that are infinite or NaN at keys which some rows of a tile see and others do not: with split keys, wide groups, many tiles before them,
and scores so large that a wave leaves the loop for ordinary ones."""
import math

import pytest
import torch

from attention_reference import attend, check
from paper_2507_17511_amd.attention import AttentionSession
from test_gpu_attention import BF, DEV, HF, gen, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128), (BF, 256)])
@pytest.mark.parametrize("hq,hk,tq,tk", [(4, 1, 20, 3000), (10, 2, 70, 700), (2, 2, 130, 130), (3, 3, 9, 2000)])
@pytest.mark.parametrize("back", [1, 7])
def test_rows_before_an_odd_value(bad, dtype, dim, hq, hk, tq, tk, back):
    """The value of one key, `back` from the end, is odd in every fifth place: rows that see it have it there, and nothing of it elsewhere."""
    g = gen(101)
    q, k, v = randn(g, tq, hq, dim, dtype=dtype) * 0.3, randn(g, tk, hk, dim, dtype=dtype), randn(g, tk, hk, dim, dtype=dtype)
    clean = v.clone()
    v[tk - back, :, ::5] = bad
    s = AttentionSession(hq, hk, dim, dtype=dtype)
    lse = torch.empty(tq, hq, device=DEV)
    out = s.prompt(q, k, v, starts([tq]), starts([tk]), causal=True, lse=lse)
    seen = [i + 1 + tk - tq for i in range(tq)]
    sees = torch.tensor([n > tk - back for n in seen])
    odd = torch.arange(dim) % 5 == 0
    there = out[sees][..., odd]
    assert bool((torch.isnan(there) if math.isnan(bad) else there == bad).all())
    for h in range(hq):
        o, l, to, tl = attend(q[:, h], k[:, h // (hq // hk)], clean[:, h // (hq // hk)], seen, 1 / math.sqrt(dim))
        check("rows before it", out[~sees, h], o[~sees], to[~sees])
        check("places beside it", out[:, h, ~odd], o[:, ~odd], to[:, ~odd])
        check("lse", lse[:, h], l, tl)


@pytest.mark.parametrize("dtype,dim", [(BF, 64), (HF, 128), (BF, 256)])
def test_odd_values_next_to_large_scores(dtype, dim):
    """Scores near 2^31 (fp16: by the scale): each row's output is the value of its largest score, whatever later keys hold."""
    g = gen(102)
    hq, hk, n = 2, 1, 200
    size = 2.0 ** 14 if dtype == BF else 2.0 ** 6
    q, k, v = randn(g, n, hq, dim, dtype=dtype) * size, randn(g, n, hk, dim, dtype=dtype) * size, randn(g, n, hk, dim, dtype=dtype)
    scale = 1.0 if dtype == BF else 2.0 ** 16
    v[150:] = math.nan
    out = AttentionSession(hq, hk, dim, dtype=dtype, scale=scale).prompt(q, k, v, starts([n]), causal=True)
    score = torch.stack([q[:, h].double().cpu() @ k[:, 0].double().cpu().t() for h in range(hq)], 1) * scale
    score = score.masked_fill(torch.arange(n)[None, None] > torch.arange(n)[:, None, None], -math.inf)
    top = score.topk(2, -1).values
    size_of = torch.stack([q[:, h].double().cpu().abs() @ k[:, 0].double().cpu().abs().t() for h in range(hq)], 1).amax(-1) * scale
    clear = (top[..., 0] - top[..., 1] > 2 * dim * 2.0 ** -23 * size_of + 200) & (torch.arange(n) < 150)[:, None]
    assert int(clear.sum()) > 250
    want = v[:, 0].double().cpu()[score.argmax(-1)]
    u = 2.0 ** -8 if dtype == BF else 2.0 ** -11
    off = (out.double().cpu() - want).abs()[clear]
    assert bool((off <= 1.05 * 2 * u * want.abs()[clear] + 2.0 ** -25).all())
    assert bool(torch.isnan(out[150:].float()).all())
