"""The join at every number of parts: rows that some or all parts have no keys for, outputs of such parts that are not read."""
import math

import pytest
import torch

from attention_reference import U, check
from paper_2507_17511_amd.attention import AttentionSession
from test_gpu_attention import BF, DEV, HF, gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,wide,dim", [(BF, False, 64), (HF, True, 128), (BF, True, 256), (HF, False, 256)])
@pytest.mark.parametrize("parts", [1, 2, 4, 5, 8, 9, 16, 17, 33, 63, 64])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (37, 3)])
def test_join_of_any_number_of_parts(dtype, wide, dim, parts, tokens, heads):
    g = gen(71)
    ps = torch.stack([randn(g, tokens, heads, dim, dtype=torch.float32 if wide else dtype) for _ in range(parts)])
    ls = torch.randn(parts, tokens, heads, generator=g, device=DEV) * 5
    gone = torch.rand(parts, tokens, heads, generator=g, device=DEV) < 0.3
    if tokens > 1:
        gone[:, 5], gone[:, 6] = True, False
        gone[:-1, 7], gone[-1, 7] = True, False
    ls[gone], ps[gone] = -math.inf, math.nan
    lse = torch.empty(tokens, heads, device=DEV)
    out = AttentionSession(heads, heads, dim, dtype=dtype).join(list(ps), list(ls), lse=lse)
    l = ls.double().cpu()
    total = torch.logsumexp(l, 0)
    w = torch.where(l == -math.inf, torch.zeros_like(l), torch.exp(l - total))[..., None]
    x = torch.where(gone.cpu()[..., None], torch.zeros(1, dtype=torch.float64), ps.double().cpu())
    want, spread = (w * x).sum(0), (w * x.abs()).sum(0)
    # fp32 throughout: the exponent of a weight is off by a few 2^-24 of a difference of 40 at most; one rounding to the type, whose steps
    # below 2^-14 are 2^-24 in fp16
    check("out", out, want, 1.05 * U[dtype] * want.abs() + 2.0 ** -16 * spread + (2.0 ** -25 if dtype == HF else 0.0))
    check("lse", lse, total, 2.0 ** -20 * (1 + total.abs()))
