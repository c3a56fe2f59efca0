"""Attention in 64 bits, sequence by sequence and head by head, and how far the kernels may be from it.

Tolerances.  With u the unit roundoff of the 16-bit type (2^-8 bf16, 2^-11 fp16), p the weights of a row and A = sum_j p_j |v_j|:
the kernels round every unnormalised weight once, by a relative u at most, which moves an output by at most u A; the
output is rounded once, by u |o|.  fp16 weights below 2^-14 are rounded by an absolute 2^-25 instead, against a sum of at
least 1: n 2^-25 max|v| over a row of n keys.  Everything else is fp32: a score of D products is off by at most D 2^-24
sum|q k| scale (and again so much for its scaling), which is the relative error of its weight.  Factor 1.05 for second-order terms."""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attend(q, k, v, seen, scale):
    """q [R, D], k and v [K, D], row r sees the first seen[r] keys. -> outputs, log-sum-exps, tolerances of both; 64 bits."""
    dt = q.dtype
    q, k, v = q.double().cpu(), k.double().cpu(), v.double().cpu()
    out, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for n in sorted(set(int(x) for x in seen)):         # rows that see the same keys together; no masked key enters at all
        rows = [r for r, x in enumerate(seen) if int(x) == n]
        if n <= 0:
            continue
        s = q[rows] @ k[:n].t() * scale
        lse[rows] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[rows][:, None])
        out[rows] = p @ v[:n]
        spread = p @ v[:n].abs()
        off = (2.0 ** -23 * q.shape[1] * scale * (q[rows].abs() @ k[:n].abs().t())).amax(1)
        u = U[dt]
        tol_o[rows] = 1.05 * (u * (spread + out[rows].abs()) + (2 * off[:, None] + 2.0 ** -20) * spread) + (n * 2.0 ** -25 * v[:n].abs().max() if dt == torch.float16 else 0.0)
        tol_l[rows] = 1.05 * off + 2.0 ** -20 * (1 + lse[rows].abs())
    return out, lse, tol_o, tol_l


def check(name, got, want, tol):
    got = got.double().cpu()
    off = (got - want).abs()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = ~(same | (off <= tol))
    assert not bool(bad.any()), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / tol.clamp(min=1e-30))[bad].max()):.3g} times the tolerance, first at {bad.nonzero()[0].tolist()}: got {got[bad][0]:.6g}, want {want[bad][0]:.6g}"
