"""The cache in 8 bits in plain Python and 64 bits: codes, plans, and the attention over codes.

Codes.  A number below 448 scales has 4 significant bits, or is a multiple of 2^-9 scales: rounding it once is off by at most 2^-4 of it, or by
2^-10 scales.  Nothing else is rounded but the rotation: three fp32 operations of terms |a cos| and |b sin|, 2 x 2^-24 of their sum in all."""
import math

import torch

from attention_reference import attend

LEAST, MOST = -100, 119
MOST_VALUE = {torch.bfloat16: 448.0 * 2.0 ** 119, torch.float16: 240.0 * 2.0 ** 8}


def exponent_for(most):
    """The least e in range with most <= 448 x 2^e."""
    e = LEAST
    while e < MOST and most > math.ldexp(448.0, e):
        e += 1
    return e


def e4m3(x):
    """fp64 -> the nearest code's value, ties to even; NaN stays."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def rotate(x, cos, sin, rotary, interleaved):
    """x [tokens, heads, dim] fp64, cos and sin rows of the tokens.  -> rotated, and the sum of the terms' magnitudes."""
    y, size = x.clone(), x.abs()
    i = torch.arange(rotary // 2)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    a, b, c, s = x[..., first], x[..., second], cos.double()[:, None], sin.double()[:, None]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first], size[..., second] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, size


class Cache:
    """k or v as appends leave it: codes' values and exponents, on the host."""

    def __init__(self, codes, scale, bounds=None):
        self.codes, self.scale = codes.float().double().cpu(), scale.double().cpu()
        self.bounds = None if bounds is None else bounds.double().cpu()

    def append(self, x, slots, dtype):
        """x [tokens, heads, dim] fp64, slots a list (None or outside: left out); tokens of a page are neighbours."""
        pages, heads, page = self.codes.shape[:3]
        x = x.clamp(-MOST_VALUE[dtype], MOST_VALUE[dtype])
        for p in dict.fromkeys(s // page for s in slots if s is not None and 0 <= s < pages * page):
            rows = [t for t, s in enumerate(slots) if s is not None and s // page == p]
            begun = any(slots[t] % page == 0 for t in rows)
            for h in range(heads):
                e = exponent_for(float(x[rows, h].abs().nan_to_num(nan=0.0).max()))
                old = self.scale[p, h].item()
                if not begun:
                    e = max(e, int(math.log2(old)))
                    if 2.0 ** e > old:
                        self.codes[p, h] = e4m3(self.codes[p, h] * (old / 2.0 ** e))
                self.scale[p, h] = 2.0 ** e
                y = e4m3(x[rows, h] / 2.0 ** e)
                for i, t in enumerate(rows):
                    self.codes[p, h, slots[t] % page] = y[i]
                if self.bounds is not None:
                    y, none = y * 2.0 ** e, y.isnan().all(0)
                    low, high = (torch.where(none, 0.0, f(torch.where(y.isnan(), z, y), 0)) for f, z in ((torch.amin, math.inf), (torch.amax, -math.inf)))
                    if not begun:
                        low, high = torch.where(none, self.bounds[p, h, 0], low), torch.where(none, self.bounds[p, h, 1], high)
                        low, high = torch.minimum(low, self.bounds[p, h, 0]), torch.maximum(high, self.bounds[p, h, 1])
                    self.bounds[p, h, 0], self.bounds[p, h, 1] = low, high

    def values(self):
        return self.codes * self.scale[:, :, None, None]


def keys_of(cache, row, n, head, blocks=None):
    """cache: values, fp64 [pages, heads, page, dim].  -> [keys, dim] of a context's pages, or of those that are listed."""
    page = cache.shape[2]
    held = -(-n // page)
    listed = range(held) if blocks is None else [j for j in blocks[:held] if 0 <= j < held]
    got = [cache[row[j], head, :min(page, n - j * page)] for j in listed]
    return torch.cat(got) if got else torch.zeros((0, cache.shape[3]), dtype=torch.float64)


def attention(q, k, v, table, lens, scale, blocks=None):
    """Over Cache k and v.  -> outputs, log-sum-exps, and their tolerances (attention_reference)."""
    n, hq, hk, q, k, v = q.shape[0], q.shape[1], k.codes.shape[1], q.cpu(), k.values(), v.values()
    out, lse = torch.zeros(q.shape, dtype=torch.float64), torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    tol_o, tol_l = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(n):
        for h in range(hk):
            rows = slice(h * (hq // hk), (h + 1) * (hq // hk))
            listed = None if blocks is None else blocks[b][h]
            kk, vv = keys_of(k, table[b], lens[b], h, listed), keys_of(v, table[b], lens[b], h, listed)
            if len(kk):
                out[b, rows], lse[b, rows], tol_o[b, rows], tol_l[b, rows] = attend(q[b, rows], kk, vv, [len(kk)] * (hq // hk), scale)
    return out, lse, tol_o, tol_l


def select(q, bounds, table, lens, page, count, first, recent):
    """Lists of pages, by the sum of the heads' bounds in fp64 and by place."""
    n, hq, hk = q.shape[0], q.shape[1], bounds.shape[1]
    q, bounds, got = q.double().cpu(), bounds.double().cpu(), []
    for b in range(n):
        held = -(-lens[b] // page)
        got.append([])
        for h in range(hk):
            low, high = bounds[table[b][:held], h, 0], bounds[table[b][:held], h, 1]
            score = sum(torch.maximum(low * x, high * x).sum(-1) for x in q[b, h * (hq // hk):(h + 1) * (hq // hk)]).tolist() if held else []
            always = [j for j in range(held) if j < first or j >= held - recent] if held > count else list(range(held))
            others = sorted((j for j in range(held) if j not in always), key=lambda j: (-score[j] if score[j] == score[j] else math.inf, j))
            got[-1].append(sorted(always + others[:count - len(always)]) + [-1] * max(0, count - held))
    return got


def plan(lens, news, table, ring, state, page, tokens):
    """-> table, ring, state, lens, cu, slots, positions, refused after the call."""
    table, ring, (taken, put) = [list(r) for r in table], list(ring), state
    was, free, used, short, refused = list(ring), put - taken, 0, False, 0
    cu, out, slots, positions, at = [0], [], [], [], 0
    back = 0
    for row, n, new in zip(table, lens, news):
        held = -(-n // page)
        if new < 0:
            for j in range(held):
                ring[(put + back) % len(ring)] = row[j]
                back += 1
            out.append(0)
            cu.append(min(at, tokens))
            continue
        at += new
        cu.append(min(at, tokens))
        fits = n + new <= len(row) * page
        need = -(-(n + new) // page) - held
        short |= fits and need > 0 and used + need > free
        ok = fits and at <= tokens and not (short and need)
        if not ok:
            refused += new > 0
            out.append(n)
            slots += [-1] * new
            positions += [-1] * new
            continue
        for j in range(need):
            row[held + j] = was[(taken + used + j) % len(ring)]
        used += need
        out.append(n + new)
        positions += range(n, n + new)
        slots += [row[p // page] * page + p % page for p in range(n, n + new)]
    slots, positions = (slots + [-1] * tokens)[:tokens], (positions + [-1] * tokens)[:tokens]
    return table, ring, [taken + used, put + back], out, cu, slots, positions, refused
