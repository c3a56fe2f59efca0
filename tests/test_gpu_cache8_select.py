"""Which pages are selected where scores are infinite, and in contexts of more pages than the threads of a workgroup hold: against a stable sort of scores in 64 bits."""
import math
import random

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession, PagedCache8
from test_gpu_cache8 import BF, DEV, HF, gen, ints, randn

pytestmark = pytest.mark.gpu


def wanted(q, bounds, rows, lens, page, count, first, recent):
    """The largest scores, of equal ones the earlier, NaN last."""
    q, bounds, got = q.double().cpu(), bounds.double().cpu(), []
    group = q.shape[1] // bounds.shape[1]
    for b, n in enumerate(lens):
        held = -(-n // page)
        got.append([])
        for h in range(bounds.shape[1]):
            if held <= count:
                got[-1].append(list(range(held)) + [-1] * (count - held))
                continue
            low, high = bounds[rows[b][:held], h, 0], bounds[rows[b][:held], h, 1]
            score = sum(torch.maximum(low * x, high * x).sum(-1) for x in q[b, h * group:(h + 1) * group])[first:held - recent]
            order = torch.sort(score.nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf), descending=True, stable=True)[1]
            order = order[torch.sort(score[order].isnan().int(), stable=True)[1]]
            got[-1].append(list(range(first)) + sorted((order[:count - first - recent] + first).tolist()) + list(range(held - recent, held)))
    return got


def run(seed, dtype, hq, hk, dim, page, lens, count, first=0, recent=0, change=None, pages=None, workspace_bytes=cf.CF_ATTN_WORKSPACE_BYTES):
    """Lists go into the middle of a larger buffer, of which nothing else changes."""
    g, r = gen(seed), random.Random(seed)
    per = [max(1, -(-n // page)) for n in lens]
    pages = pages or sum(per)
    x = randn(g, pages, hk, 2, dim) + torch.tensor([-1.0, 1.0], device=DEV, dtype=BF)[:, None]
    bounds = torch.stack((x.amin(2), x.amax(2)), 2)
    q = randn(g, len(lens), hq, dim, dtype=dtype)
    if change is not None:
        change(q, bounds)
    codes = torch.zeros((1, hk, page, dim), dtype=torch.float8_e4m3fn, device=DEV).expand(pages, hk, page, dim).contiguous()
    cache = PagedCache8(codes, codes.clone(), *torch.ones((2, pages, hk), device=DEV), bounds)
    rows = [[r.randrange(pages) for _ in range(p)] for p in per]
    table = torch.full((len(lens), max(per)), -3, dtype=torch.int32)
    for b, row in enumerate(rows):
        table[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    out = torch.full((len(lens) + 2, hk, count), 7, dtype=torch.int32, device=DEV)
    s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace_bytes)
    s.select(cache, q, table.to(DEV), ints(lens), count, first=first, recent=recent, out=out[1:-1])
    torch.cuda.synchronize()
    assert bool((out[[0, -1]] == 7).all())
    assert out[1:-1].tolist() == wanted(q, bounds, rows, lens, page, count, first, recent)


def split_signs(bounds, channel):
    """Half of the pages have a channel's keys on one side of zero, half on the other; none is zero."""
    bounds[..., channel] = torch.tensor([0.5, 2.0], dtype=BF, device=DEV)
    bounds[::2, ..., channel] = torch.tensor([-2.0, -0.5], dtype=BF, device=DEV)


def one(q, bounds):
    split_signs(bounds, 3)
    q[:, :, 3] = math.inf


def minus(q, bounds):
    split_signs(bounds, 3)
    q[:, :, 3] = -math.inf


def finite_or_infinite(q, bounds):         # the infinite channel's keys lie on both sides of zero on some pages: all of those score +infinity
    split_signs(bounds, 3)
    bounds[::3, ..., 3] = torch.tensor([-1.0, 1.0], dtype=BF, device=DEV)
    q[0, :, 3], q[1:, 0, 3] = math.inf, -math.inf


def largest(q, bounds):                    # +infinity, and the largest finite numbers of either sign
    split_signs(bounds, 3)
    bounds[:, :, :, 5] = torch.tensor([-3.0e38, -2.0e38], dtype=BF, device=DEV)
    bounds[::5, :, :, 5] = torch.tensor([2.0e38, 3.0e38], dtype=BF, device=DEV)
    q[:, :, 5] = 60000.0
    q[::2, 0, 3] = math.inf


def both_and_nan(q, bounds):               # infinities of both signs meet: NaN on some pages
    split_signs(bounds, 3)
    split_signs(bounds, 7)
    bounds[1::3, ..., 7] *= -1
    bounds.copy_(torch.stack((bounds.amin(2), bounds.amax(2)), 2))
    q[:, 0, 3], q[:, -1, 7] = math.inf, math.inf
    q[0, 0, 9] = math.nan


@pytest.mark.parametrize("change", [one, minus, finite_or_infinite, largest, both_and_nan])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("count,first,recent", [(1, 0, 0), (10, 0, 0), (50, 1, 1), (470, 3, 2)])
def test_infinite_scores(change, dtype, count, first, recent):
    run(51, dtype, 4, 2, 64, 16, [1600, 16 * 900, 100, 16 * 60], count, first, recent, change)
    run(52, dtype, 4, 2, 128, 16, [16 * 2500, 1600, 100], count, first, recent, change)
    run(53, dtype, 6, 2, 256, 32, [32 * 700, 3200], count, first, recent, change, pages=60)


# Contexts past the 8192 pages whose scores stay in registers: 8 a thread, 1024 threads.

LONG = [16 * 20001 - 3, 16 * 8193, 16 * 8192, 16 * 16384, 1600, 0]


@pytest.mark.parametrize("count,first,recent", [(1, 0, 0), (100, 1, 1), (9000, 0, 0), (8200, 8190, 4), (15000, 8193, 3), (15000, 2, 11900), (20000, 0, 0), (12000, 6000, 6000)])
@pytest.mark.parametrize("pages", [40, None])
def test_contexts_whose_scores_are_read_again(count, first, recent, pages):
    """Few physical pages: many equal scores on both sides of a turn's border.  Pages of their own: scores that differ."""
    run(54, BF, 4, 2, 64, 16, LONG, count, first, recent, pages=pages)


def nothing(q, bounds):
    q.zero_()


def nan_here_and_there(q, bounds):
    bounds[::3, :, 1, 5] = math.nan
    q[1, 0, 3] = math.nan


def two_scores(q, bounds):                 # one of 1 on every seventh page, 0 elsewhere: ties that lie across all turns
    bounds.zero_()
    bounds[::7, :, 1, 0] = 1.0
    q.zero_()
    q[:, 0, 0] = 1.0


@pytest.mark.parametrize("change", [nothing, nan_here_and_there, two_scores, one, both_and_nan])
@pytest.mark.parametrize("count,first,recent", [(100, 1, 1), (2000, 0, 0), (8192, 0, 1), (8193, 1, 0), (16385, 100, 100)])
def test_equal_scores_across_turns(change, count, first, recent):
    run(55, BF, 2, 1, 64, 16, LONG, count, first, recent, change)
    run(56, HF, 4, 2, 128, 16, LONG[:4], count, first, recent, change, pages=77)


def test_long_contexts_some_heads_at_a_time():
    """A workspace for the scores of three heads of the eight."""
    run(57, BF, 4, 2, 64, 16, LONG[:4], 100, 1, 1, workspace_bytes=cf.CF_ATTN_COUNTER_BYTES + 3 * 20001 * 8 // 256 * 256 + 256)
