"""Codes of all finite numbers of both types; and appends of as many rows as let a workgroup look for pages among more tokens, up to 64, with pages' tokens
on both sides of its border.  References are in 64 bits and for all pages at once; nothing of them is rounded but codes, so that without a rotation everything is equal."""
import math
import random

import pytest
import torch

import cache8_reference as ref
from paper_2507_17511_amd.attention import AttentionSession, PagedCache8
from test_gpu_cache8 import BF, DEV, HF, filled, gen, ints, randn

pytestmark = pytest.mark.gpu


def exponents(most):
    """The least e in range with most <= 448 x 2^e = 0.875 x 2^(e + 9)."""
    m, k = torch.frexp(most)
    return torch.where(most == 0, ref.LEAST, torch.where(m <= 0.875, k - 9, k - 8)).clamp(ref.LEAST, ref.MOST)


def finite(dtype):
    x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype)
    return x[x.isfinite()]


def same_codes(got, want):
    """Numbers and their signs, those of zeros among them."""
    return torch.equal(got.double(), want) and torch.equal(got.double().signbit(), want.signbit())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_every_number_up_to_448_at_a_scale_of_1(dtype):
    """Both signs, zeros and subnormal numbers among them.  448 at every page's first place."""
    x = finite(dtype)
    x = x[x.abs() <= 448]
    page, heads, dim = 128, 4, 64
    each = (page - 1) * heads * dim
    pages = -(-x.numel() // each)
    x = x.repeat(2)[:pages * each]                      # all of them, and some again
    assert x.view(torch.int16).unique().numel() == {BF: 34754, HF: 48642}[dtype]
    k = torch.full((pages, page, heads, dim), 448.0, dtype=dtype)
    k[:, 1:] = x.view(pages, page - 1, heads, dim)
    k = k.view(pages * page, heads, dim).to(DEV)
    cache = PagedCache8.empty(pages, heads, dim, page)
    AttentionSession(heads, heads, dim, dtype=dtype).append8(cache, k, k, torch.arange(pages * page, device=DEV))
    torch.cuda.synchronize()
    assert bool((cache.k_scale == 1).all()) and bool((cache.v_scale == 1).all())
    got = cache.k.cpu().float().permute(0, 2, 1, 3).reshape(k.shape)
    assert same_codes(got, ref.e4m3(k.double().cpu())) and torch.equal(got, k.float().cpu().to(torch.float8_e4m3fn).float())
    assert torch.equal(cache.v.view(torch.uint8), cache.k.view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("lone", [True, False])
def test_every_finite_number_next_to_those_of_its_size(dtype, lone):
    """In the order of their magnitudes, a token of 64 or a page of 16 x 64 at a time: scales from the least to the largest, numbers past what a code holds."""
    x = finite(dtype)
    x = x[torch.argsort(x.abs().float(), stable=True)]
    page, dim = 16, 64
    tokens = -(-x.numel() // (page * dim)) * page
    k = torch.cat((x, x[-1:].expand(tokens * dim - x.numel()))).view(tokens, 1, dim)
    at = torch.arange(tokens) * page if lone else torch.arange(tokens)
    pages = tokens if lone else tokens // page
    cache = PagedCache8.empty(pages, 1, dim, page)
    AttentionSession(1, 1, dim, dtype=dtype).append8(cache, k.to(DEV), k.to(DEV), at.to(DEV))
    torch.cuda.synchronize()
    y = k.double().clamp(-ref.MOST_VALUE[dtype], ref.MOST_VALUE[dtype]).view(pages, -1, dim)
    e = exponents(y.abs().amax((1, 2)))
    assert torch.equal(cache.k_scale.double().cpu()[:, 0], torch.exp2(e.double())) and torch.equal(cache.v_scale, cache.k_scale)
    want = ref.e4m3(y * torch.exp2(-e.double())[:, None, None])
    got = cache.k.cpu().float()[:, 0, :y.shape[1]]
    assert same_codes(got, want) and torch.equal(cache.v.cpu().float()[:, 0, :y.shape[1]], got)
    assert torch.equal(cache.bounds[:, 0, 0].double().cpu(), (want * torch.exp2(e.double())[:, None, None]).amin(1))
    assert torch.equal(cache.bounds[:, 0, 1].double().cpu(), (want * torch.exp2(e.double())[:, None, None]).amax(1))


# ---------------------------------------------------------------- how a call's tokens are dealt out

def dealt(seed, n, page, chunk, left_out):
    """Slots of n tokens, each page's neighbours of one another: lone tokens and runs, pages that begin in the last places that a workgroup looks at and go on
    in the next ones'; tokens without a place in between.  -> slots, and pages."""
    r, slots, pages = random.Random(seed), [], 0
    while len(slots) < n:
        at = len(slots) % chunk
        if left_out and r.random() < 0.15:
            slots += [r.choice([-1, -9, 10 ** 15])]
            continue
        alone = 0.95 if len(slots) // (4 * chunk) % 2 else 0.5          # stretches of tokens that have a page each, and others
        lone = r.random() < (0.2 if at in (0, chunk - 2, chunk - 1) else alone)
        count = 1 if lone else r.randint(2, page)
        first = r.choice([0, r.randrange(page - count + 1)])
        slots += [pages * page + first + i for i in range(count)]
        pages += 1
    return slots[:n], pages


def over_pages(pages, of, x, how, start):
    """x [tokens, ...]: the largest (least) of each page's tokens."""
    return torch.full((pages, *x.shape[1:]), start, dtype=x.dtype, device=x.device).scatter_reduce_(0, of.view(-1, *[1] * (x.dim() - 1)).expand_as(x), x, how)


def append_and_compare(seed, dtype, n, hq, hk, dim, page, chunk, rotary=0, left_out=True):
    assert min(64, -(--(-n * 2 * hk // 2048) // 8) * 8) == chunk       # what the call's sizes lead to
    g = gen(seed)
    slots, pages = dealt(seed, n, page, chunk, left_out)
    at = torch.tensor(slots, device=DEV)
    k, v = randn(g, n, hk, dim, dtype=dtype), randn(g, n, hk, dim, dtype=dtype, scale=3.0)
    size = torch.exp2(torch.randint(-12, 12, (n, hk, 1), generator=g, device=DEV)).to(dtype)
    k, v = k * size, v * size
    cache = filled(seed + 1, pages, hk, page, dim, True)
    was = [x.float().double() for x in (cache.k, cache.v)], [x.double() for x in (cache.k_scale, cache.v_scale)], cache.bounds.double()
    s, q = AttentionSession(hq, hk, dim, dtype=dtype), randn(g, n, hq, dim, dtype=dtype)
    there = (at >= 0) & (at < pages * page)
    kw, turned = {}, [k.double(), q.double(), k.double().abs(), q.double().abs()]
    if rotary:
        angle = torch.arange(500, dtype=torch.float64)[:, None] * 100.0 ** -(torch.arange(rotary // 2, dtype=torch.float64) / (rotary // 2))
        positions = torch.randint(-30 if left_out else 0, 500, (n,), generator=g, device=DEV, dtype=torch.int32)
        kw = dict(positions=positions, cos=angle.cos().float().to(DEV), sin=angle.sin().float().to(DEV))
        there &= positions >= 0
        rows = [x[positions.clamp(min=0).long()].cpu() for x in (kw["cos"], kw["sin"])]
        turned = [x.to(DEV) for pair in zip(*(ref.rotate(x.double().cpu(), *rows, rotary, False) for x in (k, q))) for x in pair]
    out = s.append8(cache, k, v, at, q=q, q_out=torch.full_like(q, 7.0), **kw)
    torch.cuda.synchronize()
    known = torch.ones_like(there)
    if rotary:
        known = positions >= 0
        u = {BF: 2.0 ** -8, HF: 2.0 ** -11}[dtype]
        assert bool(((out.double() - turned[1]).abs() <= 1.01 * u * turned[1].abs() + 2.0 ** -23 * turned[3] + 2.0 ** -25)[known].all())
    else:
        assert torch.equal(out, q)
    assert bool((out[~known] == 7).all())
    of = at[there] // page
    place = at[there] % page
    begun = torch.zeros(pages, dtype=torch.bool, device=DEV)
    begun[of[place == 0]] = True
    used = torch.zeros(pages, dtype=torch.bool, device=DEV)
    used[of] = True
    for name, codes, scale, x, got, got_scale in (("k", was[0][0], was[1][0], turned[0], cache.k, cache.k_scale), ("v", was[0][1], was[1][1], v.double(), cache.v, cache.v_scale)):
        x = x[there].clamp(-ref.MOST_VALUE[dtype], ref.MOST_VALUE[dtype])
        most = over_pages(pages, of, x.abs().amax(2), "amax", 0.0)
        e = exponents(most)
        before = torch.log2(scale).round().int()
        e = torch.where(used[:, None], torch.where(begun[:, None], e, torch.maximum(e, before)), before)
        grown = used & ~begun
        codes[grown] = torch.where((e > before)[grown][..., None, None], ref.e4m3(codes[grown] * torch.exp2((before - e)[grown].double())[..., None, None]), codes[grown])
        y = ref.e4m3(x * torch.exp2(-e[of].double())[..., None])
        codes[of, :, place] = y
        scale = torch.exp2(e.double())
        assert torch.equal(got_scale.double(), scale)
        got = got.float().double()
        if name == "v" or not rotary:
            assert torch.equal(got, codes)
        else:               # the rotation's rounding lets a code go the other way next to a tie
            step = torch.exp2(torch.floor(torch.log2(codes.abs().clamp(min=2.0 ** -6))) - 3)
            assert bool(((got - codes).abs() <= step).all()) and float((got != codes).double().mean()) < 1e-3
            y = got[of, :, place]
        if name == "k":
            y = y * scale[of][..., None]
            for i, least in ((0, True), (1, False)):
                want = over_pages(pages, of, y, "amin" if least else "amax", math.inf if least else -math.inf)
                old = was[2][:, :, i]
                kept = torch.minimum(want, old) if least else torch.maximum(want, old)
                want = torch.where(used[:, None, None], torch.where(begun[:, None, None], want, kept), old)
                assert torch.equal(cache.bounds[:, :, i].double(), want)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("chunk,n,hk", [(64, 2400, 24), (64, 7200, 8), (40, 4700, 8), (24, 2400, 10)])
def test_pages_among_up_to_64_tokens(dim, page, chunk, n, hk):
    append_and_compare(61, BF if dim != 128 else HF, n, 2 * hk if hk == 8 else hk, hk, dim, page, chunk)


@pytest.mark.parametrize("dim,rotary", [(64, 32), (128, 128), (256, 64)])
@pytest.mark.parametrize("chunk,n,hk", [(64, 7200, 8), (48, 6001, 8)])
def test_rotated_pages_among_up_to_64_tokens(dim, rotary, chunk, n, hk):
    """Positions outside of the angles' leave tokens of a run out."""
    append_and_compare(62, BF, n, hk, hk, dim, 32, chunk, rotary)


def test_a_long_prompt():
    """Every place taken, page after page: 16 sequences of 16384 tokens in all."""
    append_and_compare(63, BF, 16384, 8, 8, 128, 64, 64, 128, left_out=False)


# ---------------------------------------------------------------- two tokens of a call in one slot

@pytest.mark.parametrize("dim,page", [(64, 64), (128, 32), (128, 128), (256, 16), (256, 64)])
@pytest.mark.parametrize("first", [0, 3])
def test_two_tokens_in_one_slot_that_two_waves_have(dim, page, first):
    """Runs that all waves of a workgroup share, the same slots twice: elements of either, the first ones and the last ones of a token alike;
    scales and bounds are those of all tokens."""
    g, hk = gen(64), 2
    n = page - first                        # tokens i and n + i go to one slot: another wave's, or another round's
    cache = filled(65, 3, hk, page, dim, True)
    k = randn(g, 2 * n, hk, dim, dtype=BF, scale=2.0)
    slots = (torch.arange(2 * n, device=DEV) % n) + page + first
    want = [ref.Cache(cache.k, cache.k_scale, cache.bounds) for _ in range(2)]
    AttentionSession(hk, hk, dim).append8(cache, k, k, slots)
    torch.cuda.synchronize()
    for w, order in zip(want, (list(range(2 * n)), list(range(n, 2 * n)) + list(range(n)))):
        w.append(k.double().cpu()[order], slots.tolist(), BF)
    got = cache.k.float().double().cpu()
    assert torch.equal(cache.k_scale.double().cpu(), want[0].scale) and torch.equal(cache.bounds.double().cpu(), want[0].bounds)
    assert bool(((got == want[0].codes) | (got == want[1].codes)).all())
    for p in (0, 2):
        assert torch.equal(got[p], want[0].codes[p])
