"""Serving from a cache in 8 bits against a plain evaluation in 64 bits: codes and scales as tokens are appended, attention over them, the pages that a
score selects, and the plan of a step."""
import math
import random

import pytest
import torch

import paper_2507_17511_amd as cf
import cache8_reference as ref
from attention_reference import check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache8, PageTables

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=BF, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


def filled(seed, pages, heads, page, dim, bounds=False, spread=2.0):
    """A cache in use: codes of any size that are numbers, scales of several powers of two, up to 2^7: fp16 holds 448 times that."""
    g = gen(seed)
    k, v = ((torch.randn((pages, heads, page, dim), generator=g, device=DEV) * 60).clamp(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.exp2((torch.round(torch.randn((pages, heads), generator=g, device=DEV) * spread) - 6).clamp(max=7)) for _ in range(2))
    b = None
    if bounds:
        x = k.float() * ks[..., None, None]
        b = torch.stack((x.amin(2), x.amax(2)), 2).to(BF)
    return PagedCache8(k, v, ks, vs, b)


# ---------------------------------------------------------------- codes

def test_codes_of_all_numbers_are_those_of_the_format():
    """Every finite bf16 number between 2^-12 and 448, and every fp16 number: rounded as the format says, ties to even."""
    for dtype in (BF, HF):
        x = torch.arange(65536, dtype=torch.int32).to(torch.uint16).view(dtype) if hasattr(torch, "uint16") else None
        x = x[x.isfinite() & (x.abs() <= 448)].to(DEV)
        x = x[:x.numel() // 1024 * 1024]
        page, dim = 128, 64
        n = x.numel() // (dim * 4) // page * page                # tokens of 4 heads
        k = x[:n * 4 * dim].view(n, 4, dim).clone()
        k[::page, :, 0] = 448.0                                  # every page's scale is 1
        for h in range(4):
            k[::page, h, 0] = 448.0
        cache = PagedCache8.empty(n // page, 4, dim, page_size=page)
        AttentionSession(4, 4, dim, dtype=dtype).append8(cache, k, k, torch.arange(n, device=DEV))
        torch.cuda.synchronize()
        assert bool((cache.k_scale == 1).all()) and bool((cache.v_scale == 1).all())
        got = cache.k.float().permute(0, 2, 1, 3).reshape(n, 4, dim).cpu()
        want = k.float().cpu().to(torch.float8_e4m3fn).float()
        assert torch.equal(got, want) and torch.equal(got.double(), ref.e4m3(k.double().cpu()))
        assert torch.equal(cache.v.view(torch.uint8), cache.k.view(torch.uint8))


def append_and_compare(seed, dtype, hq, hk, dim, page, runs, rotary=0, interleaved=False, bounds=True, scale=1.0, packed=False, shuffle=True):
    """runs: (place on a page where the tokens begin, how many) of each sequence; what was before is random.  Compares everything."""
    g, r = gen(seed), random.Random(seed)
    per = [-(-(at + n) // page) for at, n in runs]
    pages = sum(per) + 2
    order = list(range(pages))
    if shuffle:
        r.shuffle(order)
    slots, positions, first = [], [], 0
    for (at, n), p in zip(runs, per):
        slots += [order[first + (at + i) // page] * page + (at + i) % page for i in range(n)]
        positions += [at + i for i in range(n)]
        first += p
    n = len(slots)
    if packed:
        x = randn(g, n, hq + 2 * hk, dim, dtype=dtype, scale=scale)
        q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
    else:
        q, k, v = randn(g, n, hq, dim, dtype=dtype, scale=scale), randn(g, n, hk, dim, dtype=dtype, scale=scale), randn(g, n, hk, dim, dtype=dtype, scale=scale)
    cache = filled(seed + 1, pages, hk, page, dim, bounds)
    want_k, want_v = ref.Cache(cache.k, cache.k_scale, cache.bounds), ref.Cache(cache.v, cache.v_scale)
    angle = torch.arange(max(positions) + 1, dtype=torch.float64)[:, None] * 100.0 ** -(torch.arange(max(rotary // 2, 1), dtype=torch.float64) / max(rotary // 2, 1))
    cos, sin = angle.cos().float(), angle.sin().float()
    s = AttentionSession(hq, hk, dim, dtype=dtype)
    kw = dict(positions=ints(positions), cos=cos.to(DEV), sin=sin.to(DEV), interleaved=interleaved) if rotary else {}
    out = s.append8(cache, k, v, ints(slots, torch.int64), q=q, **kw)
    torch.cuda.synchronize()
    turned = [ref.rotate(x.double().cpu(), cos[positions], sin[positions], rotary, interleaved) if rotary else (x.double().cpu(), x.double().abs().cpu()) for x in (q, k)]
    want_k.append(turned[1][0], slots, dtype)
    want_v.append(v.double().cpu(), slots, dtype)
    u = {BF: 2.0 ** -8, HF: 2.0 ** -11}[dtype]
    check("q", out, turned[0][0], 1.01 * u * turned[0][0].abs() + 2.0 ** -23 * turned[0][1] + 2.0 ** -25)
    # scales are the same but where a largest magnitude lies next to a border, which these inputs do not
    assert torch.equal(cache.k_scale.double().cpu(), want_k.scale) and torch.equal(cache.v_scale.double().cpu(), want_v.scale)
    assert torch.equal(cache.v.float().double().cpu(), want_v.codes)        # not rotated: exact
    got = cache.k.float().double().cpu()
    if not rotary:
        assert torch.equal(got, want_k.codes)
        if bounds:
            assert torch.equal(cache.bounds.double().cpu(), want_k.bounds)
        return
    # rotated: rounding goes the other way only next to a tie
    differ = got != want_k.codes
    step = torch.exp2(torch.floor(torch.log2(want_k.codes.abs().clamp(min=2.0 ** -6))) - 3)
    assert bool(((got - want_k.codes).abs() <= step).all()) and float(differ.double().mean()) < 1e-3
    if bounds:
        check("bounds", cache.bounds, want_k.bounds, 0.126 * want_k.bounds.abs() + 2.0 ** -9 * want_k.scale[:, :, None, None] if bool(differ.any()) else torch.zeros_like(want_k.bounds))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_types_dimensions_and_pages(dtype, dim, page):
    append_and_compare(1, dtype, 4, 2, dim, page, [(0, 1), (3, 1), (0, page), (page - 1, 2), (5, 2 * page + 1), (0, 3 * page)])


@pytest.mark.parametrize("rotary,interleaved", [(16, False), (64, False), (128, False), (16, True), (64, True), (128, True)])
@pytest.mark.parametrize("packed", [True, False])
def test_append_rotations(rotary, interleaved, packed):
    append_and_compare(2, BF, 6, 3, 128, 32, [(0, 7), (30, 40), (0, 65)], rotary, interleaved, packed=packed)
    append_and_compare(3, HF, 3, 3, 256, 16, [(0, 7), (9, 40)], rotary, interleaved, packed=packed)


@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 1), (10, 10)])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_append_of_many_tokens(hq, hk, page):
    """Past 32768 (token, head) rows a workgroup takes the pages of 16 tokens."""
    many = 32768 // (2 * hk) + 100
    rest = many - 16 * 40
    append_and_compare(4, BF, hq, hk, 64, page, [(i % page, 16) for i in range(40)] + [(page // 2 + 1, rest)], 16)


@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-4, 100.0, 3e4])
def test_append_magnitudes(scale):
    """Scales grow on pages that are in use (their codes are rounded again), or stay; zeros take the least."""
    append_and_compare(5, BF, 2, 2, 128, 32, [(0, 3), (3, 1), (17, 30), (0, 70)], scale=scale)
    if scale <= 100.0:
        append_and_compare(6, HF, 2, 2, 64, 16, [(0, 3), (3, 1), (7, 30)], scale=scale)


def test_append_one_token_after_another():
    """A page filled by single tokens of growing size: as the reference does it, and near to the tokens."""
    g, page, dim = gen(7), 32, 128
    cache = PagedCache8.empty(2, 1, dim, page_size=page)
    want = ref.Cache(cache.k, cache.k_scale, cache.bounds)
    s = AttentionSession(1, 1, dim)
    x = randn(g, page, 1, dim) * torch.exp2(torch.arange(page, device=DEV)[:, None, None] * 0.5).to(BF)
    for i in range(page):
        s.append8(cache, x[i:i + 1], x[i:i + 1], ints([page + i], torch.int64))
        want.append(x[i:i + 1].double().cpu(), [page + i], BF)
        torch.cuda.synchronize()
        assert torch.equal(cache.k_scale.double().cpu()[1], want.scale[1])
        assert torch.equal(cache.k[1, :, :i + 1].float().double().cpu(), want.codes[1, :, :i + 1])
        assert torch.equal(cache.bounds[1].double().cpu(), want.bounds[1])
    got = cache.k[1, 0].float().double() * cache.k_scale[1, 0].double()
    # every step up rounds by half a least step of the scale at most, 2^-10 of it: 17 of them, of scales that double
    off = (got - x[:, 0].double()).abs()
    assert bool((off <= 2.0 ** -4 * x[:, 0].double().abs() + 2 * 2.0 ** -10 * cache.k_scale[1, 0].double()).all())


@pytest.mark.parametrize("dtype", [BF, HF])
def test_append_infinities_and_nan(dtype):
    g, dim = gen(8), 64
    k = randn(g, 20, 1, dim, dtype=dtype)
    k[2, 0, 3], k[3, 0, 4], k[5, 0, 6], k[17, 0, 1] = math.inf, -math.inf, math.nan, math.nan
    cache = PagedCache8.empty(2, 1, dim, page_size=16)
    want = ref.Cache(cache.k, cache.k_scale, cache.bounds)
    AttentionSession(1, 1, dim, dtype=dtype).append8(cache, k, k, torch.arange(20, device=DEV))
    want.append(k.double().cpu(), list(range(20)), dtype)
    torch.cuda.synchronize()
    got = cache.k.float().double().cpu()[0], want.codes[0]
    assert torch.equal(got[0].isnan(), got[1].isnan()) and torch.equal(got[0].nan_to_num(nan=0.0), got[1].nan_to_num(nan=0.0))
    assert torch.equal(cache.k_scale.double().cpu(), want.scale) and torch.equal(cache.bounds.double().cpu(), want.bounds)
    assert float(got[0][0, 2, 3]) * float(want.scale[0, 0]) == ref.MOST_VALUE[dtype] and bool(cache.bounds.isfinite().all())


def test_append_leaves_out_tokens_and_places():
    """Slots outside the cache, positions outside the table; nothing else of the cache changes."""
    g, page, dim = gen(9), 16, 128
    cache = filled(10, 5, 2, page, dim, True)
    before = [x.view(torch.uint8).clone() for x in cache.written]
    k, q = randn(g, 12, 2, dim), randn(g, 12, 4, dim)
    slots = [-1, 33, 34, 35, -7, 5 * page, 10 ** 15, 49, 50, -1, -1, 70]
    positions = [0, 1, 99, 2, 3, 3, 3, -5, 1 << 30, 3, 3, 100]
    angle = torch.ones(5, dim // 2, device=DEV)
    out = torch.full_like(q, 7.0)
    want = ref.Cache(cache.k, cache.k_scale, cache.bounds)
    AttentionSession(4, 2, dim).append8(cache, k, k, ints(slots, torch.int64), positions=ints(positions), cos=angle * 0.5, sin=angle * 0.0, q=q, q_out=out)
    torch.cuda.synchronize()
    want.append(k.double().cpu() * 0.5, [s if 0 <= p < 5 else None for s, p in zip(slots, positions)], BF)
    assert torch.equal(cache.k.float().double().cpu(), want.codes) and torch.equal(cache.bounds.double().cpu(), want.bounds)
    stay = [t for t, p in enumerate(positions) if not 0 <= p < 5]
    assert bool((out[stay] == 7).all()) and torch.equal(out[[0, 1, 3]], (q[[0, 1, 3]].float() * 0.5).to(BF))
    for now, was in zip(cache.written, before):
        now = now.view(torch.uint8)
        assert all(torch.equal(now[p], was[p]) for p in (0, 1, 3, 4))
    assert not torch.equal(cache.k[2].view(torch.uint8), before[0][2])


@pytest.mark.parametrize("first", [0, 5])
def test_append_two_tokens_into_one_slot(first):
    """The place holds elements of either; scales and bounds are of both, and of the neighbour behind them."""
    g, page, dim = gen(19), 16, 128
    cache = filled(20, 3, 2, page, dim, True)
    k = randn(g, 3, 2, dim)
    want = [ref.Cache(cache.k, cache.k_scale, cache.bounds) for _ in range(2)]
    AttentionSession(2, 2, dim).append8(cache, k, k, ints([page + first, page + first, page + first + 1], torch.int64))
    torch.cuda.synchronize()
    for w, order in zip(want, ([0, 1, 2], [1, 0, 2])):
        w.append(k.double().cpu()[order], [page + first, page + first, page + first + 1], BF)
    got = cache.k.float().double().cpu()
    assert torch.equal(cache.k_scale.double().cpu(), want[0].scale) and torch.equal(cache.bounds.double().cpu(), want[0].bounds)
    assert bool(((got == want[0].codes) | (got == want[1].codes)).all())


def test_append_queries_in_place_without_and_alone():
    g = gen(11)
    q, k = randn(g, 9, 4, 64), randn(g, 9, 2, 64)
    cache = PagedCache8.empty(1, 2, 64, page_size=16, bounds=False)
    s, kw = AttentionSession(4, 2, 64), dict(positions=ints(range(9)), cos=torch.full((9, 32), 0.6, device=DEV), sin=torch.full((9, 32), 0.8, device=DEV))
    want = s.append8(cache, k, k, torch.arange(9, device=DEV), q=q, **kw)
    first = cache.k.view(torch.uint8).clone()
    assert s.append8(cache, k, k, torch.arange(9, device=DEV), q=q, q_out=q, **kw) is q and torch.equal(q, want)
    assert s.append8(cache, k, k, torch.arange(9, device=DEV), **kw) is None
    assert torch.equal(cache.k.view(torch.uint8)[:, :, :9], first[:, :, :9])


# ---------------------------------------------------------------- attention

def run_paged8(seed, dtype, hq, hk, dim, page, lens, max_len=0, blocks=None, workspace_bytes=cf.CF_ATTN_WORKSPACE_BYTES, cache=None, spread=2.0, scale=0.0):
    g, r = gen(seed), random.Random(seed)
    per = [max(1, -(-n // page)) for n in lens]
    pages = sum(per) + 2
    cache = filled(seed + 1, pages, hk, page, dim, spread=spread) if cache is None else cache
    order = list(range(pages))
    r.shuffle(order)
    rows, at = [], 0
    for p in per:
        rows.append(order[at:at + p])
        at += p
    cols = max(per)
    table = ints([row + [10 ** 9] * (cols - len(row)) for row in rows])
    q = randn(g, len(lens), hq, dim, dtype=dtype)
    # what lies behind a context's last token does not count, whatever it is
    for row, n in zip(rows, lens):
        if n % page or n == 0:
            for c in (cache.k, cache.v):
                c.view(torch.uint8)[row[-1], :, n % page:] = 0x7f
    s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace_bytes, scale=scale)
    out, lse = torch.full(q.shape, 7.0, dtype=dtype, device=DEV), torch.full(q.shape[:2], 7.0, device=DEV)
    listed = None
    if blocks is not None:
        blocks = blocks(r, [-(-n // page) for n in lens], hk)
        listed = ints(blocks)
    s.paged8(cache, q, table, ints(lens), blocks=listed, out=out, lse=lse, max_len=max_len)
    torch.cuda.synchronize()
    k, v = ref.Cache(cache.k, cache.k_scale), ref.Cache(cache.v, cache.v_scale)
    o, l, to, tl = ref.attention(q, k, v, rows, lens, scale or 1 / math.sqrt(dim), blocks)
    check("out", out, o, to)
    check("lse", lse, l, tl)
    again = s.paged8(cache, q, table, ints(lens), blocks=listed, max_len=max_len)
    assert torch.equal(again, out)
    if s.workspace is not None:
        assert not bool(s.workspace[:cf.CF_ATTN_COUNTER_BYTES].any())


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 1), (6, 2), (17, 1), (40, 1)])
@pytest.mark.parametrize("page", [16, 64])
def test_paged8_types_heads_and_dimensions(dtype, dim, hq, hk, page):
    run_paged8(21, dtype, hq, hk, dim, page, [1, 37, 130, 700])


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens", [[0], [1], [15, 16, 17], [31, 32, 33, 0], [63, 64, 65], [127, 128, 129], [255, 256, 257, 0, 1], [3000]])
def test_paged8_lengths(page, dim, lens):
    run_paged8(22, BF, 4, 2, dim, page, lens)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lens,max_len", [([5000], 0), ([9000, 1, 300], 9000), ([9000, 1, 300], 40), ([700] * 70, 0), ([0, 6000, 10] * 20, 0)])
def test_paged8_split_contexts(dim, lens, max_len):
    for bytes_ in (cf.CF_ATTN_WORKSPACE_BYTES, 0, cf.CF_ATTN_COUNTER_BYTES + 2 * len(lens) * 4 * (dim + 1) * 4 // 256 * 256 + 256):
        run_paged8(23, BF, 4, 2, dim, 32, lens, max_len=max_len, workspace_bytes=bytes_)


def test_paged8_many_sequences():
    run_paged8(24, BF, 2, 1, 64, 16, [1 + i % 40 for i in range(2500)])
    run_paged8(25, BF, 1, 1, 64, 128, [1 + i % 9 for i in range(2099)] + [20000])


@pytest.mark.parametrize("dtype", [BF, HF])
def test_paged8_scales_that_differ_widely(dtype):
    run_paged8(26, dtype, 4, 2, 128, 16, [300, 40], spread=5.0)
    run_paged8(27, dtype, 4, 2, 128, 64, [300, 40], spread=0.0, scale=0.5)


def lists(count, holes=False, twice=False):
    def make(r, held, hk):
        got = []
        for n in held:
            got.append([])
            for _ in range(hk):
                some = sorted(r.sample(range(n), min(n, count)))
                if twice and some:
                    some[-1] = some[0]
                some += [-1] * (count - len(some))
                if holes:
                    some = [x if r.random() < 0.7 else r.choice([-1, -5, n, 10 ** 9]) for x in some]
                    r.shuffle(some)
                got[-1].append(some)
        return got
    return make


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("count", [1, 3, 20])
def test_paged8_listed_pages(page, dim, count):
    run_paged8(28, BF, 6, 2, dim, page, [1, page, page + 1, 9 * page - 3, 0, 40 * page + 7], blocks=lists(count))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("page", [16, 64])
def test_paged8_lists_in_any_order_with_entries_outside(dtype, page):
    run_paged8(29, dtype, 4, 2, 128, page, [page * 30 + 5, 3, 0, page * 7], blocks=lists(12, holes=True))
    run_paged8(30, dtype, 4, 2, 128, page, [page * 30 + 5, 3, page * 7], blocks=lists(12, twice=True))
    run_paged8(31, dtype, 4, 2, 128, page, [page * 30 + 5, 3], blocks=lambda r, held, hk: [[[-1] * 4] * hk] * 2)


@pytest.mark.parametrize("page,count", [(16, 300), (64, 100), (128, 60)])
def test_paged8_long_lists_are_split(page, count):
    run_paged8(32, BF, 4, 2, 128, page, [page * 400 + 3, page * count, 5], blocks=lists(count))
    run_paged8(33, BF, 4, 2, 128, page, [page * 120 + 3] * 40, blocks=lists(count, holes=True))


# ---------------------------------------------------------------- pages by score

def run_select(seed, dtype, hq, hk, dim, page, lens, count, first=1, recent=1, max_len=0, workspace_bytes=cf.CF_ATTN_WORKSPACE_BYTES, change=None, pages=None):
    g, r = gen(seed), random.Random(seed)
    per = [max(1, -(-n // page)) for n in lens]
    pages = pages or sum(per) + 2
    bounds = torch.stack((randn(g, pages, hk, dim) - 1, randn(g, pages, hk, dim) + 1), 2)
    bounds = torch.stack((bounds.amin(2), bounds.amax(2)), 2)
    q = randn(g, len(lens), hq, dim, dtype=dtype)
    if change is not None:
        change(q, bounds)
    empty = torch.zeros((pages, hk, page, dim), dtype=torch.float8_e4m3fn, device=DEV)
    cache = PagedCache8(empty, empty.clone(), *torch.ones((2, pages, hk), device=DEV), bounds)
    rows = [[r.randrange(pages) for _ in range(p)] for p in per]
    table = ints([row + [-3] * (max(per) - len(row)) for row in rows])
    s = AttentionSession(hq, hk, dim, dtype=dtype, workspace_bytes=workspace_bytes)
    got = s.select(cache, q, table, ints(lens), count, first=first, recent=recent, max_len=max_len)
    torch.cuda.synchronize()
    want = ref.select(q, bounds, rows, lens, page, count, first, recent)
    assert got.cpu().tolist() == want
    assert torch.equal(s.select(cache, q, table, ints(lens), count, first=first, recent=recent, max_len=max_len), got)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("hq,hk", [(1, 1), (6, 2), (40, 1)])
def test_select_types_heads_and_dimensions(dtype, dim, hq, hk):
    run_select(41, dtype, hq, hk, dim, 16, [1, 37, 130, 700, 16 * 300], 9)


@pytest.mark.parametrize("lens", [[0], [1], [64 * 5], [64 * 5 + 1], [64 * 63, 64 * 64, 64 * 65], [64 * 1023, 64 * 1024 + 1, 64 * 2100]])
@pytest.mark.parametrize("count,first,recent", [(1, 0, 0), (1, 1, 0), (5, 0, 1), (5, 2, 3), (64, 1, 1), (1500, 3, 4)])
def test_select_lengths_and_counts(lens, count, first, recent):
    run_select(42, BF, 4, 2, 64, 64, lens, count, first, recent)


def test_select_takes_the_earlier_of_equal_scores():
    def zero(q, bounds):
        q.zero_()
    def few(q, bounds):
        bounds.copy_(torch.round(bounds))
        q.copy_(torch.round(q))
    def signs(q, bounds):       # scores on both sides of zero, some of them -0
        bounds[::3] *= -1
        bounds.copy_(torch.stack((bounds.amin(2), bounds.amax(2)), 2))
        bounds[1::5] = 0
        bounds[1::5, :, 0] *= -1
    for change in (zero, few, signs):
        run_select(43, BF, 4, 2, 64, 16, [16 * 900, 16 * 3000, 100], 50, change=change, pages=20)
        run_select(44, BF, 4, 2, 64, 16, [16 * 900, 16 * 3000, 100], 50, change=change)


def test_select_numbers_that_differ_widely_and_nan():
    def wide(q, bounds):
        bounds.mul_(torch.exp2(torch.round(6 * torch.randn(bounds.shape[:1], generator=gen(1), device=DEV)))[:, None, None, None].to(BF))
    def nan(q, bounds):
        bounds[::7, :, 1, 5] = math.nan
        q[0, 0, 3] = math.nan
    run_select(45, BF, 4, 2, 128, 16, [16 * 900, 16 * 1300, 100], 50, change=wide)
    run_select(46, BF, 4, 2, 128, 16, [16 * 900, 16 * 1300, 100], 50, change=nan)


def test_select_workspaces_and_hints():
    lens, rows = [16 * 900, 16 * 1300, 100, 16 * 60], 8
    for fit in (1, 3, 7):
        run_select(47, BF, 4, 2, 64, 16, lens, 20, workspace_bytes=cf.CF_ATTN_COUNTER_BYTES + fit * 1300 * 8)
    for max_len in (1, 2000, 16 * 1300, 10 ** 7):
        run_select(48, BF, 4, 2, 64, 16, lens, 20, max_len=max_len)


# ---------------------------------------------------------------- plans

def run_plan(lens, news, page, max_pages, ring, taken, free, tokens, seed=1, in_place=True, workspace_bytes=1 << 20, stride=0):
    r = random.Random(seed)
    pages = list(range(ring))
    r.shuffle(pages)
    table = [[pages[r.randrange(ring)] for _ in range(max_pages)] for _ in lens]
    slots = list(pages)
    want = ref.plan(lens, news, table, slots, (taken, taken + free), page, tokens)
    wide = torch.full((len(lens), max_pages + stride), -9, dtype=torch.int32, device=DEV)
    wide[:, :max_pages] = torch.tensor(table, dtype=torch.int32).view(len(lens), max_pages).to(DEV)
    t = PageTables(wide[:, :max_pages], ints(lens), ints(slots), ints([taken, taken + free], torch.int64), page)
    s = AttentionSession(1, 1, 64, workspace_bytes=workspace_bytes)
    lens_out, state_out = (None, None) if in_place else (torch.empty_like(t.lens), torch.empty_like(t.state))
    plan = s.plan(t, ints(news), tokens, lens_out=lens_out, state_out=state_out)
    torch.cuda.synchronize()
    if not in_place:
        assert t.lens.tolist() == lens and t.state.tolist() == [taken, taken + free]
    got = (t.table.tolist(), t.ring.tolist(), (t.state if in_place else state_out).tolist(), (t.lens if in_place else lens_out).tolist(), plan.cu.tolist(),
           plan.slots.tolist(), plan.positions.tolist(), plan.refused.item())
    for name, x, y in zip(("table", "ring", "state", "lens", "cu", "slots", "positions", "refused"), got, want):
        assert x == y, name
    assert bool((wide[:, max_pages:] == -9).all())
    if workspace_bytes:
        assert not bool(s.workspace.any())


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("workspace_bytes", [0, 1 << 20])
@pytest.mark.parametrize("lens,news,tokens", [([], [], 5), ([0], [0], 0), ([0], [1], 1), ([16], [1], 4), ([5, 0, 31, 32, 40], [1, 40, 1, 1, -1], 64), ([5, 0, 31], [1, 40, 1], 41),
                                              ([3, 9], [-1, -1], 3), ([100, 159, 160], [60, 1, 1], 70)])
def test_plan_small(in_place, workspace_bytes, lens, news, tokens):
    run_plan(lens, news, 16, 10, 40, 100, 12, tokens, in_place=in_place, workspace_bytes=workspace_bytes)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("free", [0, 40, 400, 6000])
def test_plan_many_sequences(seed, free):
    """More sequences than a workgroup has threads, more tokens than one takes; pages that run short; a ring that wraps."""
    r = random.Random(seed)
    n = r.choice([3, 700, 1024, 1025, 2600])
    lens = [r.choice([0, r.randrange(300), r.randrange(3000)]) for _ in range(n)]
    news = [r.choice([1, 1, 1, 0, -1, r.randrange(40), 900 if r.random() < 0.03 else 1]) for _ in range(n)]
    total = sum(max(x, 0) for x in news)
    for tokens, in_place in ((total, True), (total + 5000, False), (total * 2 // 3, True)):
        run_plan(lens, news, r.choice([16, 64]), 250, 7000 + free, r.choice([0, 12345, 10 ** 12]), free, tokens, seed, in_place, stride=r.choice([0, 3]))


def test_plan_senseless_numbers_stay_inside():
    """Lengths below zero or past the table, a ring that says it holds more than it has, or less than nothing."""
    t = PageTables(ints([[1] * 4] * 5), ints([-5, 10 ** 9, 64, 3, 3]), ints([7] * 6), ints([50, 10 ** 17], torch.int64), 16)
    s = AttentionSession(1, 1, 64)
    p = s.plan(t, ints([3, 3, 1, 2 ** 31 - 1, 20]), 40)
    assert p.refused.item() == 5 and t.lens.tolist() == [-5, 10 ** 9, 64, 3, 3] and p.slots.tolist() == [-1] * 40 and p.cu.tolist() == [0, 3, 6, 7, 40, 40]
    t = PageTables(ints([[1] * 4] * 2), ints([3, 20]), ints([7] * 6), ints([50, 3], torch.int64), 16)
    p = s.plan(t, ints([20, -1]), 40)
    assert p.refused.item() == 1 and p.slots.tolist() == [-1] * 40 and t.state.tolist() == [50, 52] and t.lens.tolist() == [3, 0]
