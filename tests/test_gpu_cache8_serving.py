"""The calls for the cache in 8 bits together, as a program that generates tokens makes them: planned, appended, selected and attended step by step, captured into a
graph, on other streams; and the places where such a program lays its tensors."""
import math
import random

import pytest
import torch

import paper_2507_17511_amd as cf
import cache8_reference as ref
from attention_reference import check
from paper_2507_17511_amd.attention import AttentionSession, PagedCache8, PageTables
from test_gpu_cache8 import BF, DEV, HF, filled, gen, ints, randn

pytestmark = pytest.mark.gpu


def rotation(n, dim):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 100.0 ** -(torch.arange(dim // 2, dtype=torch.float64) / (dim // 2))
    return angle.cos().float().to(DEV), angle.sin().float().to(DEV)


@pytest.mark.parametrize("dtype,page,hq,hk,dim", [(BF, 16, 4, 2, 64), (HF, 32, 6, 2, 128), (BF, 64, 3, 3, 256)])
def test_serving_step_by_step(dtype, page, hq, hk, dim):
    """Prompts of several sequences, then single tokens, some sequences end and others take their pages: what the cache holds is read back after every step,
    and each step's tables, selection and attention are those of the plain evaluation over it."""
    g, r, seqs, count = gen(61), random.Random(61), 5, 6
    tables, cache = PageTables.empty(seqs, 400 // page, 700 // page, page), PagedCache8.empty(700 // page, hk, dim, page)
    s, (cos, sin) = AttentionSession(hq, hk, dim, dtype=dtype), rotation(500, dim)
    state = [[[0] * (400 // page) for _ in range(seqs)], list(range(700 // page)), [0, 700 // page], [0] * seqs]
    held = [[None] * 0 for _ in range(seqs)]           # every sequence's keys and values, as appended
    served = refused = 0
    for step in range(14):
        news = [r.choice([1, 1, 0, r.randrange(1, 120), -1]) if step else r.randrange(1, 150) for _ in range(seqs)]
        total = sum(max(n, 0) for n in news)
        rows = -(-max(total, 1) // 8) * 8
        before = list(state[3])
        plan = s.plan(tables, ints(news), rows)
        want = ref.plan(before, news, state[0], state[1], state[2], page, rows)
        assert (tables.table.tolist(), tables.ring.tolist(), tables.state.tolist(), tables.lens.tolist()) == tuple(want[:4])
        assert (plan.cu.tolist(), plan.slots.tolist(), plan.positions.tolist(), plan.refused.item()) == want[4:]
        state = [want[0], want[1], want[2], want[3]]
        refused += want[7]
        q, k, v = randn(g, rows, hq, dim, dtype=dtype), randn(g, rows, hk, dim, dtype=dtype), randn(g, rows, hk, dim, dtype=dtype)
        turned = s.append8(cache, k, v, plan.slots, plan.positions, cos, sin, q=q)
        torch.cuda.synchronize()
        k64, _ = ref.rotate(k.double().cpu(), cos.cpu()[plan.positions.clamp(min=0).tolist()], sin.cpu()[plan.positions.clamp(min=0).tolist()], dim, False)
        at, last = 0, []
        for b, n in enumerate(news):
            if n < 0:
                held[b] = []
            for t in range(at, at + max(n, 0)):
                if want[5][t] >= 0:
                    served += 1
                    held[b].append((k64[t], v[t].double().cpu()))
            last.append(at + n - 1 if n > 0 and want[5][at + n - 1] >= 0 else None)
            at += max(n, 0)
        # the cache holds every served token, near to what it was
        kk, vv = ref.Cache(cache.k, cache.k_scale, cache.bounds), ref.Cache(cache.v, cache.v_scale)
        for b, tokens in enumerate(held):
            assert len(tokens) == state[3][b]
            for h in range(hk):
                for c, i in ((kk, 0), (vv, 1)):
                    if not tokens:
                        continue
                    got, x = ref.keys_of(c.values(), state[0][b], len(tokens), h), torch.stack([t[i][h] for t in tokens])
                    scale = torch.cat([c.scale[state[0][b][j], h].repeat(page) for j in range(-(-len(tokens) // page))])[:len(tokens), None]
                    # its own rounding, and one of less than a least code's half for each time that the scale has grown: 2^-10 (1 + 1/2 + ...) of it
                    assert bool(((got - x).abs() <= 2.0 ** -4 * 1.001 * x.abs() + 2.0 ** -9 * scale).all())
                    if i == 0:
                        for j in range(-(-len(tokens) // page)):
                            low, high = c.bounds[state[0][b][j], h]
                            some = got[j * page:(j + 1) * page]
                            slack = 2.0 ** -9 * c.scale[state[0][b][j], h]
                            assert bool((some >= low - slack).all()) and bool((some <= high + slack).all())
        # one query of every sequence: of its last new token, or of an older one
        pick = [t if t is not None else 0 for t in last]
        queries = turned[pick].nan_to_num()
        blocks = s.select(cache, queries, tables.table, tables.lens, count, first=1, recent=2)
        out, lse = torch.empty_like(queries), torch.empty(seqs, hq, device=DEV)
        s.paged8(cache, queries, tables.table, tables.lens, out=out, lse=lse)
        some = s.paged8(cache, queries, tables.table, tables.lens, blocks=blocks)
        torch.cuda.synchronize()
        listed = ref.select(queries, cache.bounds, state[0], state[3], page, count, 1, 2)
        assert blocks.tolist() == listed
        o, l, to, tl = ref.attention(queries, kk, vv, state[0], state[3], 1 / math.sqrt(dim))
        check("out", out, o, to)
        check("lse", lse, l, tl)
        o, l, to, tl = ref.attention(queries, kk, vv, state[0], state[3], 1 / math.sqrt(dim), listed)
        check("selected", some, o, to)
    assert served > 300 and refused > 0


def step_of(s, cache, tables, news, x, hq, hk, cos, sin, out):
    plan = s.plan(tables, news, news.numel(), *out[:3], refused=out[3])
    q = s.append8(cache, x[:, hq:hq + hk], x[:, hq + hk:], plan.slots, plan.positions, cos, sin, q=x[:, :hq], q_out=out[4])
    s.select(cache, q, tables.table, tables.lens, 3, out=out[5])
    s.paged8(cache, q, tables.table, tables.lens, blocks=out[5], out=out[6])
    s.paged8(cache, q, tables.table, tables.lens, out=out[7], lse=out[8])


def problem(seed, seqs, hq, hk, dim, page, dtype):
    g = gen(seed)
    lens = [(37 * b) % 300 + 1 for b in range(seqs)]
    pages = seqs * (400 // page + 1)
    tables = PageTables.empty(seqs, 400 // page + 1, pages, page)
    cache = filled(seed, pages, hk, page, dim, True)
    s = AttentionSession(hq, hk, dim, dtype=dtype)
    s.plan(tables, ints(lens), sum(lens))
    out = [torch.empty(seqs, dtype=torch.int64, device=DEV), torch.empty(seqs, dtype=torch.int32, device=DEV), torch.empty(seqs + 1, dtype=torch.int32, device=DEV),
           torch.empty(1, dtype=torch.int32, device=DEV), randn(g, seqs, hq, dim, dtype=dtype), torch.empty((seqs, hk, 3), dtype=torch.int32, device=DEV),
           randn(g, seqs, hq, dim, dtype=dtype), randn(g, seqs, hq, dim, dtype=dtype), torch.empty(seqs, hq, device=DEV)]
    return g, tables, cache, s, out


@pytest.mark.parametrize("dtype,seqs,hq,hk,dim,page", [(BF, 7, 8, 2, 128, 16), (HF, 70, 4, 4, 64, 64)])
def test_a_captured_step_advances_the_state_at_every_replay(dtype, seqs, hq, hk, dim, page):
    """Every replay takes tokens from its input, takes pages, and attends; compared with eager steps of a second program, with work and waits in between.  The
    two captured graphs and the eager calls share nothing but the device."""
    g, tables, cache, s, out = problem(71, seqs, hq, hk, dim, page, dtype)
    _, tables2, cache2, s2, out2 = problem(71, seqs, hq, hk, dim, page, dtype)
    cos, sin = rotation(500, dim)
    news, x = ints([1] * seqs), randn(g, seqs, hq + 2 * hk, dim, dtype=dtype)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step_of(s, cache, tables, news, x, hq, hk, cos, sin, out)
    torch.cuda.synchronize()
    for i in range(40):
        x.copy_(randn(g, seqs, hq + 2 * hk, dim, dtype=dtype, scale=1.0 + 0.2 * i))
        news.copy_(ints([1 if (i + b) % 5 else 0 for b in range(seqs)]))
        graph.replay()
        if i % 3 == 0:
            torch.cuda.synchronize()
            torch.randn(1000, device=DEV).sum()
        step_of(s2, cache2, tables2, news, x, hq, hk, cos, sin, out2)
        torch.cuda.synchronize()
        rows = tables.lens.tolist()
        assert rows == tables2.lens.tolist() and torch.equal(tables.table, tables2.table) and torch.equal(tables.state, tables2.state)
        for a, b in zip(cache.written, cache2.written):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        for a, b in zip(out, out2):
            assert torch.equal(a, b)


def test_other_streams_than_the_current_one():
    hq, hk, dim, page, seqs = 4, 2, 128, 16, 9
    g, tables, cache, _, out = problem(81, seqs, hq, hk, dim, page, BF)
    _, tables2, cache2, s2, out2 = problem(81, seqs, hq, hk, dim, page, BF)
    cos, sin = rotation(500, dim)
    stream = torch.cuda.Stream()
    s = AttentionSession(hq, hk, dim, stream=stream)
    stream.wait_stream(torch.cuda.current_stream())
    for i in range(5):
        x, news = randn(g, seqs, hq + 2 * hk, dim), ints([1] * seqs)
        stream.wait_stream(torch.cuda.current_stream())
        step_of(s, cache, tables, news, x, hq, hk, cos, sin, out)
        step_of(s2, cache2, tables2, news, x, hq, hk, cos, sin, out2)
        stream.synchronize()
        torch.cuda.synchronize()
        for a, b in zip(out, out2):
            assert torch.equal(a, b)


def test_pages_between_one_another_strides_and_slices():
    """k and v as halves of one tensor's pages, layers of one tensor; a table that is a slice of a wider one; queries and outputs that are slices, head by head."""
    g, hq, hk, dim, page, pages = gen(91), 6, 2, 128, 32, 30
    base = filled(92, pages, hk, page, dim, True)
    wide = torch.zeros((pages, 3, 2, hk, page, dim), dtype=torch.float8_e4m3fn, device=DEV)
    wide.view(torch.uint8)[:, 1, 0], wide.view(torch.uint8)[:, 1, 1] = base.k.view(torch.uint8), base.v.view(torch.uint8)
    cache = PagedCache8(wide[:, 1, 0], wide[:, 1, 1], base.k_scale.clone(), base.v_scale.clone(), base.bounds.clone())
    s = AttentionSession(hq, hk, dim)
    lens = [300, 7, 33]
    rows = [random.Random(b).sample(range(pages), 10) for b in range(3)]
    table = torch.full((3, 17), 5, dtype=torch.int32, device=DEV)
    table[:, 3:13] = ints(rows)
    q = randn(g, 3, hq + 2 * hk, dim + 8)[:, :hq, :dim]
    plain = q.contiguous()
    out = torch.full((hq, 3, dim), 7.0, dtype=BF, device=DEV)
    blocks = s.select(cache, q, table[:, 3:13], ints(lens), 4)
    s.paged8(cache, q, table[:, 3:13], ints(lens), blocks=blocks, out=out.transpose(0, 1))
    want = s.paged8(base, plain, ints(rows), ints(lens), blocks=s.select(base, plain, ints(rows), ints(lens), 4))
    torch.cuda.synchronize()
    assert torch.equal(out.transpose(0, 1), want)
    k, v, slots = randn(g, 70, hk, dim), randn(g, 70, hk, dim), torch.arange(70, device=DEV) + 40
    s.append8(cache, k, v, slots)
    s.append8(base, k, v, slots)
    torch.cuda.synchronize()
    for a, b in zip(cache.written, base.written):
        assert torch.equal(a.contiguous().view(torch.uint8), b.view(torch.uint8))
    assert not bool(wide.view(torch.uint8)[:, ::2].any())


def test_offsets_past_32_bits():
    """Pages whose codes, scales and bounds lie past 4 GiB."""
    hk, dim, page, pages = 16, 256, 128, 20000                 # 10 GiB each of keys and values
    k, v = (torch.empty((pages, hk, page, dim), dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    cache = PagedCache8(k, v, torch.ones((pages, hk), device=DEV), torch.ones((pages, hk), device=DEV), torch.empty((pages, hk, 2, dim), dtype=BF, device=DEV))
    g, s = gen(93), AttentionSession(hk, hk, dim)
    lens, rows = [300, 130], [[19999, 12345, 8191], [8193, 16385, 0]]
    slots = torch.tensor([rows[b][i // page] * page + i % page for b in range(2) for i in range(lens[b])], device=DEV)
    x, y = randn(g, sum(lens), hk, dim), randn(g, sum(lens), hk, dim)
    q = randn(g, 2, hk, dim)
    s.append8(cache, x, y, slots)
    blocks = s.select(cache, q, ints(rows), ints(lens), 2, first=0, recent=1)
    out, lse = torch.empty_like(q), torch.empty(2, hk, device=DEV)
    s.paged8(cache, q, ints(rows), ints(lens), out=out, lse=lse)
    torch.cuda.synchronize()
    used = sorted({p for row in rows for p in row})
    small = [[used.index(p) for p in row] for row in rows]
    kk, vv = ref.Cache(k[used], cache.k_scale[used], cache.bounds[used]), ref.Cache(v[used], cache.v_scale[used])
    for b, at in ((0, 0), (1, 300)):
        for h in range(hk):
            got = ref.keys_of(kk.values(), small[b], lens[b], h)
            assert bool(((got - x[at:at + lens[b], h].double().cpu()).abs() <= 2.0 ** -4 * got.abs() * 1.1 + 2.0 ** -9 * 0.1).all())
    o, l, to, tl = ref.attention(q, kk, vv, small, lens, 1 / 16)
    check("out", out, o, to)
    check("lse", lse, l, tl)
    assert blocks.tolist() == ref.select(q, cache.bounds[used], small, lens, page, 2, 0, 1)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_nan_and_largest_values_stay_with_their_rows(dtype, dim):
    """A NaN key, a NaN query, the largest values that a type holds: rows that do not see them are what they are without."""
    g, hk, page, pages, lens = gen(94), 2, 16, 40, [200, 90, 33]
    cache = filled(95, pages, hk, page, dim, True)
    rows = [list(range(0, 13)), list(range(13, 19)), list(range(19, 22))]
    table = ints([row + [0] * (13 - len(row)) for row in rows])
    q = randn(g, 3, 4, dim, dtype=dtype)
    s = AttentionSession(4, hk, dim, dtype=dtype)
    plain = s.paged8(cache, q, table, ints(lens))
    o, _, to, _ = ref.attention(q, ref.Cache(cache.k, cache.k_scale), ref.Cache(cache.v, cache.v_scale), rows, lens, 1 / math.sqrt(dim))
    for what in ("key", "query", "value"):
        changed, q2 = PagedCache8(*[x.clone() for x in cache.written]), q.clone()
        if what == "key":
            changed.k.view(torch.uint8)[2, 0, 3, 5] = 0x7f
        elif what == "query":
            q2[0, 1, 3] = math.nan
        else:
            changed.v.view(torch.uint8)[2, 0, 3, 5] = 0x7f
        got = s.paged8(changed, q2, table, ints(lens))
        torch.cuda.synchronize()
        assert torch.equal(got[1:], plain[1:]) and torch.equal(got[0, 2:], plain[0, 2:]) and bool(got[0, 1].isnan().any())
        if what == "query":                 # heads that share keys share what their weights are relative to, and no more
            check("the other head", got[0, 0], o[0, 0], to[0, 0])
        if what == "value":
            assert bool(got[0, 0, 5].isnan()) and not bool(got[0, 0, :5].isnan().any())


def test_fp16_keys_that_weigh_little_each_and_much_together():
    """A first key leads by 12 in the exponent, 20000 others weigh e^-12 each: together a tenth.  Their weights are below fp16's normal numbers."""
    n, dim, page = 20001, 64, 64
    k, v = torch.zeros(n, 1, dim, device=DEV, dtype=HF), torch.ones(n, 1, dim, device=DEV, dtype=HF)
    q = torch.zeros(1, 1, dim, device=DEV, dtype=HF)
    q[..., 0], k[0, 0, 0], v[0] = 8.0, 12.0, 0.0                # scores 12 and 0, at a scale of 1/8
    pages = -(-n // page)
    cache, s = PagedCache8.empty(pages, 1, dim, page), AttentionSession(1, 1, dim, dtype=HF)
    s.append8(cache, k, v, torch.arange(n, device=DEV))
    out = s.paged8(cache, q, torch.arange(pages, dtype=torch.int32, device=DEV)[None], ints([n]))
    want = 20000 * math.exp(-12) / (1 + 20000 * math.exp(-12))
    # every weight rounded by 2^-11 of it, or the sums of 64 off by 2^-8 of the least that counts; the output once
    assert float((out.double() - want).abs().max()) <= want * (2.0 ** -8 + 2 * 2.0 ** -11)


def test_rows_behind_the_last_sequence_stay():
    """Outputs are written for the call's sequences alone, lists for its heads alone."""
    s, cache = AttentionSession(4, 2, 64), filled(96, 9, 2, 16, 64, True)
    q, table, lens = randn(gen(97), 3, 4, 64), ints([[1, 2], [3, 4], [5, 6]]), ints([20, 0, 32])
    out, lse, blocks = torch.full((5, 4, 64), 7.0, dtype=BF, device=DEV), torch.full((5, 4), 7.0, device=DEV), torch.full((5, 2, 3), 7, dtype=torch.int32, device=DEV)
    s.paged8(cache, q, table, lens, out=out[:3], lse=lse[:3])
    s.select(cache, q, table, lens, 3, out=blocks[:3])
    torch.cuda.synchronize()
    assert bool((out[3:] == 7).all()) and bool((lse[3:] == 7).all()) and bool((blocks[3:] == 7).all())
    assert not bool(out[1].any()) and bool((lse[1] == -math.inf).all()) and bool((blocks[1] == -1).all()) and blocks[0].tolist() == [[0, 1, -1]] * 2
