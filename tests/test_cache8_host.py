"""What the entry points for the cache in 8 bits refuse, on the host and before any device work; what their session checks of tensors, that what they write counts
as changed, and that they run on the session's device.  Needs no GPU."""
import types

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd import attention
from paper_2507_17511_amd.attention import AttentionSession, PagedCache8, PageTables
from test_attention_devices_host import Tensor, machine  # noqa: F401
from test_attention_host import BAD_DESCS, INV, MB, SHAPE, WS, append, desc, paged, refused, rows

GB = 1 << 30
WORK = (GB, cf.CF_ATTN_WORKSPACE_BYTES)


def cache(**kw):
    c = dict(k=64 * MB, v=96 * MB, k_scale=128 * MB, v_scale=129 * MB, bounds=130 * MB, n_pages=10, page_stride=0, page_size=16)
    c.update(kw)
    return cf.cf_kv_cache8(**c)


def select(**kw):
    a = dict(n_seqs=3, max_pages=4, table_stride=0, max_len=0, table=1 * MB, lens=2 * MB, q=rows(3 * MB, 512, 128), count=3, first=1, recent=1, blocks=5 * MB)
    a.update(kw)
    return cf.cf_select(**a)


def plan(**kw):
    a = dict(n_seqs=3, page_size=16, max_pages=4, n_ring=100, table_stride=0, n_tokens=50, lens=1 * MB, news=2 * MB, table=3 * MB, ring=4 * MB, state=5 * MB,
             state_out=6 * MB, lens_out=7 * MB, cu=8 * MB, slots=9 * MB, positions=10 * MB, refused=11 * MB)
    a.update(kw)
    return cf.cf_plan(**a)


@pytest.mark.parametrize("d,status", BAD_DESCS)
def test_descriptors(d, status):
    refused(status, cf.cf_kv_append8, d, cache(), append())
    refused(status, cf.cf_attn_paged8, d, cache(), paged())
    refused(status, cf.cf_attn_select, d, cache(), select(), *WORK)


def test_null_arguments():
    refused(INV, cf.cf_kv_append8, desc(), None, append())
    refused(INV, cf.cf_kv_append8, desc(), cache(), None)
    refused(INV, cf.cf_attn_paged8, desc(), None, paged())
    refused(INV, cf.cf_attn_paged8, desc(), cache(), None)
    refused(INV, cf.cf_attn_select, desc(), cache(), None, *WORK)
    refused(INV, cf.cf_kv_plan, None)


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), INV), (dict(v=96 * MB + 8), INV), (dict(k_scale=None), INV), (dict(v_scale=129 * MB + 2), INV), (dict(bounds=130 * MB + 8), INV), (dict(page_size=8), SHAPE),
    (dict(page_size=48), SHAPE), (dict(page_size=256), SHAPE), (dict(n_pages=0), SHAPE), (dict(n_pages=1 << 31), SHAPE), (dict(page_stride=4088), SHAPE), (dict(page_stride=4104), SHAPE),
    (dict(page_stride=-4096), SHAPE), (dict(page_stride=(1 << 40) + 16), SHAPE), (dict(n_pages=(1 << 31) - 1, page_stride=1 << 36, v=64 * MB + 4096), SHAPE), (dict(v=64 * MB), INV),
    (dict(v=64 * MB + 4096 * 9), INV), (dict(v_scale=128 * MB + 76), INV), (dict(bounds=128 * MB), INV), (dict(k_scale=64 * MB + 4096), INV)])
def test_caches(kw, status):
    refused(status, cf.cf_kv_append8, desc(), cache(**kw), append())
    refused(status, cf.cf_attn_paged8, desc(), cache(**kw), paged())
    refused(status, cf.cf_attn_select, desc(), cache(**kw), select(), *WORK)


def test_pages_of_values_between_pages_of_keys():
    """Refused for the next reason only, so the cache is taken: the tokens' strides."""
    refused(SHAPE, cf.cf_kv_append8, desc(), cache(v=64 * MB + 4096, page_stride=8192), append(k=rows(1 * MB, 12, 128)))


@pytest.mark.parametrize("kw,status", [
    (dict(n_tokens=-1), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rotary_dim=8), SHAPE), (dict(rotary_dim=144), SHAPE), (dict(slots=None), INV), (dict(slots=3 * MB + 4), INV),
    (dict(k=rows(None, 256, 128)), INV), (dict(k=rows(1 * MB + 2, 256, 128)), INV), (dict(v=rows(2 * MB, 257, 128)), SHAPE), (dict(q=rows(None, 512, 128)), INV),
    (dict(q_out=rows(5 * MB, 256, 128)), INV), (dict(q_out=rows(4 * MB + 256, 512, 128)), INV), (dict(q_out=rows(1 * MB, 512, 128)), INV), (dict(q_out=rows(64 * MB, 512, 128)), INV),
    (dict(q_out=rows(130 * MB, 512, 128)), INV), (dict(k=rows(128 * MB - 1024, 256, 128)), INV), (dict(v=rows(96 * MB + 8192, 256, 128)), INV), (dict(positions=None), INV),
    (dict(cos=None), INV), (dict(sin=8 * MB + 4), INV), (dict(n_positions=0), SHAPE), (dict(n_tokens=1 << 30, k=rows(1 * MB, 0, 0), v=rows(2 * MB, 0, 0), q=rows(3 * MB, 0, 0)), INV)])
def test_append(kw, status):
    refused(status, cf.cf_kv_append8, desc(), cache(), append(**kw))


def test_append_of_more_work_items_than_a_launch_counts():
    one = dict(k=rows(1 * MB, 0, 0), v=rows(2 * MB, 0, 0), q=rows(None, 0, 0), q_out=rows(None, 0, 0), rotary_dim=0)
    refused(SHAPE, cf.cf_kv_append8, desc(q_heads=4, kv_heads=4), cache(v=512 * MB), append(n_tokens=1 << 30, **one))


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=-1), SHAPE), (dict(n_seqs=1 << 29), SHAPE), (dict(max_pages=0), SHAPE), (dict(table_stride=3), SHAPE), (dict(table_stride=(1 << 40) + 1), SHAPE),
    (dict(n_seqs=1 << 25, table_stride=1 << 40), SHAPE), (dict(max_len=-1), SHAPE), (dict(table=None), INV), (dict(lens=None), INV), (dict(table=1 * MB + 2), INV),
    (dict(q=rows(3 * MB + 8, 512, 128)), INV), (dict(q=rows(3 * MB, 508, 128)), SHAPE)])
def test_paged8_and_select(kw, status):
    refused(status, cf.cf_attn_paged8, desc(), cache(), paged(**kw))
    refused(status, cf.cf_attn_select, desc(), cache(), select(**kw), *WORK)


def test_paged8_alone():
    for kw in (dict(out=rows(3 * MB, 512, 128)), dict(out=rows(64 * MB, 512, 128)), dict(out=rows(129 * MB - 16, 512, 128)), dict(lse=5 * MB + 2)):
        refused(INV, cf.cf_attn_paged8, desc(), cache(), paged(**kw))
    refused(SHAPE, cf.cf_attn_paged8, desc(), cache(), paged(), cf.cf_blocks(9 * MB, 0))
    refused(SHAPE, cf.cf_attn_paged8, desc(), cache(), paged(), cf.cf_blocks(9 * MB, (1 << 20) + 1))
    refused(INV, cf.cf_attn_paged8, desc(), cache(), paged(), cf.cf_blocks(None, 3))
    refused(INV, cf.cf_attn_paged8, desc(), cache(), paged(), cf.cf_blocks(9 * MB + 2, 3))


@pytest.mark.parametrize("kw,status", [(dict(count=0), SHAPE), (dict(count=(1 << 20) + 1), SHAPE), (dict(first=-1), SHAPE), (dict(recent=-1), SHAPE), (dict(first=2, recent=2), SHAPE),
                                       (dict(first=(1 << 31) - 1, recent=(1 << 31) - 1), SHAPE), (dict(blocks=None), INV), (dict(blocks=5 * MB + 2), INV), (dict(blocks=3 * MB), INV),
                                       (dict(blocks=1 * MB + 40), INV), (dict(blocks=2 * MB), INV), (dict(blocks=130 * MB), INV)])
def test_select_alone(kw, status):
    refused(status, cf.cf_attn_select, desc(), cache(), select(**kw), *WORK)


def test_workspaces():
    refused(INV, cf.cf_attn_select, desc(), cache(bounds=None), select(), *WORK)
    for ws, n in ((None, 0), (None, 1 << 20), (GB + 128, 1 << 20), (GB, cf.CF_ATTN_COUNTER_BYTES + 31)):
        refused(WS, cf.cf_attn_select, desc(), cache(), select(), ws, n)
    for ws, n in ((None, 1 << 20), (GB + 128, 1 << 20)):
        refused(WS, cf.cf_attn_paged8, desc(), cache(), paged(), None, ws, n)
        refused(WS, cf.cf_kv_plan, plan(), ws, n)


@pytest.mark.parametrize("kw,status", [
    (dict(n_seqs=-1), SHAPE), (dict(n_seqs=(1 << 30) + 1), SHAPE), (dict(page_size=8), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=65536), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(n_ring=0), SHAPE), (dict(table_stride=3), SHAPE), (dict(n_tokens=-1), SHAPE), (dict(n_tokens=(1 << 30) + 1), SHAPE), (dict(lens=None), INV), (dict(news=None), INV),
    (dict(table=None), INV), (dict(ring=None), INV), (dict(state=None), INV), (dict(state_out=6 * MB + 4), INV), (dict(lens_out=None), INV), (dict(cu=8 * MB + 2), INV),
    (dict(slots=None), INV), (dict(slots=9 * MB + 4), INV), (dict(positions=None), INV), (dict(refused=None), INV), (dict(positions=9 * MB + 8 * 49), INV), (dict(cu=10 * MB), INV),
    (dict(lens_out=1 * MB + 4), INV), (dict(state_out=5 * MB + 8), INV), (dict(news=7 * MB), INV), (dict(ring=3 * MB + 4), INV), (dict(refused=2 * MB), INV), (dict(slots=1 * MB), INV)])
def test_plan(kw, status):
    refused(status, cf.cf_kv_plan, plan(**kw))


def test_nothing_to_do_is_done_without_a_device():
    cf.cf_kv_append8(desc(), cache(), append(n_tokens=0, k=rows(None, 0, 0), v=rows(None, 0, 0)))
    cf.cf_attn_paged8(desc(), cache(), paged(n_seqs=0, q=rows(None, 0, 0)))
    cf.cf_attn_select(desc(), cache(), select(n_seqs=0, q=rows(None, 0, 0)), *WORK)


# ---------------------------------------------------------------- the session

@pytest.fixture
def problem(monkeypatch):
    p = types.SimpleNamespace(calls=[])
    p.s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0, stream=types.SimpleNamespace(cuda_stream=0))
    p.s._lib = types.SimpleNamespace(**{name: lambda *a: p.calls.append(a) or 0 for name in ("cf_kv_append8", "cf_attn_paged8", "cf_attn_select", "cf_kv_plan")})
    monkeypatch.setattr(AttentionSession, "_call", lambda self, entry, name, *args: entry(*args))      # without the refusal of a session on the host
    p.cache = PagedCache8.empty(3, 2, 64, page_size=16, device="cpu")
    p.tables = PageTables.empty(3, 2, 9, 16, device="cpu")
    p.q, p.k, p.v, p.out = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2, 4))
    p.lse, p.cos, p.sin = torch.zeros(3, 4), torch.zeros(8, 32), torch.zeros(8, 32)
    p.numbers, p.table, p.blocks, p.slots = torch.ones(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2, 5, dtype=torch.int32), torch.arange(3)
    p.positions, p.cu, p.refused, p.lens_out, p.state_out = (torch.zeros(n, dtype=d) for n, d in ((3, torch.int32), (4, torch.int32), (1, torch.int32), (3, torch.int32), (2, torch.int64)))
    p.do = {"append8": lambda: p.s.append8(p.cache, p.k, p.v, p.slots, p.numbers, p.cos, p.sin, q=p.q, q_out=p.out),
            "paged8": lambda: p.s.paged8(p.cache, p.q, p.table, p.numbers, blocks=p.blocks, out=p.out, lse=p.lse),
            "select": lambda: p.s.select(p.cache, p.q, p.table, p.numbers, 5, out=p.blocks),
            "plan": lambda: p.s.plan(p.tables, p.numbers, 3, p.slots, p.positions, p.cu, p.lens_out, p.state_out, p.refused)}
    return p


@pytest.mark.parametrize("call,name", [("append8", x) for x in ("q", "k", "v", "cos", "sin", "out")] + [("paged8", "q"), ("paged8", "out"), ("paged8", "lse"), ("select", "q")])
def test_tensors_that_want_a_gradient(problem, call, name):
    getattr(problem, name).requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        problem.do[call]()
    with torch.no_grad():
        problem.do[call]()
    assert len(problem.calls) == 1


WRITTEN = {"append8": ["out", "cache.k", "cache.v", "cache.k_scale", "cache.v_scale", "cache.bounds"], "paged8": ["out", "lse"], "select": ["blocks"],
           "plan": ["tables.table", "tables.ring", "slots", "positions", "cu", "lens_out", "state_out", "refused"]}


@pytest.mark.parametrize("call", WRITTEN)
def test_what_is_written_counts_as_changed(problem, call):
    def find(name):
        x = problem
        for part in name.split("."):
            x = getattr(x, part)
        return x
    before = {name: find(name)._version for name in WRITTEN[call]}
    problem.do[call]()
    assert all(find(name)._version > was for name, was in before.items())


WRONG = [("append8", "slots", lambda x: x.int()), ("append8", "k", lambda x: x[:, :1]), ("append8", "k", lambda x: x.half()), ("append8", "out", lambda x: x[:2]),
         ("append8", "cos", lambda x: x.double()), ("paged8", "table", lambda x: x.long()), ("paged8", "table", lambda x: x[:2]), ("paged8", "numbers", lambda x: x.long()),
         ("paged8", "blocks", lambda x: x.long()), ("paged8", "blocks", lambda x: x[:, :1]), ("paged8", "blocks", lambda x: x[0]), ("paged8", "blocks", lambda x: x[:, :, ::2]),
         ("paged8", "lse", lambda x: x.half()), ("select", "blocks", lambda x: x[:, :, :4]), ("select", "blocks", lambda x: x.float()), ("select", "table", lambda x: x.t()),
         ("plan", "numbers", lambda x: x.long()), ("plan", "slots", lambda x: x.int()), ("plan", "positions", lambda x: x[:2]), ("plan", "cu", lambda x: x[:3]),
         ("plan", "lens_out", lambda x: x.long()), ("plan", "state_out", lambda x: x.int()), ("plan", "refused", lambda x: x.long())]


@pytest.mark.parametrize("call,name,change", WRONG)
def test_wrong_tensors(problem, call, name, change):
    setattr(problem, name, change(getattr(problem, name)))
    with pytest.raises(ValueError):
        problem.do[call]()
    assert not problem.calls


def test_caches_and_tables_that_do_not_fit(problem):
    other = AttentionSession(4, 4, 64, device="cpu", workspace_bytes=0, stream=types.SimpleNamespace(cuda_stream=0))
    other._lib = problem.s._lib
    k = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="cache"):
        other.append8(problem.cache, k, k, problem.slots)
    problem.cache.bounds = None
    with pytest.raises(ValueError, match="bounds"):
        problem.do["select"]()
    page, scale = torch.zeros(3, 2, 16, 64, dtype=torch.float8_e4m3fn), torch.ones(3, 2)
    bounds = torch.zeros(3, 2, 2, 64, dtype=torch.bfloat16)
    PagedCache8(page, page.clone(), scale, scale.clone(), bounds)
    for args in ((page.float(), page, scale, scale), (page, page[:2], scale, scale), (page, page.transpose(1, 2), scale, scale), (page, page, scale[:2], scale), (page, page, scale, scale.double()),
                 (page, page, scale, scale, bounds[:, :1]), (page, page, scale, scale, bounds.float())):
        with pytest.raises(ValueError):
            PagedCache8(*args)
    with pytest.raises(ValueError, match="gradient"):
        PagedCache8(page, page, scale.clone().requires_grad_(), scale)
    t = problem.tables
    for args in ((t.table.long(), t.lens, t.ring, t.state), (t.table, t.lens[:2], t.ring, t.state), (t.table, t.lens, t.ring.long(), t.state), (t.table, t.lens, t.ring, t.state.int()),
                 (t.table[:, ::2], t.lens, t.ring, t.state[:1]), (t.table.t().contiguous().t(), t.lens, t.ring, t.state)):
        with pytest.raises(ValueError):
            PageTables(*args, 16)


@pytest.mark.parametrize("mine,current", [(1, 0), (0, 1), (1, 1)])
def test_calls_are_made_on_the_sessions_device(machine, mine, current):  # noqa: F811
    machine.device = current
    s = AttentionSession(4, 2, 64, device=f"cuda:{mine}", workspace_bytes=0)
    s._lib = types.SimpleNamespace(**{name: machine.entry for name in ("cf_kv_append8", "cf_attn_paged8", "cf_attn_select", "cf_kv_plan")})

    def on(*shape, dtype=torch.bfloat16):
        return Tensor(shape, dtype, mine)

    cache = types.SimpleNamespace(heads=2, head_dim=64, index=mine, ref=None, k=on(1), written=[], bounds=on(1))
    tables = types.SimpleNamespace(seqs=3, index=mine, head=(3, 16, 2, 9, 0), at=(0, 0, 0), lens=on(3, dtype=torch.int32), state=on(2, dtype=torch.int64), table=None, ring=None)
    numbers, table, q = on(3, dtype=torch.int32), on(3, 2, dtype=torch.int32), on(3, 4, 64)
    s.append8(cache, on(3, 2, 64), on(3, 2, 64), on(3, dtype=torch.int64), q=q, q_out=on(3, 4, 64))
    s.select(cache, q, table, numbers, 5, out=on(3, 2, 5, dtype=torch.int32))
    s.paged8(cache, q, table, numbers, out=on(3, 4, 64))
    s.plan(tables, numbers, 3, on(3, dtype=torch.int64), on(3, dtype=torch.int32), on(4, dtype=torch.int32), refused=on(1, dtype=torch.int32))
    assert machine.calls == [mine] * 4 and machine.device == current


def test_tensors_of_the_host_do_not_reach_the_library():
    s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0)
    calls = []
    s._lib = types.SimpleNamespace(**{name: lambda *a: calls.append(a) or 0 for name in ("cf_kv_append8", "cf_attn_paged8", "cf_attn_select", "cf_kv_plan")})
    cache, tables = PagedCache8.empty(3, 2, 64, page_size=16, device="cpu"), PageTables.empty(3, 2, 9, 16, device="cpu")
    q, k, numbers, table = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.ones(3, dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32)
    for call in (lambda: s.append8(cache, k, k, torch.arange(3)), lambda: s.paged8(cache, q, table, numbers), lambda: s.select(cache, q, table, numbers, 2),
                 lambda: s.plan(tables, numbers, 3)):
        with pytest.raises(ValueError, match="cpu"):
            call()
    assert not calls
