"""A tensor that is put in another's place in a cache, or in the tables of a batch, is checked as the first one was and is what the next call is given: no call
is left with the address of one that may be gone.  Needs no GPU."""
import pytest
import torch

from paper_2507_17511_amd import attention
from paper_2507_17511_amd.attention import PagedCache, PagedCache8, PageTables
from test_cache8_host import problem  # noqa: F401

PLAN = ("seqs", "page_size", "max_pages", "n_ring", "stride", "tokens", "lens", "news", "table", "ring", "state", "state_out", "lens_out", "cu", "slots", "positions", "refused")


def planned(p):
    p.s.plan(p.tables, p.numbers, 3, p.slots, p.positions, p.cu, refused=p.refused)
    return dict(zip(PLAN, attention._PLAN.unpack(p.calls[-1][0])))


@pytest.mark.parametrize("name,new", [("table", torch.zeros(3, 7, dtype=torch.int32)), ("lens", torch.ones(3, dtype=torch.int32)), ("ring", torch.zeros(20, dtype=torch.int32)),
                                      ("state", torch.ones(2, dtype=torch.int64))])
def test_a_plan_is_given_what_the_tables_hold(problem, name, new):  # noqa: F811
    before = planned(problem)
    setattr(problem.tables, name, new)
    after = planned(problem)
    assert getattr(problem.tables, name) is new and after[name] == new.data_ptr() != before[name]
    changed = {name} | {"table": {"max_pages", "stride"}, "ring": {"n_ring"}, "state": {"state_out"}, "lens": {"lens_out"}}[name]
    assert {k for k in PLAN if after[k] != before[k]} == changed
    assert after["max_pages"] == problem.tables.table.shape[1] and after["n_ring"] == problem.tables.ring.numel()


@pytest.mark.parametrize("name,wrong", [("table", torch.zeros(4, 7, dtype=torch.int32)), ("table", torch.zeros(3, 7)), ("table", torch.zeros(3, 7, dtype=torch.int32)[:, ::2]),
                                        ("lens", torch.ones(2, dtype=torch.int32)), ("lens", torch.ones(3, dtype=torch.int64)), ("ring", torch.ones(20, dtype=torch.int64)),
                                        ("state", torch.ones(2, dtype=torch.int32)), ("state", torch.ones(3, dtype=torch.int64))])
def test_tables_that_do_not_fit_are_refused_and_the_old_ones_stay(problem, name, wrong):  # noqa: F811
    before = planned(problem)
    with pytest.raises(ValueError):
        setattr(problem.tables, name, wrong)
    assert planned(problem) == before


def codes(n, page=16):
    return torch.zeros(n, 2, page, 64, dtype=torch.float8_e4m3fn)


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale", "bounds"])
def test_a_cache_in_8_bits(name):
    cache = PagedCache8.empty(3, 2, 64, page_size=16, device="cpu")
    new = getattr(cache, name).clone()
    setattr(cache, name, new)
    assert getattr(cache, name) is new and getattr(cache.struct, name) == new.data_ptr() and cache.ref._obj is cache.struct
    assert any(x is new for x in cache.written) and len(cache.written) == 5
    with pytest.raises(ValueError):
        setattr(cache, name, new[:2])
    assert getattr(cache, name) is new


def test_a_cache_in_8_bits_without_bounds_any_more():
    cache = PagedCache8.empty(3, 2, 64, page_size=16, device="cpu")
    cache.bounds = None
    assert cache.struct.bounds is None and len(cache.written) == 4
    with pytest.raises(ValueError):
        cache.k = codes(3, 32)


@pytest.mark.parametrize("name", ["k", "v"])
def test_a_cache_in_16_bits(name):
    cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    new = getattr(cache, name).clone()
    setattr(cache, name, new)
    assert getattr(cache, name) is new and getattr(cache.struct, name) == new.data_ptr()
    with pytest.raises(ValueError):
        setattr(cache, name, new.half())
    assert getattr(cache, name) is new


def test_other_attributes_may_be_set():
    for x in (PagedCache.empty(1, 1, 64, 16, device="cpu"), PagedCache8.empty(1, 1, 64, 16, device="cpu"), PageTables.empty(1, 1, 1, 16, device="cpu")):
        x.layer = 3
        assert x.layer == 3
