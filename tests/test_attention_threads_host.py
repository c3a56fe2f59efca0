"""One session used by several threads: each call reaches the library with its own arguments.  The interpreter's lock is free during a call, so that what a call hands
over must not be another's to overwrite.  A stand-in for the library looks at it after others have had their turn."""
import ctypes
import threading
import time
import types

import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession, PagedCache

ENTRIES = {"cf_kv_append": (2, cf.cf_append), "cf_attn_prompt": (1, cf.cf_prompt), "cf_attn_paged": (2, cf.cf_paged), "cf_attn_join": (1, cf.cf_join)}


@pytest.mark.parametrize("name", list(ENTRIES))
def test_arguments_are_the_callers_own(monkeypatch, name):
    where, kind = ENTRIES[name]
    threads = 4
    together, out_of = threading.Barrier(threads), {"cf_kv_append": "q_out"}
    seen = {}

    def entry(*args):
        together.wait(20)               # every thread has handed its arguments over
        given = args[where]
        given = given._obj if hasattr(given, "_obj") else ctypes.cast(given, ctypes.POINTER(kind)).contents
        seen[threading.get_ident()] = getattr(given, out_of.get(name, "out")).data
        together.wait(20)
        return 0

    s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0, stream=types.SimpleNamespace(cuda_stream=0))
    s._lib = types.SimpleNamespace(**{name: entry})
    q, k, v = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2))
    cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    numbers, starts, table, lses = torch.ones(3, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32), [torch.zeros(3, 4)] * 2
    calls = {"cf_kv_append": lambda out: s.append(cache, k, v, torch.arange(3), q=q, q_out=out), "cf_attn_prompt": lambda out: s.prompt(q, k, v, starts, out=out),
             "cf_attn_paged": lambda out: s.paged(cache, q, table, numbers, out=out), "cf_attn_join": lambda out: s.join([q, q], lses, out=out)}
    monkeypatch.setattr(AttentionSession, "_call", lambda self, entry, name, *args: entry(*args))      # without the refusal of a session on the host
    wrong = []

    def work():
        out = torch.empty_like(q)
        calls[name](out)
        if seen[threading.get_ident()] != out.data_ptr():
            wrong.append(threading.get_ident())

    workers = [threading.Thread(target=work) for _ in range(threads)]
    for w in workers:
        w.start()
    for w in workers:
        w.join(60)
    assert len(seen) == threads and not wrong


@pytest.mark.parametrize("name", ["cf_attn_prompt", "cf_attn_paged"])
def test_calls_with_the_workspace_come_one_after_another(monkeypatch, name):
    """A call enqueues two kernels at most, of which the second reads from the workspace what the first wrote there."""
    inside, most = [0], [0]

    def entry(*args):
        inside[0] += 1
        most[0] = max(most[0], inside[0])
        time.sleep(0.05)
        inside[0] -= 1
        return 0

    s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=1 << 20)
    s._lib = types.SimpleNamespace(**{name: entry})
    monkeypatch.setattr(AttentionSession, "_call", lambda self, entry, name, *args: entry(*args))
    q, k, v = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2))
    cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    numbers, starts, table = torch.ones(3, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32)
    out = torch.empty_like(q)
    call = {"cf_attn_prompt": lambda: s.prompt(q, k, v, starts, out=out), "cf_attn_paged": lambda: s.paged(cache, q, table, numbers, out=out)}[name]
    workers = [threading.Thread(target=call) for _ in range(4)]
    for w in workers:
        w.start()
    for w in workers:
        w.join(60)
    assert most[0] == 1
