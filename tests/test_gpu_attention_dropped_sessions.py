"""Sessions that are dropped while a call of theirs on a busy stream is yet to run: memory that is allocated next is not their workspace.  And one that is made
during a capture, where its zero fill is only recorded."""
import pytest
import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession
from test_gpu_attention import DEV
from test_gpu_attention_streams import D, HK, HQ, busy, check_out, problem

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("own", [False, True])
def test_a_session_dropped_before_its_call_runs(own):
    cache, q, table, lens = problem()
    work, side = torch.randn(6144, 6144, device=DEV).bfloat16(), torch.cuda.Stream()
    torch.mm(work, work)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    with torch.cuda.stream(side):
        for _ in range(10):             # some 200 ms: longer than the allocations below
            busy(work)
    if own:
        s = AttentionSession(HQ, HK, D, stream=side)
        workspace = s.workspace.data_ptr()
        out = s.paged(cache, q, table, lens)
    else:
        s = AttentionSession(HQ, HK, D)
        workspace = s.workspace.data_ptr()
        with torch.cuda.stream(side):
            out = s.paged(cache, q, table, lens)
    del s
    junk = [torch.full((cf.CF_ATTN_WORKSPACE_BYTES,), 255, dtype=torch.uint8, device=DEV) for _ in range(3)]
    assert side.query() or all(j.data_ptr() != workspace for j in junk)      # not while the call is yet to run
    torch.cuda.synchronize()
    check_out(cache, q, out)


def test_a_session_made_during_a_capture():
    cache, q, table, lens = problem()
    AttentionSession(HQ, HK, D).paged(cache, q, table, lens)
    out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        s = AttentionSession(HQ, HK, D)
        s.paged(cache, q, table, lens, out=out)
    check_out(cache, q, s.paged(cache, q, table, lens))         # before the graph has run
    for _ in range(3):
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_out(cache, q, out)
        check_out(cache, q, s.paged(cache, q, table, lens))
        torch.cuda.synchronize()
