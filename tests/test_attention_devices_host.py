"""On which device the library is called.  Kernels launched with the null stream run on the device that is current, so that a session must make
its own current, whichever the caller has: with a stand-in for the library, needs no GPU."""
import types

import pytest
import torch

from paper_2507_17511_amd import attention, session
from paper_2507_17511_amd.attention import AttentionSession


class Tensor:
    """As much of a tensor on some device as a session looks at."""
    requires_grad = False

    def __init__(self, shape, dtype=torch.bfloat16, index=1):
        self.shape, self.dtype, self.index = torch.Size(shape), dtype, index
        self.device = torch.device("cuda", index)

    def get_device(self):
        return self.index

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self):
        return torch.empty(self.shape, device="meta").stride()

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


@pytest.fixture
def machine(monkeypatch):
    """Two devices, of which 0 is current; where `calls` were made."""
    now = types.SimpleNamespace(device=0, calls=[])

    class guard:
        def __init__(self, device):
            self.device = device if isinstance(device, int) else torch.device(device).index

        def __enter__(self):
            self.before, now.device = now.device, self.device

        def __exit__(self, *error):
            now.device = self.before

    monkeypatch.setattr(torch.cuda, "device", guard)
    for module in (attention, session):
        monkeypatch.setattr(module, "_current_device", lambda: now.device, raising=False)
    monkeypatch.setattr(attention, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(attention, "_written", lambda tensors: None)

    def entry(*args):
        now.calls.append(now.device)
        return 0

    now.entry = entry
    now.library = types.SimpleNamespace(**{name: entry for name in ("cf_kv_append", "cf_attn_prompt", "cf_attn_paged", "cf_attn_join")})
    return now


@pytest.mark.parametrize("mine,current", [(1, 0), (0, 1), (1, 1), (0, 0)])
def test_attention_is_called_on_the_sessions_device(machine, mine, current):
    machine.device = current
    s = AttentionSession(4, 2, 64, device=f"cuda:{mine}", workspace_bytes=0)
    s._lib = machine.library

    def on(*shape, dtype=torch.bfloat16):
        return Tensor(shape, dtype, mine)

    cache = types.SimpleNamespace(heads=2, head_dim=64, dtype=torch.bfloat16, index=mine, ref=None, k=on(1), v=on(1))
    numbers = on(3, dtype=torch.int32)
    q, k, v, out = on(3, 4, 64), on(3, 2, 64), on(3, 2, 64), on(3, 4, 64)
    table = on(3, 2, dtype=torch.int32)
    s.append(cache, k, v, on(3, dtype=torch.int64), q=q, q_out=out)
    s.prompt(q, k, v, on(2, dtype=torch.int32), out=out)
    s.paged(cache, q, table, numbers, out=out)
    s.join([q, q], [on(3, 4, dtype=torch.float32)] * 2, out=out)
    assert machine.calls == [mine] * 4 and machine.device == current


@pytest.mark.parametrize("mine,current", [(1, 0), (0, 1), (1, 1), (0, 0)])
def test_the_codec_is_called_on_the_sessions_device(machine, monkeypatch, mine, current):
    machine.device = current
    for name in ("cf_warmup", "cf_step_fused", "cf_compress", "cf_decompress"):
        monkeypatch.setattr(session.cf, name, machine.entry)
    s = session.CodecSession.__new__(session.CodecSession)          # its buffers are not looked at here
    s.device, s.n, s.ctx, s._stream = torch.device("cuda", mine), 1, None, types.SimpleNamespace(cuda_stream=0)
    s.p_recon = s.p_err = s.p_codes = s.p_scales = (None,)
    x = Tensor((4, 64), index=mine)
    monkeypatch.setattr(session.cf, "ptr_array", lambda xs: xs)
    s.warmup([x])
    s.step_fused([x])
    s.compress([x])
    s.decompress()
    assert machine.calls == [mine] * 4 and machine.device == current


def test_the_workspace_is_recorded_on_every_stream_that_uses_it(machine, monkeypatch):
    """The allocator must not hand it out again while a call on some other stream than the one it was made on is under way."""
    now, recorded = types.SimpleNamespace(handle=0), []
    monkeypatch.setattr(attention, "_raw_stream", lambda index: now.handle)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=now.handle))
    s = AttentionSession(4, 2, 64, device="cuda:0", workspace_bytes=0)
    s._lib, s.ws_bytes = machine.library, 1 << 20
    s.workspace, s._ws = types.SimpleNamespace(record_stream=lambda stream: recorded.append(stream.cuda_stream)), 1 << 20
    cache = types.SimpleNamespace(heads=2, head_dim=64, dtype=torch.bfloat16, index=0, ref=None, k=Tensor((1,)), v=Tensor((1,)))
    q, k, v, out = (Tensor((3, h, 64), index=0) for h in (4, 2, 2, 4))
    starts, table, lens = (Tensor(shape, torch.int32, 0) for shape in ((2,), (3, 2), (3,)))
    for handle in (0, 0, 7, 7, 9, 7, 0):
        now.handle = handle
        s.prompt(q, k, v, starts, out=out)
        s.paged(cache, q, table, lens, out=out)
    assert set(recorded) >= {7, 9} and len(recorded) <= 3       # each once, the one it was made on at most once


def test_a_workspace_made_during_a_capture_is_zero_for_calls_outside_of_it(machine, monkeypatch):
    """The fill that zeroes it is captured, not run: calls until the first one outside of a capture zero the counters themselves."""
    capturing, found = [True], []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(torch, "zeros", lambda n, dtype, device: torch.full((n,), 255, dtype=dtype))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda x, stream: None)
    s = AttentionSession(4, 2, 64, device="cuda:0", workspace_bytes=1 << 20)
    counters = s.workspace[:attention.cf.CF_ATTN_COUNTER_BYTES]

    def entry(*args):
        found.append(int(counters.max()))
        return 0

    s._lib = types.SimpleNamespace(cf_attn_paged=entry)
    cache = types.SimpleNamespace(heads=2, head_dim=64, dtype=torch.bfloat16, index=0, ref=None, k=Tensor((1,)), v=Tensor((1,)))
    q, out, table, lens = Tensor((3, 4, 64), index=0), Tensor((3, 4, 64), index=0), Tensor((3, 2), torch.int32, 0), Tensor((3,), torch.int32, 0)
    for now in (True, True, False, True, False):
        capturing[0] = now
        s.paged(cache, q, table, lens, out=out)
        if now and len(found) < 3:
            counters.fill_(255)             # what the captured call did has not happened
        elif len(found) == 3:
            counters[5] = 9                 # every call leaves them zero, so that no later one has to: this would stay
    assert found == [0, 0, 0, 9, 9]


@pytest.mark.parametrize("stream", [None, types.SimpleNamespace(cuda_stream=0)])
def test_tensors_of_the_host_do_not_reach_the_library(stream):
    """Its kernels would read and write the host's addresses."""
    calls = []
    s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0, stream=stream)
    s._lib = types.SimpleNamespace(**{name: lambda *a: calls.append(a) or 0 for name in ("cf_kv_append", "cf_attn_prompt", "cf_attn_paged", "cf_attn_join")})
    q, k, v = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2))
    cache = attention.PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    numbers, starts = torch.ones(3, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)
    out = torch.empty_like(q)
    for call in (lambda: s.append(cache, k, v, torch.arange(3), q=q, q_out=out), lambda: s.prompt(q, k, v, starts, out=out),
                 lambda: s.paged(cache, q, torch.zeros(3, 2, dtype=torch.int32), numbers, out=out), lambda: s.join([q, q], [torch.zeros(3, 4)] * 2, out=out)):
        with pytest.raises(ValueError, match="cpu"):
            call()
    assert not calls
