"""The attention calls have no gradients: tensors that want one are refused while gradients are recorded, and what a call writes counts as
changed, so that autograd notices where it had kept it for a backward pass.  With a stand-in for the library, needs no GPU."""
import types

import pytest
import torch

from paper_2507_17511_amd.attention import AttentionSession, PagedCache


@pytest.fixture
def problem(monkeypatch):
    p = types.SimpleNamespace()
    p.s = AttentionSession(4, 2, 64, device="cpu", workspace_bytes=0, stream=types.SimpleNamespace(cuda_stream=0))
    p.s._lib = types.SimpleNamespace(**{name: lambda *a: 0 for name in ("cf_kv_append", "cf_attn_prompt", "cf_attn_paged", "cf_attn_join")})
    monkeypatch.setattr(AttentionSession, "_call", lambda self, entry, name, *args: entry(*args))      # without the refusal of a session on the host
    p.cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
    p.q, p.k, p.v, p.out = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2, 4))
    p.lse, p.parts, p.lses = torch.zeros(3, 4), [torch.zeros(3, 4, 64, dtype=torch.bfloat16) for _ in range(2)], [torch.zeros(3, 4) for _ in range(2)]
    p.cos, p.sin = torch.zeros(8, 32), torch.zeros(8, 32)
    numbers, starts, table = torch.ones(3, dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32), torch.zeros(3, 2, dtype=torch.int32)
    p.calls = {"append": lambda: p.s.append(p.cache, p.k, p.v, torch.arange(3), numbers, p.cos, p.sin, q=p.q, q_out=p.out),
               "prompt": lambda: p.s.prompt(p.q, p.k, p.v, starts, out=p.out, lse=p.lse), "paged": lambda: p.s.paged(p.cache, p.q, table, numbers, out=p.out, lse=p.lse),
               "join": lambda: p.s.join(p.parts, p.lses, out=p.out, lse=p.lse)}
    return p


READ = [("append", "q"), ("append", "k"), ("append", "v"), ("append", "cos"), ("append", "sin"), ("prompt", "q"), ("prompt", "k"), ("prompt", "v"), ("paged", "q"), ("join", "parts"),
        ("join", "lses")]
WRITTEN = [("append", "out"), ("prompt", "out"), ("prompt", "lse"), ("paged", "out"), ("paged", "lse"), ("join", "out"), ("join", "lse")]


@pytest.mark.parametrize("call,name", READ + WRITTEN)
def test_tensors_that_want_a_gradient(problem, call, name):
    x = getattr(problem, name)
    (x[-1] if isinstance(x, list) else x).requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        problem.calls[call]()
    with torch.no_grad():
        problem.calls[call]()
    with torch.inference_mode():
        problem.calls[call]()


def test_a_cache_that_wants_a_gradient():
    page = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    for k, v in ((page.clone().requires_grad_(), page), (page, page.clone().requires_grad_() * 1)):
        with pytest.raises(ValueError, match="gradient"):
            PagedCache(k, v)
        with torch.no_grad():
            PagedCache(k, v)


@pytest.mark.parametrize("call,name", WRITTEN + [("append", "cache")])
def test_what_is_written_counts_as_changed(problem, call, name):
    for x in (problem.cache.k, problem.cache.v) if name == "cache" else (getattr(problem, name),):
        for mode in (torch.enable_grad(), torch.no_grad()):
            before = x._version
            with mode:
                problem.calls[call]()
            assert x._version > before
    before = problem.q._version, problem.k._version, problem.parts[0]._version
    problem.calls[call]()
    assert before == (problem.q._version, problem.k._version, problem.parts[0]._version)


@pytest.mark.parametrize("call", ["append", "prompt", "paged", "join"])
def test_tensors_made_for_inference(problem, call):
    """They have no versions, and may be given to every call."""
    with torch.inference_mode():
        problem.out, problem.lse = torch.zeros_like(problem.out), torch.zeros_like(problem.lse)
        problem.cache = PagedCache.empty(3, 2, 64, page_size=16, device="cpu")
        problem.calls[call]()
    problem.calls[call]()


def test_a_changed_output_is_noticed_by_the_backward_pass(problem):
    x = torch.ones(3, 4, 64, dtype=torch.bfloat16, requires_grad=True)
    y = x * problem.out                     # keeps problem.out
    problem.calls["prompt"]()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
