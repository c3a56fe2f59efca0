"""The attention operators next to the codec, as calls that can be timed: keys and values appended to a paged cache,
attention over whole prompts, attention of one new token over the cache, and the join of partial attentions.

A case is one call.  With `own` false a pass computes it from elementary torch operations in fp32, rounded once at the
end; with `own` true it is the framework's call on the same buffers.  `exact` computes the same outputs in fp64, sequence
by sequence and without either of the two.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---------------------------------------------------------------- the cases

def _append(name, tokens, q_heads, kv_heads, dim, dtype, page, spare, rotated, style, packed):
    return {"name": name, "op": "append", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
            "page": page, "spare": spare,        # tokens a page holds; slots of the cache that the call leaves alone, per token appended
            "rotated": rotated, "style": style,  # leading dimensions that are rotated, and which two make a pair: "half" or "pairs"
            "packed": packed,                    # q, k and v are slices of the one product they came from
            "scattered": tokens <= 512}          # a token of every sequence (any page), or whole prompts (page after page)


def _prompt(name, seqs, longest, ragged, past, q_heads, kv_heads, dim, dtype, causal, lse, packed, lengths=1):
    return {"name": name, "op": "prompt", "seqs": seqs, "longest": longest, "ragged": ragged,
            "past": past,                        # keys of every sequence ahead of the new tokens
            "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "causal": causal,
            "lse": lse,                          # the rows' log-sum-exps are asked for too, so that the output can be joined
            "packed": packed, "lengths": lengths}


def _paged(name, seqs, longest, ragged, q_heads, kv_heads, dim, dtype, page, lengths=1):
    return {"name": name, "op": "paged", "seqs": seqs, "longest": longest, "ragged": ragged, "q_heads": q_heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page, "lengths": lengths}


def _join(name, parts, tokens, heads, dim, part_dtype, dtype):
    return {"name": name, "op": "join", "parts": parts, "tokens": tokens, "heads": heads, "dim": dim, "part_dtype": part_dtype, "dtype": dtype}


def listed():
    return [
        # a serving step's new tokens, one of each of 48 sequences: rotated, put wherever their sequences' last pages are
        _append("append_step", 48, 32, 8, 128, "bf16", 16, 8.0, 128, "half", True),
        # a long prompt's tokens at once, as many as the video workload has; half of every head is rotated, in pairs
        _append("append_prompt", 16384, 24, 8, 128, "f16", 64, 0.5, 64, "pairs", True),
        # three short requests that came in together, the shortest one token: only latency counts
        _prompt("prompt_few", 3, 45, True, 0, 8, 2, 64, "bf16", True, False, True),
        # a batch of chat-sized prompts packed one after another, from one token to two thousand
        _prompt("prompt_packed", 14, 2003, True, 0, 32, 8, 128, "bf16", True, False, True),
        # the image workload's full sequence, every token over all keys: one hop of ring attention, to be joined
        _prompt("prompt_ring_hop", 1, 4096, False, 0, 24, 24, 128, "bf16", False, True, False),
        # the next 333 tokens of two long prompts over what came before: few rows, many keys, wide heads
        _prompt("prompt_chunk", 2, 333, False, 20000, 16, 2, 256, "f16", True, False, False),
        # two long prompts of odd length
        _prompt("prompt_long", 2, 8191, False, 0, 32, 8, 128, "bf16", True, False, False),
        # the video workload's sequence: the largest product
        _prompt("prompt_video", 1, 16384, False, 0, 24, 24, 128, "bf16", False, False, False),
        # one request alone, a short context: only latency counts
        _paged("paged_one", 1, 901, False, 8, 2, 128, "bf16", 16),
        # a full batch of requests whose contexts differ widely
        _paged("paged_batch", 96, 16000, True, 32, 8, 128, "bf16", 16),
        # two requests of a very long context each: few rows, one long axis; a head of keys for each of queries, narrow ones
        _paged("paged_long", 2, 131100, False, 24, 24, 64, "f16", 64),
        # the end of ring attention over four peers' shards of the image workload
        _join("join_ring", 4, 4096, 24, 128, "bf16", "bf16"),
    ]


# What a drawn case may cost, by operator: no more than the largest listed one.
MOST_PAIRS_FLOPS = 3.2e12               # prompt_video
MOST_SCORES = 6.0e9                     # ... whose plain form holds so many scores
MOST_CACHE_BYTES = 1.6e9                # paged_long
MOST_APPEND_BYTES = 4.0e8
MOST_JOIN_BYTES = 2.2e8


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    kv = rng.choice([1, 2, 3, 4, 8, 8, 10])
    return kv * rng.choice([1, 2, 3, 4, 4, 5, 8]), kv


def draw(rng):
    """One more case: any operator, heads, dimensions and types, lengths from one to the longest listed."""
    op = rng.choices(["prompt", "paged", "append", "join"], [5, 4, 2, 1])[0]
    q_heads, kv_heads = _heads(rng)
    dim = rng.choice([64, 128, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    while True:
        if op == "prompt":
            seqs = _log_uniform(rng, 1, 24)
            c = _prompt("", seqs, _log_uniform(rng, 1, 16384), seqs > 1 and rng.random() < 0.7, rng.choice([0, 0, 0, _log_uniform(rng, 1, 30000)]),
                        q_heads, kv_heads, dim, dtype, rng.random() < 0.7, rng.random() < 0.3, rng.random() < 0.5, rng.randrange(1, 1000))
            fits = work(c)["flops"] <= MOST_PAIRS_FLOPS and seqs * q_heads * c["longest"] * (c["longest"] + c["past"]) <= MOST_SCORES
        elif op == "paged":
            seqs = _log_uniform(rng, 1, 200)
            c = _paged("", seqs, _log_uniform(rng, 1, 131100), seqs > 1 and rng.random() < 0.7, q_heads, kv_heads, dim, dtype,
                       rng.choice([16, 16, 32, 64, 128]), rng.randrange(1, 1000))
            fits = work(c)["bytes"] <= MOST_CACHE_BYTES and 4 * seqs * c["longest"] * kv_heads * dim <= 4 * MOST_CACHE_BYTES
        elif op == "append":
            c = _append("", _log_uniform(rng, 1, 20000), q_heads, kv_heads, dim, dtype, rng.choice([16, 16, 32, 64, 128]), rng.choice([0.5, 2.0]),
                        rng.choice([dim, dim, dim // 2, dim // 4]), rng.choice(["half", "pairs"]), rng.random() < 0.5)
            fits = work(c)["bytes"] <= MOST_APPEND_BYTES
        else:
            part_dtype = rng.choice(["f32", dtype])
            c = _join("", rng.randrange(2, 9), _log_uniform(rng, 1, 8192), q_heads, dim, part_dtype, dtype)
            fits = work(c)["bytes"] <= MOST_JOIN_BYTES
        if fits:
            del c["name"]
            return c


def _lengths(case):
    """Tokens of every sequence: a property of the case.  Ragged ones spread from one token to the longest."""
    if not case["ragged"]:
        return [case["longest"]] * case["seqs"]
    r = random.Random(case["lengths"])
    got = [max(1, min(case["longest"], _log_uniform(r, max(1, case["longest"] / 100), case["longest"]))) for _ in range(case["seqs"])]
    got[r.randrange(case["seqs"])] = case["longest"]
    if case["seqs"] > 2:
        got[(got.index(case["longest"]) + 1) % case["seqs"]] = 1
    return got


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    d = case["dim"]
    if case["op"] == "append":
        t, rows = case["tokens"], case["q_heads"] + 2 * case["kv_heads"]
        table = t * case["rotated"] * 4             # a row of cosines and one of sines for every token
        return {"bytes": 2 * t * rows * d * 2 + table + t * 12, "flops": 3 * t * (case["q_heads"] + case["kv_heads"]) * case["rotated"]}
    if case["op"] == "prompt":
        lens = _lengths(case)
        tq, tk = sum(lens), sum(lens) + case["past"] * len(lens)
        pairs = sum(n * case["past"] + (n * (n + 1) // 2 if case["causal"] else n * n) for n in lens)
        out = tq * case["q_heads"] * (2 * d + (4 if case["lse"] else 0))
        return {"bytes": 2 * d * (tq * case["q_heads"] + 2 * tk * case["kv_heads"]) + out, "flops": 4 * pairs * case["q_heads"] * d}
    if case["op"] == "paged":
        keys = sum(_lengths(case))
        return {"bytes": 4 * keys * case["kv_heads"] * d + 4 * case["seqs"] * case["q_heads"] * d + 4 * (keys // case["page"]),
                "flops": 4 * keys * case["q_heads"] * d}
    rows = case["tokens"] * case["heads"]
    return {"bytes": rows * (case["parts"] * (d * size[case["part_dtype"]] + 4) + d * size[case["dtype"]] + 4), "flops": 2 * rows * case["parts"] * d}


# ---------------------------------------------------------------- what a program has in hand before the call

def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _qkv(g, tokens_q, tokens_k, case):
    """Queries, keys and values as projections give them: channels of unlike size, keys with an offset per channel, which
    all queries' scores share, and values around a mean of their own."""
    dt, d, hq, hk = DTYPES[case["dtype"]], case["dim"], case["q_heads"], case["kv_heads"]
    if case["packed"] and tokens_q == tokens_k:
        all_ = _randn(g, (tokens_q, hq + 2 * hk, d), dt)
        q, k, v = all_[:, :hq], all_[:, hq:hq + hk], all_[:, hq + hk:]
    else:
        q, k, v = _randn(g, (tokens_q, hq, d), dt), _randn(g, (tokens_k, hk, d), dt), _randn(g, (tokens_k, hk, d), dt)
    q.mul_((0.6 + 0.8 * torch.rand(hq, d, generator=g, device="cuda")).to(dt))
    k.mul_((0.6 + 0.8 * torch.rand(hk, d, generator=g, device="cuda")).to(dt)).add_(_randn(g, (hk, d), dt).mul_(0.5))
    v.add_(_randn(g, (hk, d), dt).mul_(0.3))
    return q, k, v


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _session(case):
    from paper_2507_17511_amd.attention import AttentionSession
    heads = case.get("heads", case.get("q_heads"))
    return AttentionSession(heads, case.get("kv_heads", heads), case["dim"], dtype=DTYPES[case["dtype"]])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, dt, s = case["dim"], DTYPES[case["dtype"]], {"case": case}
    if case["op"] == "append":
        t, ps, hk = case["tokens"], case["page"], case["kv_heads"]
        pages = -(-int(t * (1 + case["spare"])) // ps) + 1
        s["q"], s["k"], s["v"] = _qkv(g, t, t, case)
        s["k_cache"], s["v_cache"] = (_randn(g, (pages, hk, ps, d), dt) for _ in range(2))
        if case["scattered"]:       # every token has a page of its own where there are enough
            page = torch.randperm(pages, generator=g, device="cuda")
            at = torch.arange(t, device="cuda")
            off = torch.randint(0, ps, (pages,), generator=g, device="cuda")
            s["slots"] = page[at % pages] * ps + (off[at % pages] + at // pages) % ps
            s["positions"] = torch.randint(0, 4096, (t,), generator=g, device="cuda", dtype=torch.int32)
        else:                       # one prompt, its pages in any order
            page = torch.randperm(pages, generator=g, device="cuda")
            at = torch.arange(t, device="cuda")
            s["slots"] = page[at // ps] * ps + at % ps
            s["positions"] = at.to(torch.int32)
        angle = torch.arange(max(4096, t), device="cuda")[:, None] * 10000.0 ** (-torch.arange(0, case["rotated"], 2, device="cuda") / case["rotated"])
        s["cos"], s["sin"] = angle.cos(), angle.sin()
        s["q_out"] = torch.empty((t, case["q_heads"], d), dtype=dt, device="cuda")
    elif case["op"] == "prompt":
        lens = _lengths(case)
        keys = [n + case["past"] for n in lens]
        s["q"], s["k"], s["v"] = _qkv(g, sum(lens), sum(keys), case)
        s["cu_q"], s["cu_k"], s["max_q"], s["max_k"] = _starts(lens), _starts(keys), max(lens), max(keys)
        s["out"] = torch.empty((sum(lens), case["q_heads"], d), dtype=dt, device="cuda")
        s["lse"] = torch.empty((sum(lens), case["q_heads"]), device="cuda") if case["lse"] else None
    elif case["op"] == "paged":
        lens, ps = _lengths(case), case["page"]
        per = [-(-n // ps) for n in lens]
        pages = sum(per) + 3
        s["q"], k, v = _qkv(g, case["seqs"], 1, dict(case, packed=False))
        s["k_cache"], s["v_cache"] = _randn(g, (pages, case["kv_heads"], ps, d), dt), _randn(g, (pages, case["kv_heads"], ps, d), dt)
        s["k_cache"].add_(k[0, :, None])
        s["v_cache"].add_(v[0, :, None])
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros((case["seqs"], max(per)), dtype=torch.int32, device="cuda")
        used = torch.arange(max(per), device="cuda")[None] < torch.tensor(per, device="cuda")[:, None]
        table[used] = order[:sum(per)]
        s["table"], s["lens"], s["max_len"] = table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens)
        s["out"] = torch.empty((case["seqs"], case["q_heads"], d), dtype=dt, device="cuda")
    else:
        t, h, pdt = case["tokens"], case["heads"], DTYPES[case["part_dtype"]]
        s["parts"] = [_randn(g, (t, h, d), pdt) for _ in range(case["parts"])]
        s["lses"] = [_randn(g, (t, h), torch.float32).mul_(1.5).add_(7.0) for _ in range(case["parts"])]
        s["lses"][-1][torch.rand(t, h, generator=g, device="cuda") < 0.05] = -math.inf      # rows whose keys are all on other peers
        s["out"], s["lse"] = torch.empty((t, h, d), dtype=dt, device="cuda"), torch.empty((t, h), device="cuda")
    if own:
        s["session"] = _session(case)
        if "k_cache" in s:
            from paper_2507_17511_amd.attention import PagedCache
            s["cache"] = PagedCache(s["k_cache"], s["v_cache"])
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)[s["case"]["op"]](s)


def _own_append(s):
    s["session"].append(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], cos=s["cos"], sin=s["sin"],
                        q=s["q"], q_out=s["q_out"], interleaved=s["case"]["style"] == "pairs")
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": s["q_out"]}


def _own_prompt(s):
    s["session"].prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=s["case"]["causal"], out=s["out"], lse=s["lse"], max_k=s["max_k"])
    return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]


def _own_paged(s):
    s["session"].paged(s["cache"], s["q"], s["table"], s["lens"], out=s["out"], max_len=s["max_len"])
    return [s["out"]]


def _own_join(s):
    s["session"].join(s["parts"], s["lses"], out=s["out"], lse=s["lse"])
    return [s["out"], s["lse"]]


_run_own = {"append": _own_append, "prompt": _own_prompt, "paged": _own_paged, "join": _own_join}


def _rotated(x, cos, sin, rotated, style):
    x = x.float()
    if style == "half":
        a, b = x[..., :rotated // 2], x[..., rotated // 2:rotated]
        y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., :rotated:2], x[..., 1:rotated:2]
        y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((y, x[..., rotated:]), -1)


def _plain_append(s):
    c, at = s["case"], s["positions"].long()
    cos, sin = s["cos"][at][:, None], s["sin"][at][:, None]
    page, off, head = (s["slots"] // c["page"])[:, None], (s["slots"] % c["page"])[:, None], torch.arange(c["kv_heads"], device="cuda")[None]
    s["k_cache"][page, head, off] = _rotated(s["k"], cos, sin, c["rotated"], c["style"]).to(s["k_cache"].dtype)
    s["v_cache"][page, head, off] = s["v"]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "q": _rotated(s["q"], cos, sin, c["rotated"], c["style"]).to(s["q"].dtype)}


def _softmax_product(q, k, v, hide):
    """q [B, Hk, R, D], k and v [B, Hk, K, D] fp32, hide [B, 1, R or 1, K]: -> rows' outputs and log-sum-exps; a row without keys gives zeros."""
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(1.0 / math.sqrt(q.shape[-1]))
    if hide is not None:
        p.masked_fill_(hide, -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return o, (total.log() + m).squeeze(-1)


def _plain_prompt(s):
    c, lq, lk = s["case"], s["max_q"], s["max_k"]
    hq, hk, d, n = c["q_heads"], c["kv_heads"], c["dim"], c["seqs"]
    start_q, start_k = s["cu_q"].long(), s["cu_k"].long()
    i, j = torch.arange(lq, device="cuda"), torch.arange(lk, device="cuda")
    at_q = (start_q[:-1, None] + i).clamp_(max=s["q"].shape[0] - 1)
    at_k = (start_k[:-1, None] + j).clamp_(max=s["k"].shape[0] - 1)
    len_q, len_k = start_q.diff(), start_k.diff()
    q = s["q"][at_q].float().view(n, lq, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(n, hk, hq // hk * lq, d)
    k, v = (s[x][at_k].float().transpose(1, 2).contiguous() for x in ("k", "v"))
    hide = None
    if c["causal"] or n > 1:
        hide = (j[None, None] >= len_k[:, None, None]).expand(n, lq, lk)
        if c["causal"]:
            hide = hide | (j[None, None] > i[None, :, None] + (len_k - len_q)[:, None, None])
        hide = hide[:, None, None].expand(n, 1, hq // hk, lq, lk).reshape(n, 1, hq // hk * lq, lk)
    o, lse = _softmax_product(q, k, v, hide)
    token = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.searchsorted(start_q, token, right=True) - 1
    row = token - start_q[seq]
    o = o.view(n, hq, lq, d).transpose(1, 2)[seq, row].to(s["out"].dtype)
    return [o, lse.view(n, hq, lq).transpose(1, 2)[seq, row]] if c["lse"] else [o]


def _plain_paged(s):
    c = s["case"]
    n, hq, hk, d = c["seqs"], c["q_heads"], c["kv_heads"], c["dim"]
    k, v = (s[x][s["table"].long()].transpose(1, 2).reshape(n, hk, -1, d).float() for x in ("k_cache", "v_cache"))
    hide = (torch.arange(k.shape[2], device="cuda")[None] >= s["lens"][:, None])[:, None, None]
    o, _ = _softmax_product(s["q"].float().view(n, hk, hq // hk, d), k, v, hide)
    return [o.reshape(n, hq, d).to(s["q"].dtype)]


def _plain_join(s):
    lse = torch.stack(s["lses"])
    m = lse.amax(0)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    w = (lse - m).exp_()
    total = w.sum(0)
    o = (torch.stack(s["parts"]).float() * w[..., None]).sum(0) / torch.where(total == 0, torch.ones_like(total), total)[..., None]
    return [o.to(s["out"].dtype), total.log() + m]


_run_plain = {"append": _plain_append, "prompt": _plain_prompt, "paged": _plain_paged, "join": _plain_join}


# ---------------------------------------------------------------- the definition, in 64 bits

def _attend64(q, k, v, visible):
    """q [R, D], k and v [K, D] in fp64; row r sees the first visible[r] keys (None: all).  -> outputs, log-sum-exps."""
    score = (q @ k.t().contiguous()) / math.sqrt(q.shape[1])
    if visible is not None:
        score = torch.where(torch.arange(k.shape[0], device="cuda")[None] < visible[:, None], score, torch.full_like(score, -math.inf))
    lse = torch.logsumexp(score, 1)
    score -= torch.where(lse.isinf(), torch.zeros_like(lse), lse)[:, None]
    return score.exp_() @ v, lse


def exact(case, seed):
    s = prepare(case, seed)
    d = case["dim"]
    if case["op"] == "append":
        r, at = case["rotated"], s["positions"].long()
        c, z = s["cos"].double()[at][:, None], s["sin"].double()[at][:, None]
        first = torch.arange(r // 2, device="cuda") * (1 if case["style"] == "half" else 2)
        second = first + (r // 2 if case["style"] == "half" else 1)
        q, k = s["q"].double(), s["k"].double()
        for x in (q, k):
            a, b = x[..., first].clone(), x[..., second].clone()
            x[..., first], x[..., second] = a * c - b * z, a * z + b * c
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        by_slot_k, by_slot_v = kc.transpose(1, 2).reshape(-1, case["kv_heads"], d), vc.transpose(1, 2).reshape(-1, case["kv_heads"], d)
        by_slot_k[s["slots"]], by_slot_v[s["slots"]] = k, s["v"].double()
        back = [x.view(-1, case["page"], case["kv_heads"], d).transpose(1, 2).contiguous() for x in (by_slot_k, by_slot_v)]
        return {"k_cache": back[0], "v_cache": back[1], "q": q}
    if case["op"] == "join":
        lse = torch.stack([x.double() for x in s["lses"]])
        total = torch.logsumexp(lse, 0)
        o = sum(torch.exp(l - total)[..., None] * p.double() for l, p in zip(lse, s["parts"]))
        return [o, total]
    group = case["q_heads"] // case["kv_heads"]
    lens = _lengths(case)
    out, lses = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda"), torch.empty(s["out"].shape[:2], dtype=torch.float64, device="cuda")
    q0 = k0 = 0
    for b, n in enumerate(lens):
        if case["op"] == "paged":
            rows, at = 1, torch.arange(n, device="cuda")
            page = s["table"][b].long()[at // case["page"]]
            keys, values = s["k_cache"][page, :, at % case["page"]], s["v_cache"][page, :, at % case["page"]]
            visible = None
        else:
            rows, nk = n, n + case["past"]
            keys, values = s["k"][k0:k0 + nk], s["v"][k0:k0 + nk]
            visible = torch.arange(n, device="cuda") + case["past"] + 1 if case["causal"] else None
            k0 += nk
        for h in range(case["q_heads"]):
            o, l = _attend64(s["q"][q0:q0 + rows, h].double(), keys[:, h // group].double(), values[:, h // group].double(), visible)
            out[q0:q0 + rows, h], lses[q0:q0 + rows, h] = o, l
        q0 += rows
    return [out, lses] if case["op"] == "prompt" and case["lse"] else [out]
