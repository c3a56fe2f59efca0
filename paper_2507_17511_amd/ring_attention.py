"""Sequence-parallel attention over compressed keys and values, and decoding from the cache they fill: every attention
entry point next to the codec, as a serving program would run them.

    python -m paper_2507_17511_amd.ring_attention

`peers` devices hold a shard of one layer's tokens each (they take turns on one GPU here; the packed codes in its memory stand in for the
wire).  In every step each peer sends its keys and values through the codec, and attends its own queries to one shard after
another -- its own as they are, the others as reconstructed -- joining the hops by their log-sum-exps (arxiv 2507.17511, App. B
Alg. 2); a hop's output is rounded to bf16 before that.  After the last step one peer takes all keys and values into a paged cache, rotated by their positions, and decodes
tokens from it.  Inputs are synthetic; the command prints how far each result is from fp32 attention over the same keys and values.
"""
from __future__ import annotations

import argparse
import math
from typing import List

import torch

import paper_2507_17511_amd as cf
from paper_2507_17511_amd.attention import AttentionSession, PagedCache
from paper_2507_17511_amd.session import CodecSession


class RingAttention:
    """One layer's exchange among `peers`: tokens / peers tokens each, 2-bit codes with channel scales."""

    def __init__(self, peers: int, tokens: int, q_heads: int, kv_heads: int, head_dim: int, device: str | torch.device = "cuda:0"):
        if tokens % peers:
            raise ValueError("every peer has as many tokens")
        self.peers, self.shard, self.kv_heads, self.head_dim = peers, tokens // peers, kv_heads, head_dim
        desc = cf.desc(self.shard, kv_heads * head_dim, cf.CF_BF16, 2, cf.CF_SCALE_CHANNEL)
        self.codec = CodecSession([desc] * (2 * peers), device=device)          # K and V of every peer
        self.attention = AttentionSession(q_heads, kv_heads, head_dim, device=device)
        self.cu = torch.tensor([0, self.shard], dtype=torch.int32, device=device)

    def exchange(self, k: List[torch.Tensor], v: List[torch.Tensor], first: bool):
        """Sends every peer's K and V.  -> what the others have of them: reconstructions, exact after the first step."""
        x = [t.view(self.shard, -1) for pair in zip(k, v) for t in pair]
        if first:
            self.codec.warmup(x)
        else:
            self.codec.step_fused(x)
        shape = (self.shard, self.kv_heads, self.head_dim)
        return [t.view(shape) for t in self.codec.recon[0::2]], [t.view(shape) for t in self.codec.recon[1::2]]

    def attend(self, peer: int, q: torch.Tensor, k: List[torch.Tensor], v: List[torch.Tensor], own_k: torch.Tensor, own_v: torch.Tensor) -> torch.Tensor:
        """Attention of one peer's queries over all shards, hop by hop: its own first, then those of the peers behind it."""
        parts, lses = [], []
        for hop in range(self.peers):
            from_peer = (peer - hop) % self.peers
            kk, vv = (own_k, own_v) if hop == 0 else (k[from_peer], v[from_peer])
            lses.append(torch.empty(q.shape[:2], device=q.device))
            parts.append(self.attention.prompt(q, kk, vv, self.cu, causal=False, lse=lses[-1], max_k=self.shard))
        return self.attention.join(parts, lses)

    def close(self) -> None:
        self.codec.close()


def rotation(positions: int, rotary_dim: int, device, base: float = 10000.0):
    angle = torch.arange(positions, device=device)[:, None] * base ** (-torch.arange(0, rotary_dim, 2, device=device) / rotary_dim)
    return angle.cos(), angle.sin()


def plain_attention(q, k, v):
    """fp32 attention [tokens, heads, dim] over all keys: what the results are compared with."""
    group = q.shape[1] // k.shape[1]
    k, v = (x.float().repeat_interleave(group, 1).transpose(0, 1).contiguous() for x in (k, v))
    s = torch.matmul(q.float().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(q.shape[2])
    return torch.matmul(torch.softmax(s, -1), v).transpose(0, 1)


def apart(x, y) -> float:
    return float((x.float() - y.float()).norm() / y.float().norm())


def run(peers: int = 4, tokens: int = 4096, q_heads: int = 24, kv_heads: int = 24, head_dim: int = 128, steps: int = 4, decode: int = 8,
        page_size: int = 64, device: str = "cuda:0", say=print):
    """-> (worst distance of a ring step from attention over the same keys and values, from attention over the uncompressed ones, and of a decoded token)."""
    g = torch.Generator(device=device)
    g.manual_seed(11)
    ring = RingAttention(peers, tokens, q_heads, kv_heads, head_dim, device)
    n = ring.shard

    def randn(heads):
        return torch.randn(n, heads, head_dim, generator=g, device=device)

    state = [(randn(q_heads), randn(kv_heads), randn(kv_heads)) for _ in range(peers)]
    worst = [0.0, 0.0, 0.0]
    for step in range(steps):
        q, k, v = ([s[i].to(torch.bfloat16) for s in state] for i in range(3))
        recon_k, recon_v = ring.exchange(k, v, step == 0)
        for peer in range(peers):
            out = ring.attend(peer, q[peer], recon_k, recon_v, k[peer], v[peer])
            seen_k, seen_v = ([own[p] if p == peer else got[p] for p in range(peers)] for own, got in ((k, recon_k), (v, recon_v)))
            worst[0] = max(worst[0], apart(out, plain_attention(q[peer], torch.cat(seen_k), torch.cat(seen_v))))
            if step == steps - 1:
                worst[1] = max(worst[1], apart(out, plain_attention(q[peer], torch.cat(k), torch.cat(v))))
        state = [tuple(x + 0.03 * torch.randn(x.shape, generator=g, device=device) for x in s) for s in state]
    say(f"ring attention: {peers} peers x {n} tokens, {q_heads} heads of {head_dim}: {worst[0]:.2e} from fp32 over the same keys and values, "
        f"{worst[1]:.2e} from fp32 over the uncompressed ones")

    # the cache: all keys and values, rotated, on pages in any order; then one token after another
    total = tokens + decode
    pages = -(-total // page_size)
    cache = PagedCache.empty(pages + 2, kv_heads, head_dim, page_size, device=device)
    table = torch.randperm(pages + 2, generator=g, device=device)[None, :pages].to(torch.int32)
    cos, sin = rotation(total, head_dim, device)
    att, at = ring.attention, torch.arange(total, device=device)
    slots = table[0].long()[at // page_size] * page_size + at % page_size
    at = at.to(torch.int32)
    all_k, all_v = torch.cat(recon_k), torch.cat(recon_v)
    att.append(cache, all_k, all_v, slots[:tokens], at[:tokens], cos, sin)
    for i in range(tokens, total):
        q, k, v = (torch.randn(1, h, head_dim, generator=g, device=device).to(torch.bfloat16) for h in (q_heads, kv_heads, kv_heads))
        here = slice(i, i + 1)
        turned = att.append(cache, k, v, slots[here], at[here], cos, sin, q=q)
        out = att.paged(cache, turned, table, torch.tensor([i + 1], dtype=torch.int32, device=device), max_len=total)
        used = table[0].long()
        keys, values = (x[used].transpose(1, 2).reshape(-1, kv_heads, head_dim)[:i + 1] for x in (cache.k, cache.v))
        worst[2] = max(worst[2], apart(out, plain_attention(turned, keys, values)))
        all_v = torch.cat((all_v, v))
    if not torch.equal(values, all_v):
        raise RuntimeError("the cache does not hold the appended values")
    say(f"decoded {decode} tokens from {pages} pages of {page_size}: {worst[2]:.2e} from fp32")
    ring.close()
    return tuple(worst)


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--peers", type=int, default=4)
    p.add_argument("--tokens", type=int, default=4096)
    p.add_argument("--q-heads", type=int, default=24)
    p.add_argument("--kv-heads", type=int, default=24)
    p.add_argument("--head-dim", type=int, default=128)
    p.add_argument("--steps", type=int, default=4)
    p.add_argument("--decode", type=int, default=8)
    a = p.parse_args()
    run(a.peers, a.tokens, a.q_heads, a.kv_heads, a.head_dim, a.steps, a.decode)


if __name__ == "__main__":
    main()
