"""A bounded 4-bit context: what retrieval puts before the model, held in a fixed size.

An agent's retrieved records and its own tokens enter the model's key/value cache
chunk by chunk.  ``BoundedContext`` holds that cache in 4 bits and in at most
``budget`` tokens a sequence: each step quantizes the new keys and values into it
(``kv_append``), attends over it while it counts what every cached token receives
(``kv_attend`` with weights), and gives up the tokens that received least
(``kv_evict``); the first and the newest tokens stay in any case.

    python examples/bounded_context.py [--tokens 8192] [--budget 2048] [--seqs 8]

runs a stream of synthetic keys, values and queries through it: prompts in chunks,
then single tokens, with the time of both, the size of the cache, and how near the
results are to attention over everything in full precision.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_32256_amd as lam  # noqa: E402


class BoundedContext:
    """The key/value cache of ``n_seqs`` sequences of one layer.  A step takes at most
    ``chunk`` tokens a sequence."""

    def __init__(self, n_seqs: int, kv_heads: int, head_dim: int, budget: int, chunk: int, recent: int = 0,
                 sinks: int = 0, page_size: int = 64, device="cuda"):
        self.budget, self.chunk, self.recent, self.sinks, self.head_dim = budget, chunk, recent, sinks, head_dim
        slots = budget + chunk
        per_seq = -(-slots // page_size)
        self.pages = lam.kv_pages(n_seqs * per_seq, kv_heads, head_dim, page_size, device=device)
        self.table = torch.arange(n_seqs * per_seq, dtype=torch.int32, device=device).view(n_seqs, per_seq)
        self.weights = torch.zeros((n_seqs, kv_heads, slots), device=device)
        self.positions = torch.full((n_seqs, kv_heads, slots), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(n_seqs, dtype=torch.int32, device=device)   # cached tokens
        self.lengths_next = torch.zeros_like(self.lengths)   # their own memory, see step()
        self.seen = torch.zeros(n_seqs, dtype=torch.int32, device=device)      # tokens so far: the next position
        self.status = torch.zeros(3, dtype=torch.int32, device=device)

    def step(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> torch.Tensor:
        """The next n tokens of every sequence, sequence after sequence: q (n_seqs * n,
        q_heads, head_dim), k and v likewise with kv_heads.  Returns their attention."""
        n, rest = divmod(q.shape[0], self.lengths.shape[0])
        if rest or n > self.chunk:
            raise ValueError(f"a step takes the same number of tokens of every sequence, at most {self.chunk}")
        self.lengths += n
        lam.kv_append(k, v, self.pages, self.table, self.lengths, weights=self.weights, positions=self.positions,
                      first=self.seen, status=self.status)
        self.seen += n
        out = lam.kv_attend(q, self.pages, self.table, self.lengths, weights=self.weights)
        # No sequence has more than budget + n tokens here.  With columns for those alone, and new
        # lengths in memory of their own, the eviction after a few tokens is one launch.
        slots = self.budget + n
        lam.kv_evict(self.pages, self.table, self.lengths, self.weights[..., :slots], self.budget, self.head_dim,
                     recent=self.recent, sinks=self.sinks, positions=self.positions[..., :slots],
                     out=(self.weights, self.positions, self.lengths_next))
        self.lengths, self.lengths_next = self.lengths_next, self.lengths
        return out

    def check(self) -> None:
        """Raise if a step met input that it could not hold (waits for the device)."""
        bad, over, lost = self.status.tolist()
        if bad or over or lost:
            raise ValueError(f"non-finite: {bad}, out of range: {over}, without a place: {lost}")

    def bytes(self) -> int:
        return self.pages.numel()


def stream(n_seqs, tokens, kv_heads, q_heads, head_dim, seed=0, device="cuda"):
    """Keys, values and queries of a stream in which a few tokens are often attended to."""
    g = torch.Generator(device=device).manual_seed(seed)
    k = torch.randn((tokens, n_seqs, kv_heads, head_dim), generator=g, device=device)
    v = torch.randn(k.shape, generator=g, device=device)
    q = torch.randn((tokens, n_seqs, q_heads, head_dim), generator=g, device=device)
    topic = torch.randn((1, n_seqs, kv_heads, head_dim), generator=g, device=device)
    marked = torch.rand((tokens, n_seqs, kv_heads, 1), generator=g, device=device) < 0.05
    k = torch.where(marked, 0.6 * k + 0.8 * topic, k)
    q += 0.7 * topic.repeat_interleave(q_heads // kv_heads, dim=2)
    return tuple(x.to(torch.bfloat16) for x in (q, k, v))


def attention(q, k, v):
    """Plain attention in float32 of one token q (seqs, q_heads, D) over k, v (t, seqs, kv_heads, D)."""
    group = q.shape[1] // k.shape[2]
    k, v = (x.float().permute(1, 2, 0, 3).repeat_interleave(group, dim=1) for x in (k, v))
    p = torch.softmax((k @ q.float()[..., None]).squeeze(-1) * q.shape[-1] ** -0.5, dim=-1)
    return (p[:, :, None, :] @ v).squeeze(2)


def run(tokens, budget, n_seqs, chunk=512, decode=64, kv_heads=8, q_heads=32, head_dim=128, recent=None, sinks=4,
        seed=0):
    """Prompts of ``tokens`` tokens, then ``decode`` single ones.  A dict of what was measured."""
    q, k, v = stream(n_seqs, tokens + decode, kv_heads, q_heads, head_dim, seed)
    ctx = BoundedContext(n_seqs, kv_heads, head_dim, budget, chunk, budget // 4 if recent is None else recent, sinks)

    def rows(x, a, b):
        return x[a:b].transpose(0, 1).flatten(0, 1)

    torch.cuda.synchronize()
    began = time.perf_counter()
    for a in range(0, tokens, chunk):
        b = min(tokens, a + chunk)
        ctx.step(rows(q, a, b), rows(k, a, b), rows(v, a, b))
    torch.cuda.synchronize()
    prompt_s = time.perf_counter() - began
    began = time.perf_counter()
    for t in range(tokens, tokens + decode):
        out = ctx.step(q[t], k[t], v[t])
    torch.cuda.synchronize()
    decode_s = time.perf_counter() - began
    ctx.check()
    last = tokens + decode
    full = attention(q[last - 1], k[:last], v[:last])
    error = ((out.float() - full).norm() / full.norm()).item()
    return dict(prompt_tokens_per_s=n_seqs * tokens / prompt_s, decode_steps_per_s=decode / decode_s,
                cache_bytes=ctx.bytes(), full_bytes=4 * k[:last].numel(), cached=ctx.lengths.tolist(),
                relative_error=error)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=8192)
    p.add_argument("--budget", type=int, default=2048)
    p.add_argument("--seqs", type=int, default=8)
    a = p.parse_args()
    run(1024, 512, a.seqs, decode=4)   # the first calls load the kernels
    r = run(a.tokens, a.budget, a.seqs)
    print(f"prompts: {r['prompt_tokens_per_s']:.0f} tokens/s; single tokens: {r['decode_steps_per_s']:.0f} steps/s "
          f"of {a.seqs} sequences")
    print(f"cache: {r['cache_bytes'] / 1e6:.1f} MB against {r['full_bytes'] / 1e6:.1f} MB of every token in 16 bits")
    print(f"last token against attention over everything: relative error {r['relative_error']:.3f}")


if __name__ == "__main__":
    main()
