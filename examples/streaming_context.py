"""A stream of any length over a fixed number of pages: the newest tokens and the first.

``StreamingContext`` holds the keys and values of one attention layer in 4 bits.  A step takes the
layer's projections of its next tokens, as one product leaves them (queries, keys and values side by
side): heads are normed and turned by their positions on the way into the cache, the queries with them
(``kv_rotate_append``), and each token attends over the last ``window`` tokens and the first ``sinks``
(``kv_attend``).  A page that the window has left behind goes back to the pool.

    python examples/streaming_context.py [--tokens 32768] [--window 2048] [--seqs 8]

runs synthetic projections through it: prompts in chunks, then single tokens, with the time of both,
the pages in use, and how near the last results are to attention in full precision over the same window.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_32256_amd as lam  # noqa: E402


class StreamingContext:
    """The cache of ``n_seqs`` sequences of one layer that grow together, at most ``chunk`` tokens a step
    and ``longest`` in all."""

    def __init__(self, n_seqs, q_heads, kv_heads, head_dim, window, sinks, chunk, longest, q_norm=None, k_norm=None,
                 page_size=64, rotary=None, device="cuda"):
        self.heads, self.head_dim = (q_heads, kv_heads), head_dim
        self.window, self.sinks, self.chunk, self.page_size = window, sinks, chunk, page_size
        self.q_norm, self.k_norm = q_norm, k_norm
        self.frequencies, self.amplitude = rotary or lam.rotary_frequencies(head_dim, device=device)
        # a step's rows see the window of the first of them; pages are partly used at both ends
        self.front = -(-sinks // page_size)
        per_seq = self.front + (window + chunk - 2) // page_size + 2
        self.pages = lam.kv_pages(n_seqs * per_seq, kv_heads, head_dim, page_size, device=device)
        self.table = torch.full((n_seqs, -(-longest // page_size)), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(n_seqs, dtype=torch.int32, device=device)
        self.status = torch.zeros(3, dtype=torch.int32, device=device)
        self.free = torch.arange(n_seqs * per_seq, dtype=torch.int32, device=device).view(per_seq, n_seqs)
        self.n_free, self.length, self.left = per_seq, 0, self.front   # left: first column not given back yet

    def step(self, projections: torch.Tensor) -> torch.Tensor:
        """projections: (n_seqs * n, q_heads + 2 kv_heads, head_dim), sequence after sequence.
        Returns the attention (n_seqs * n, q_heads, head_dim)."""
        n, rest = divmod(projections.shape[0], self.lengths.shape[0])
        if rest or not 0 < n <= self.chunk or self.length + n > self.table.shape[1] * self.page_size:
            raise ValueError(f"a step takes the same number of tokens of every sequence, at most {self.chunk}, while there is room")
        q, k, v = projections.split((self.heads[0], self.heads[1], self.heads[1]), dim=1)
        # pages that no row of this step or a later one sees go back, then new ones are taken
        behind = max(self.length - self.window + 1, 0) // self.page_size
        for col in range(self.left, behind):
            self.free[self.n_free] = self.table[:, col]
            self.table[:, col] = -1
            self.n_free += 1
        self.left = max(self.left, behind)
        for col in range(-(-self.length // self.page_size), -(-(self.length + n) // self.page_size)):
            self.n_free -= 1
            self.table[:, col] = self.free[self.n_free]
        self.length += n
        self.lengths += n
        q = lam.kv_rotate_append(q, k, v, self.pages, self.table, self.lengths, self.frequencies, amplitude=self.amplitude,
                                 q_norm=self.q_norm, k_norm=self.k_norm, status=self.status)
        return lam.kv_attend(q, self.pages, self.table, self.lengths, window=self.window, sinks=self.sinks,
                             max_length=self.length)

    def check(self) -> None:
        """Raise if a step met input that it could not hold (waits for the device)."""
        bad, over, lost = self.status.tolist()
        if bad or over or lost:
            raise ValueError(f"non-finite: {bad}, out of range: {over}, without a place: {lost}")


def turned(x, gain, positions, frequencies, amplitude):
    """Heads normed and turned in halves, in float64."""
    x = x.double()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain.double()
    a = positions.double()[:, None, None] * frequencies
    u, v = x.chunk(2, dim=-1)
    return amplitude * torch.cat([u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()], dim=-1)


def run(tokens, window, n_seqs, chunk=1024, decode=64, q_heads=32, kv_heads=8, head_dim=128, sinks=4, seed=0):
    """Prompts of ``tokens`` tokens, then ``decode`` single ones.  A dict of what was measured."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    heads, last = q_heads + 2 * kv_heads, tokens + decode
    x = torch.randn((n_seqs, last, heads, head_dim), generator=g, device="cuda").to(torch.bfloat16)
    gains = [1 + 0.1 * torch.randn(head_dim, generator=g, device="cuda") for _ in range(2)]
    ctx = StreamingContext(n_seqs, q_heads, kv_heads, head_dim, window, sinks, chunk, last, *gains)
    steps = [x[:, a:min(a + chunk, tokens)].flatten(0, 1) for a in range(0, tokens, chunk)]
    steps += [x[:, t] for t in range(tokens, last)]
    times = []
    for part in (steps[:-decode], steps[-decode:]):
        torch.cuda.synchronize()
        began = time.perf_counter()
        for s in part:
            out = ctx.step(s)
        torch.cuda.synchronize()
        times.append(time.perf_counter() - began)
    ctx.check()
    at = torch.tensor(sorted(set(range(min(sinks, last))) | set(range(max(0, last - window), last))), device="cuda")
    error = 0.0
    for b in range(n_seqs):
        q = turned(x[b, -1:, :q_heads], gains[0], at[-1:], ctx.frequencies, ctx.amplitude)[0]
        k = turned(x[b, at, q_heads:q_heads + kv_heads], gains[1], at, ctx.frequencies, ctx.amplitude)
        k, v = (y.repeat_interleave(q_heads // kv_heads, dim=1) for y in (k, x[b, at, q_heads + kv_heads:].double()))
        p = torch.softmax((k * q).sum(-1) * head_dim ** -0.5, dim=0)
        want = (p[..., None] * v).sum(0)
        error = max(error, ((out[b].double() - want).norm() / want.norm()).item())
    return dict(prompt_tokens_per_s=n_seqs * tokens / times[0], decode_steps_per_s=decode / times[1],
                pages=ctx.pages.shape[0], pages_of_all=n_seqs * ctx.table.shape[1], relative_error=error)


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--tokens", type=int, default=32768)
    p.add_argument("--window", type=int, default=2048)
    p.add_argument("--seqs", type=int, default=8)
    a = p.parse_args()
    run(2048, 512, a.seqs, decode=4)   # the first calls load the kernels
    r = run(a.tokens, a.window, a.seqs)
    print(f"prompts: {r['prompt_tokens_per_s']:.0f} tokens/s; single tokens: {r['decode_steps_per_s']:.0f} steps/s "
          f"of {a.seqs} sequences")
    print(f"pages: {r['pages']} against {r['pages_of_all']} of every token")
    print(f"last token against the same window in full precision: relative error {r['relative_error']:.3f}")


if __name__ == "__main__":
    main()
