"""Norm, rotation, append and windowed attention together, as examples/streaming_context.py uses
them, against the same steps in binary64: pages go back to the pool and are taken again, and what
they held before does not matter.  Tolerances as in test_gpu_kv_attend.py (bfloat16), where the
queries are those that the library has turned (test_gpu_kv_rotate.py)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import kv
from test_gpu_kv_attend import Case

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example(lam):
    spec = importlib.util.spec_from_file_location("streaming_context", os.path.join(ROOT, "examples", "streaming_context.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("window,sinks,steps", [
    (70, 4, (5, 60, 1, 1, 40, 1, 64, 1, 1, 1)), (33, 0, (64, 64, 64, 1)), (1, 40, (1,) * 12 + (64, 1)), (500, 70, (64,) * 6),
])
def test_steps(lam, example, window, sinks, steps):
    B, Hq, Hk, D, T = 2, 6, 2, 64, 32
    g = torch.Generator(device="cuda").manual_seed(window)
    gains = [torch.rand(D, generator=g, device="cuda") + 0.5 for _ in range(2)]
    ctx = example.StreamingContext(B, Hq, Hk, D, window, sinks, 64, sum(steps), *gains, page_size=T)
    ctx.pages.fill_(255)
    ks, vs, at = [[] for _ in range(B)], [[] for _ in range(B)], 0
    freq = ctx.frequencies.cpu().numpy()
    for n in steps:
        x = torch.randn((B * n, Hq + 2 * Hk, D), generator=g, device="cuda").to(torch.bfloat16)
        out = ctx.step(x)
        pos = list(range(at, at + n))
        at += n
        q = lam.kv_rotate(x[:, :Hq], ctx.frequencies, torch.tensor(pos * B, dtype=torch.int32, device="cuda"), q_norm=gains[0])
        for b in range(B):
            mine = slice(b * n, b * n + n)
            ks[b].append(kv.rounded(kv.rotate(_np(x[mine, Hq:Hq + Hk]), pos, freq, gain=_np(gains[1]))[0]))
            vs[b].append(kv.rounded(_np(x[mine, Hq + Hk:])))
        c = Case.__new__(Case)
        c.D, c.Hk, c.G, c.dt, c.rows, c.lens = D, Hk, Hq // Hk, "bf16", [n] * B, [at] * B
        c.q, c.starts = q, [n * b for b in range(B + 1)]
        c.k, c.v = [np.concatenate(k) for k in ks], [np.concatenate(v) for v in vs]
        c.check(out, mask=[[kv.in_window(n, at, window, sinks)]] * B)
    ctx.check()
    used = int((ctx.table >= 0).sum())
    assert used <= ctx.pages.shape[0] and len(set(ctx.table[ctx.table >= 0].tolist())) == used


def test_the_example_runs(example):
    r = example.run(700, 128, 3, chunk=256, decode=5, q_heads=8, kv_heads=2, head_dim=64)
    assert r["pages"] < r["pages_of_all"] and r["relative_error"] < 1


def test_bad_steps(example):
    ctx = example.StreamingContext(2, 4, 2, 64, 32, 1, 16, 40)
    x = torch.zeros((2, 8, 64), dtype=torch.bfloat16, device="cuda")
    for rows in (3, 34, 0):
        with pytest.raises(ValueError):
            ctx.step(x[:1].expand(rows, 8, 64))
    x[1, 5, 3] = float("nan")
    ctx.step(x)
    with pytest.raises(ValueError):
        ctx.check()
