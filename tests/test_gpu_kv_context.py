"""The operators of the 4-bit cache together, as examples/bounded_context.py uses
them, against the same steps in binary64: append, attention with accumulated
weights and eviction over a stream, until the selection by weights would depend on
rounding; and without eviction, against attention over all rounded tokens.

Tolerances as in test_gpu_kv_attend.py (bfloat16)."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import kv

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example(lam):
    spec = importlib.util.spec_from_file_location("bounded_context", os.path.join(ROOT, "examples", "bounded_context.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


class Plain:
    """One head's bounded context in binary64; positions, and weights a slot."""

    def __init__(self, budget, recent, sinks):
        self.budget, self.recent, self.sinks = budget, recent, sinks
        self.k, self.v, self.w, self.pos, self.seen = [], [], [], [], 0

    def step(self, q, k, v, slots):
        """q [heads of the group][n][D]; slots: which old slot each new one took, as the
        library chose.  (results, whether its choice is right up to rounding)"""
        for a, b in zip(k, v):
            self.k.append(a), self.v.append(b), self.w.append(0.0), self.pos.append(self.seen)
            self.seen += 1
        rs = [kv.attend(x, np.array(self.k), np.array(self.v), x.shape[-1] ** -0.5) for x in q]
        self.w = list(np.array(self.w) + sum(r["p"].sum(0) for r in rs))
        ok = True
        if len(self.k) > self.budget:
            chosen = sorted(slots)
            want = kv.evict(self.w, self.pos, self.budget, self.recent, self.sinks)
            # slots that one side keeps and the other does not differ by rounding only
            odd = set(chosen) ^ set(want)
            if odd:
                ws = [self.w[t] for t in odd]
                ok = max(ws) - min(ws) <= 1e-4 * max(ws)
            kept = list(slots)
            for name in ("k", "v", "w", "pos"):
                x = getattr(self, name)
                setattr(self, name, [x[t] for t in kept])
        return rs, ok


def test_stream_against_plain_steps(example, lam):
    n_seqs, Hk, G, D, budget, chunk, recent, sinks = 2, 2, 2, 64, 96, 40, 16, 2
    q, k, v = example.stream(n_seqs, 300, Hk, Hk * G, D, seed=3)
    ctx = example.BoundedContext(n_seqs, Hk, D, budget, chunk, recent, sinks, page_size=32)
    plain = [[Plain(budget, recent, sinks) for _ in range(Hk)] for _ in range(n_seqs)]
    at = 0
    for n in (40, 1, 17, 40, 1, 1, 1, 33, 2, 40, 1, 1):
        ids = ctx.seen.clone()
        part = [x[at:at + n].transpose(0, 1).flatten(0, 1) for x in (q, k, v)]
        out = _np(ctx.step(*part)).reshape(n_seqs, n, Hk * G, D)
        pos = ctx.positions.cpu().numpy()
        lens = ctx.lengths.tolist()
        for s in range(n_seqs):
            assert lens[s] == min(budget, len(plain[s][0].k) + n)
            for h in range(Hk):
                p = plain[s][h]
                # where the library put each position, told by the positions it keeps
                before = {x: t for t, x in enumerate(p.pos + list(range(p.seen, p.seen + n)))}
                slots = [before[int(x)] for x in pos[s, h, : lens[s]]]
                assert len(set(slots)) == len(slots)
                qs = [_np(q[at:at + n, s, j]) for j in range(h * G, (h + 1) * G)]
                rs, ok = p.step(qs, kv.rounded(_np(k[at:at + n, s, h])), kv.rounded(_np(v[at:at + n, s, h])), slots)
                assert ok
                for j, r in enumerate(rs):
                    d = r["slack"] * (D + 8) * 2.0 ** -24 + 2.0 ** -20
                    tol = 2.0 ** -8 * np.abs(r["out"]) + (2.0 ** -11 + 2 * d)[:, None] * r["mean"] + 2.0 ** -32 * r["total"]
                    assert (np.abs(out[s, :, h * G + j] - r["out"]) <= tol).all()
                w = ctx.weights[s, h, : lens[s]].cpu().numpy().astype(np.float64)
                assert np.allclose(w, p.w, rtol=1e-4, atol=1e-6)
        at += n
        assert torch.equal(ctx.seen, ids + n)
    ctx.check()


def test_run_reports(example):
    r = example.run(300, 4096, 2, chunk=128, decode=3, kv_heads=2, q_heads=4, head_dim=128)
    assert r["cached"] == [303, 303] and r["relative_error"] < 0.5      # nothing evicted: 4-bit rounding alone
    r = example.run(900, 256, 2, chunk=128, decode=3, kv_heads=2, q_heads=4, head_dim=128)
    assert r["cached"] == [256, 256]


def test_bad_steps_are_refused_or_reported(example):
    ctx = example.BoundedContext(2, 1, 64, 64, 16)
    q = torch.zeros((2, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        ctx.step(q[:1], q[:1], q[:1])
    with pytest.raises(ValueError):
        ctx.step(*(x.repeat(17, 1, 1) for x in (q, q, q)))
    k = q.clone()
    k[0, 0, 5] = float("nan")
    ctx.step(q, k, q)
    with pytest.raises(ValueError):
        ctx.check()


def test_a_step_of_few_tokens_evicts_in_one_launch(example, lam):
    """Whatever chunk the context has room for: the tokens given up are moved by the launch that
    selects them."""
    n_seqs, budget, chunk = 2, 128, 512
    ctx = example.BoundedContext(n_seqs, 1, 64, budget, chunk, recent=8, sinks=2)
    q, k, v = example.stream(n_seqs, 300, 1, 2, 64, seed=5)

    def step(at, n):
        return ctx.step(*(x[at:at + n].transpose(0, 1).flatten(0, 1) for x in (q, k, v)))

    step(0, 250)
    lib = lam.default_context()
    lib.profile(True)
    lib.profile_reset()
    step(250, 1)
    step(251, 40)
    lib.synchronize()
    selects, moves = lib.profile_read("kv_select")[1], lib.profile_read("kv_move")[1]
    lib.profile(False)
    assert (selects, moves) == (2, 0)
    assert ctx.lengths.tolist() == [budget] * n_seqs
    newest = set(range(291 - 8, 291))
    for s in range(n_seqs):
        assert newest <= set(ctx.positions[s, 0, :budget].tolist())
