"""Attention over the 4-bit cache on the GPU against the binary64 oracle.

Tolerances, per element: half a unit in the last place of the output's type
(2^-8 of bfloat16's and 2^-11 of float16's value), the weights' rounding to
float16 before they meet the values (2^-11 of sum p |v|, which bounds the sum of
their errors, and for the smallest, which are below float16's normal numbers,
2^-32 of sum |v|: half of float16's last place, 2^-25, where the largest weight is
at least 2^7), and the scores' float32 error (D + 8 roundings of 2^-24 against
the largest scale * sum |q k| of the row, which moves p by twice that relative;
2^-20 covers the exponential and the sums).
"""
import math

import numpy as np
import pytest
import torch

from oracle import kv

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    """Sequences in a cache whose unwritten bytes are all 0xFF (scales that are not numbers)."""

    def __init__(self, lam, D, T, Hk, G, dt, rows, lens, seed=0, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lam, self.D, self.T, self.Hk, self.G, self.dt = lam, D, T, Hk, G, dt
        self.rows, self.lens, B = rows, lens, len(lens)
        cols = max(1, -(-max(lens) // T))
        perm = np.random.default_rng(seed).permutation(B * cols + 2)[: B * cols]
        self.table = _i32(perm.reshape(B, cols).tolist())
        self.pool = torch.full((B * cols + 2, Hk, kv.page_bytes(D, T)), 255, dtype=torch.uint8, device="cuda")
        def draw(n, h):
            return torch.randn((n, h, D), generator=g, device="cuda").to(DT[dt])
        starts = np.concatenate([[0], np.cumsum(lens)])
        k, v = draw(starts[-1], Hk), draw(starts[-1], Hk)
        self.lengths = _i32(lens)
        lam.kv_append(k, v, self.pool, self.table, self.lengths, starts=_i32(starts.tolist()))
        self.k = [kv.rounded(_np(k[starts[b]:starts[b + 1]])) for b in range(B)]
        self.v = [kv.rounded(_np(v[starts[b]:starts[b + 1]])) for b in range(B)]
        self.q = (draw(sum(rows), Hk * G) * spread).to(DT[dt])
        self.starts = np.concatenate([[0], np.cumsum(rows)])

    def call(self, **kw):
        st = None if len(set(self.rows)) == 1 and not kw.pop("force_starts", False) else _i32(self.starts.tolist())
        return self.lam.kv_attend(self.q, self.pool, self.table, self.lengths, starts=st, **kw)

    def check(self, out, causal=True, mask=None, scale=None, lse=None, weights=None, times=1, rows_ok=None):
        D, q, o = self.D, _np(self.q), _np(out)
        scale = D ** -0.5 if scale is None else scale
        for b, n in enumerate(self.rows):
            at = slice(self.starts[b], self.starts[b + 1])
            for h in range(self.Hk):
                w = np.zeros(self.lens[b])
                w_tol = np.zeros(self.lens[b])
                for j in range(h * self.G, (h + 1) * self.G):
                    m = None if mask is None else mask[b][h % len(mask[b])]
                    r = kv.attend(q[at, j], self.k[b][:, h], self.v[b][:, h], scale, causal, m)
                    d = r["slack"] * (D + 8) * 2.0 ** -24 + 2.0 ** -20
                    tol = ULP[self.dt] * np.abs(r["out"]) + (2.0 ** -11 + 2 * d)[:, None] * r["mean"] + 2.0 ** -32 * r["total"]
                    err = np.abs(o[at, j] - r["out"])
                    bad = ~(err <= tol)
                    if rows_ok is not None:
                        bad &= rows_ok[at, j][:, None]
                    assert not bad.any(), (b, h, j, np.argwhere(bad)[:3], err[bad][:3], tol[bad][:3])
                    if lse is not None:
                        e = lse[at, j].cpu().numpy().astype(np.float64)
                        empty = np.isneginf(r["lse"])
                        assert np.array_equal(np.isneginf(e), empty)
                        e, de, want = e[~empty], d[~empty], r["lse"][~empty]
                        assert (np.abs(e - want) <= de + 2.0 ** -22 * np.abs(want)).all()
                    w += r["p"].sum(0)
                    w_tol += ((2 * d + 2.0 ** -21)[:, None] * r["p"]).sum(0)
                if weights is not None:
                    got = weights[b, h, : self.lens[b]].cpu().numpy().astype(np.float64)
                    assert (np.abs(got - times * w) <= times * w_tol + 2.0 ** -22 * (1 + times * w)).all(), (b, h)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D,T,Hk,G,lens", [
    (128, 64, 2, 4, [1, 31, 32, 33, 64, 65, 130, 300]),
    (64, 32, 3, 1, [1, 2, 47, 128, 129]),
    (128, 32, 1, 7, [500, 0, 3, 127]),
    (256, 64, 2, 2, [5, 70, 200]),
    (128, 256, 1, 16, [257, 700]),
    (64, 128, 2, 40, [77, 300]),
])
def test_single_tokens(lam, D, T, Hk, G, lens, dt):
    c = Case(lam, D, T, Hk, G, dt, [1] * len(lens), lens, seed=D + G)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    c.check(c.call(lse=lse), lse=lse)
    c.check(c.call(force_starts=True))
    w = torch.zeros((len(lens), Hk, max(lens)), device="cuda")
    for _ in range(2):
        out = c.call(weights=w)
    c.check(out, weights=w, times=2)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D,T,Hk,G,rows,lens", [
    (128, 64, 1, 4, [3, 3], [200, 90]),
    (128, 64, 2, 4, [70, 1, 0, 17], [70, 1, 40, 300]),
    (64, 32, 1, 1, [150, 33], [150, 290]),
    (64, 128, 2, 3, [65, 129], [300, 129]),
    (256, 32, 1, 2, [40, 90], [333, 91]),
    (128, 64, 1, 8, [130], [421]),
    (128, 128, 1, 1, [257], [600]),
])
def test_chunks(lam, D, T, Hk, G, rows, lens, causal, dt):
    c = Case(lam, D, T, Hk, G, dt, rows, lens, seed=len(rows) + D)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    w = torch.zeros((len(lens), Hk, max(lens)), device="cuda")
    out = c.call(causal=causal, lse=lse, weights=w)
    c.check(out, causal=causal, lse=lse, weights=w)
    c.check(c.call(causal=causal, max_length=max(lens)), causal=causal)


def test_more_rows_than_tokens(lam):
    """The first rows of a causal chunk that is longer than its cache see nothing."""
    for n, length in ((40, 7), (5, 0), (300, 100)):
        c = Case(lam, 64, 32, 1, 2, "bf16", [n], [length], seed=n)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        w = torch.zeros((1, 1, max(1, length)), device="cuda")
        c.check(c.call(lse=lse, weights=w), lse=lse, weights=w)


@pytest.mark.parametrize("n", [1, 2, 80])
@pytest.mark.parametrize("shared", [True, False])
def test_masks(lam, n, shared):
    lens, Hk = [40, 130, 290, 33], 2
    c = Case(lam, 64, 32, Hk, 3, "f16", [n] * 4, lens, seed=n)
    rng = np.random.default_rng(n)
    m = rng.random((4, 1 if shared else Hk, 290)) > 0.4
    m[0] = False                                   # nothing left for a sequence
    m[1, 0, :] = False                             # or a head
    m[1, 0, 129] = shared
    m[3, 0, :32] = False                           # a whole strip
    for cols in (290, 100):                        # tokens past its columns are masked
        mm = torch.from_numpy(m[:, :, :cols].copy()).cuda()
        full = m & (np.arange(290) < cols)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        w = torch.zeros((4, Hk, 290), device="cuda")
        for causal in (True, False):
            w.zero_()
            out = c.call(causal=causal, mask=mm, lse=lse, weights=w)
            c.check(out, causal=causal, mask=[full[b][:, : lens[b]] for b in range(4)], lse=lse, weights=w)
    # any byte but 0 keeps a token; strided masks
    mm = torch.from_numpy(m).cuda().to(torch.uint8) * 3
    wide = torch.zeros((4, mm.shape[1], 580), dtype=torch.uint8, device="cuda")
    wide[..., ::2] = mm
    out = c.call(mask=wide[..., ::2])
    c.check(out, mask=[m[b][:, : lens[b]] for b in range(4)])


@pytest.mark.parametrize("n", [1, 90])
def test_peaked_and_flat_scores(lam, n):
    for spread, scale in ((30.0, None), (1e-3, None), (1.0, 3.0), (1.0, -0.5), (1.0, 0.0)):
        c = Case(lam, 128, 64, 1, 4, "bf16", [n], [700], seed=int(spread), spread=spread)
        c.check(c.call(scale=scale), scale=scale)


@pytest.mark.parametrize("n", [1, 100])
def test_rising_scores(lam, n):
    """Scores that grow along the length by more than the exponent's range, strip after strip."""
    D, L = 128, 900
    c = Case(lam, D, 64, 1, 2, "bf16", [n], [L], seed=3)
    ramp = torch.linspace(-8, 8, L, device="cuda")[:, None, None].to(torch.bfloat16)
    k = ramp.expand(L, 1, D).contiguous()
    for sign in (1, -1):
        kk = (k * sign).contiguous()
        v = torch.randn((L, 1, D), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
        lam.kv_append(kk, v, c.pool, c.table, c.lengths)
        c.k, c.v = [kv.rounded(_np(kk))], [kv.rounded(_np(v))]
        c.q = torch.ones((n, 2, D), dtype=torch.bfloat16, device="cuda") * 4
        w = torch.zeros((1, 1, L), device="cuda")
        lse = torch.empty((n, 2), device="cuda")
        c.check(c.call(weights=w, lse=lse), weights=w, lse=lse)


@pytest.mark.parametrize("n", [1, 3, 70])
def test_spoiled_queries_stay_alone(lam, n):
    c = Case(lam, 128, 64, 2, 4, "f16", [n, n], [300, 50], seed=n)
    ok = np.ones(c.q.shape[:2], dtype=bool)
    for r, j, v in ((0, 1, math.nan), (n, 6, math.inf), (2 * n - 1, 3, -math.inf)):
        c.q[r, j, 17] = v
        ok[r, j] = False
    out = c.call()
    spoiled = ~ok
    spoiled[n:][: max(0, n - 50)] = False                     # rows that see no token give 0 whatever they hold
    assert torch.isnan(out[torch.from_numpy(spoiled).cuda()]).any(dim=-1).all()
    q = c.q.clone()
    c.q = torch.where(torch.isfinite(q), q, torch.zeros_like(q))   # the oracle's rows that are not compared
    c.check(out, rows_ok=ok)


def test_splits_and_lengths(lam):
    """However the length is split, and where the bound of lengths cuts it."""
    c = Case(lam, 128, 64, 1, 4, "bf16", [1, 1], [5000, 1200], seed=9)
    c.check(c.call())
    c.check(c.call(max_length=5000))
    out = c.call(causal=False, max_length=777)
    k, v, lens = c.k, c.v, c.lens
    c.k, c.v, c.lens = [x[:777] for x in k], [x[:777] for x in v], [777, 777]
    c.check(out, causal=False)
    # every sequence has its own number of parts
    c = Case(lam, 64, 32, 2, 1, "f16", [1] * 6, [3000, 1, 700, 0, 129, 2048], seed=10)
    c.check(c.call(max_length=3000))


def test_bad_pages_are_masked(lam):
    c = Case(lam, 128, 32, 2, 2, "bf16", [1, 60], [100, 100], seed=4)
    c.table[0, 1] = -1
    c.table[1, 0] = 1 << 20
    m = np.ones((2, 1, 100), dtype=bool)
    m[0, 0, 32:64] = False
    m[1, 0, :32] = False
    w = torch.zeros((2, 2, 100), device="cuda")
    lse = torch.empty(c.q.shape[:2], device="cuda")
    out = c.call(weights=w, lse=lse)
    c.check(out, mask=m, lse=lse, weights=w)


def test_query_layouts(lam):
    D, Hk, G, n = 128, 2, 4, 5
    c = Case(lam, D, 64, Hk, G, "bf16", [n], [200], seed=6)
    want = c.call()
    flat = torch.zeros(n * 16 * D + 8, dtype=torch.bfloat16, device="cuda")
    for off in (0, 1, 5):
        q = flat[off: off + n * 16 * D].view(n, 16, D)[:, 3:3 + Hk * G]
        q.copy_(c.q)
        assert torch.equal(lam.kv_attend(q, c.pool, c.table, c.lengths), want)
    q = c.q.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    assert torch.equal(lam.kv_attend(q, c.pool, c.table, c.lengths), want)
    out = torch.empty_like(want)
    assert lam.kv_attend(c.q, c.pool, c.table, c.lengths, out=out) is out and torch.equal(out, want)


def test_runs_agree_bit_for_bit(lam):
    c = Case(lam, 128, 64, 2, 4, "bf16", [33, 33], [900, 400], seed=8)
    got = []
    for _ in range(3):
        w = torch.zeros((2, 2, 900), device="cuda")
        got.append((c.call(weights=w), w))
    for o, w in got[1:]:
        assert torch.equal(o, got[0][0]) and torch.equal(w, got[0][1])


def test_another_stream_and_a_graph(lam):
    """A decode step (append, attention with weights, eviction) on a stream of its
    own, and replayed from a graph with the program's own work in between."""
    D, T, Hk, G, L, budget = 128, 64, 2, 4, 400, 256
    c = Case(lam, D, T, Hk, G, "bf16", [1], [L], seed=12)
    k, v = (torch.randn((1, Hk, D), device="cuda").to(torch.bfloat16) for _ in range(2))
    start = c.pool.clone()
    length, one = _i32([L]), _i32([L])
    w0 = torch.rand((1, Hk, L), device="cuda")
    w = w0.clone()

    def step(ctx):
        lam.kv_append(k, v, c.pool, c.table, one, weights=w, ctx=ctx)
        o = lam.kv_attend(c.q, c.pool, c.table, one, weights=w, ctx=ctx)
        return (o,) + lam.kv_evict(c.pool, c.table, length, w, budget, D, recent=8, sinks=2, ctx=ctx)

    want = [x.clone() for x in step(None)] + [c.pool.clone(), w.clone()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ctx = lam.Context(stream=s)
        c.pool.copy_(start)
        w.copy_(w0)
        got = step(ctx)
        s.synchronize()
        for a, b in zip(list(got) + [c.pool, w], want):
            assert torch.equal(a, b)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            held = step(ctx)
    for i in range(4):
        c.pool.copy_(start)
        w.copy_(w0)
        torch.cuda.synchronize()
        g.replay()
        junk = torch.rand(1 << 20, device="cuda").sum()      # the program's own work
        torch.cuda.synchronize()
        for a, b in zip(list(held) + [c.pool, w], want):
            assert torch.equal(a, b), i
    del junk
