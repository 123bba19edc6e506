"""Attention with a sliding window and first tokens that stay visible, over the 4-bit cache
on the GPU, against the binary64 oracle.  Tolerances as in test_gpu_kv_attend."""
import numpy as np
import pytest
import torch

from oracle import kv
from test_gpu_kv_attend import Case, _i32

pytestmark = pytest.mark.gpu


def _seen(c, window, sinks, mask=None):
    """Of each sequence, [n, length] for the oracle."""
    out = []
    for b, (n, length) in enumerate(zip(c.rows, c.lens)):
        m = kv.in_window(n, length, window, sinks)
        out.append([m] if mask is None else [m & x[None, :length] for x in mask[b]])
    return out


def _poison(c, window, sinks, causal):
    """Tokens that no row sees: bytes of 0xFF, and pages of such tokens alone taken away."""
    D, T, run = c.D, c.T, c.D // 32
    cut = T * D // 2
    table = c.table.cpu().numpy()
    for b, (n, length) in enumerate(zip(c.rows, c.lens)):
        seen = kv.in_window(n, length, window, sinks)
        if causal:
            seen &= np.arange(length)[None, :] <= length - n + np.arange(n)[:, None]
        gone = ~seen.any(axis=0) if n else np.ones(length, dtype=bool)
        for col in range(table.shape[1]):
            page = table[b, col]
            at = np.arange(col * T, (col + 1) * T)
            mine = at[at < length]
            if len(mine) == 0 or gone[mine].all():
                c.pool[int(page)] = 255
                table[b, col] = (-1, 1 << 30, -(1 << 31))[col % 3]
                continue
            for t in mine[gone[mine]] % T:
                t, j = int(t), np.arange(D // 2)
                where = np.concatenate([t * (D // 2) + j, cut + ((t // 4 * 16 + j // run) * 4 + t % 4) * run + j % run,
                                        2 * cut + t * run + np.arange(run),
                                        2 * cut + T * run + (t // 4 * run + np.arange(run)) * 4 + t % 4])
                c.pool[int(page)][:, torch.from_numpy(where).cuda()] = 255
    c.table = _i32(table.tolist())


def _run(c, window, sinks, causal=True, mask=None, weights=True, **kw):
    lse = torch.full(c.q.shape[:2], float("nan"), device="cuda")
    w = torch.zeros((len(c.lens), c.Hk, max(max(c.lens), 1)), device="cuda") if weights else None
    out = c.call(causal=causal, lse=lse, weights=w, window=window, sinks=sinks, mask=mask, **kw)
    m = None
    if mask is not None:
        m = [[x.cpu().numpy() for x in mask[b]] for b in range(len(c.lens))]
    c.check(out, causal=causal, mask=_seen(c, window, sinks, m), lse=lse, weights=w)
    return out


WINDOWS = [(1, 0), (1, 1), (31, 0), (32, 33), (33, 4), (100, 32), (64, 200), (1000, 3), (1 << 40, 0)]


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("D,T,Hk,G,dt,lens", [
    (128, 64, 2, 4, "bf16", [1, 31, 32, 33, 64, 65, 130, 300]),
    (64, 32, 3, 1, "f16", [1, 2, 47, 128, 129]),
    (128, 32, 1, 7, "f16", [500, 0, 3, 127]),
    (256, 64, 2, 2, "bf16", [5, 70, 200]),
    (64, 128, 2, 40, "bf16", [77, 300]),
])
def test_single_tokens(lam, D, T, Hk, G, dt, lens, window, sinks):
    c = Case(lam, D, T, Hk, G, dt, [1] * len(lens), lens, seed=D + G)
    _poison(c, window, sinks, True)
    a = _run(c, window, sinks)
    b = _run(c, window, sinks, weights=False, force_starts=True)
    assert torch.equal(a, b)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window,sinks", [(1, 0), (17, 3), (32, 32), (70, 65), (129, 0), (5000, 1)])
@pytest.mark.parametrize("D,T,Hk,G,dt,rows,lens", [
    (128, 64, 1, 4, "bf16", [3, 3], [200, 90]),              # few rows: scores kept
    (128, 64, 2, 4, "f16", [70, 1, 0, 17], [70, 1, 40, 300]),
    (64, 32, 1, 1, "bf16", [150, 33], [150, 290]),
    (64, 128, 2, 3, "f16", [65, 129], [300, 129]),
    (256, 32, 1, 2, "bf16", [40, 90], [333, 91]),
    (128, 64, 1, 8, "bf16", [130], [421]),
    (128, 128, 1, 1, "f16", [257], [600]),
    (64, 64, 8, 1, "f16", [100, 60], [600, 200]),            # heads by XCD
])
def test_chunks(lam, D, T, Hk, G, dt, rows, lens, window, sinks, causal):
    c = Case(lam, D, T, Hk, G, dt, rows, lens, seed=len(rows) + D)
    _poison(c, window, sinks, causal)
    _run(c, window, sinks, causal)
    _run(c, window, sinks, causal, weights=False, max_length=max(lens))


@pytest.mark.parametrize("D,T,Hk,G,dt,rows,lens,window,sinks", [
    (128, 64, 1, 4, "bf16", [1, 1], [9000, 5000], 4000, 4),          # single tokens, the window split
    (128, 64, 2, 4, "bf16", [1, 1, 1], [9000, 100, 5000], 2500, 40),
    (128, 64, 1, 4, "bf16", [1], [9000], 100, 2500),                 # the sinks split
    (64, 256, 1, 1, "f16", [4, 4], [20000, 20000], 8192, 1),
    (256, 64, 1, 2, "f16", [3, 1], [6000, 3000], 2100, 0),
    (128, 64, 1, 2, "bf16", [300, 50], [3000, 5000], 1500, 10),      # chunks, split
    (64, 64, 1, 1, "f16", [129], [6000], 4000, 64),
    (256, 64, 1, 4, "bf16", [60, 90], [4000, 3100], 2000, 7),
    (128, 64, 1, 1, "bf16", [1500], [4000], 300, 4),                 # not split: the window is short
])
@pytest.mark.parametrize("masked", [False, True])
def test_long_lengths(lam, D, T, Hk, G, dt, rows, lens, window, sinks, masked):
    c = Case(lam, D, T, Hk, G, dt, rows, lens, seed=window)
    _poison(c, window, sinks, True)
    mask = None
    if masked:
        g = torch.Generator(device="cuda").manual_seed(window)
        mask = (torch.rand((len(lens), 1, -(-max(lens) // 16)), generator=g, device="cuda") > 0.3).repeat_interleave(16, -1)
        mask[:, :, 512:1024] = False
    _run(c, window, sinks, mask=mask)
    _run(c, window, sinks, mask=mask, weights=False)


@pytest.mark.parametrize("D,B,Hk,n,window", [
    (64, 1, 8, 410, 100), (64, 8, 8, 410, 100), (64, 25, 8, 410, 100), (64, 50, 8, 410, 100),   # by 1 and 8, 2 and 8, 2 and 4, 4 and 4
    (128, 1, 8, 410, 100), (128, 6, 8, 410, 100), (128, 8, 8, 410, 100), (128, 25, 8, 410, 100),  # 1 and 8, 2 and 8, 4 and 8, 4 and 4
    (64, 8, 8, 70, 200), (128, 8, 8, 70, 200), (256, 2, 2, 410, 100),                           # 2 and 4
])
def test_weights_by_every_tile(lam, D, B, Hk, n, window):
    """Strips and waves of the weights' second pass, which go by how many workgroups have work."""
    c = Case(lam, D, 64, Hk, 1, "bf16", [n] * B, [420 - b % 5 for b in range(B)], seed=B)
    _poison(c, window, 5, True)
    _run(c, window, 5)


def test_many_sequences(lam):
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 400, 130)]
    c = Case(lam, 64, 32, 2, 2, "bf16", [1 if x else 0 for x in lens], lens, seed=1)
    _poison(c, 50, 5, True)
    _run(c, 50, 5)


@pytest.mark.parametrize("n,length", [(40, 7), (5, 0), (300, 100), (70, 69)])
@pytest.mark.parametrize("causal", [True, False])
def test_more_rows_than_tokens(lam, n, length, causal):
    c = Case(lam, 64, 32, 1, 2, "bf16", [n], [length], seed=n)
    for window, sinks in ((3, 2), (20, 0)):
        _run(c, window, sinks, causal)


def test_a_mask_that_leaves_nothing_of_a_window(lam):
    c = Case(lam, 128, 64, 2, 4, "f16", [2, 2], [500, 130], seed=8)
    mask = torch.ones((2, 2, 500), dtype=torch.bool, device="cuda")
    mask[0, 0, 300:] = False                                 # the window of one head
    mask[1, :, 2:] = False                                   # all but two of the first tokens
    _run(c, 100, 0, mask=mask)
    _run(c, 100, 3, mask=mask)
    mask[0, 0, :3] = False
    _run(c, 100, 3, mask=mask)


@pytest.mark.parametrize("D,G,rows,lens,before,after", [
    (128, 4, [1, 1, 1], [300, 0, 77], 2, 3),
    (128, 4, [1, 1], [5000, 40], 1, 700),
    (64, 2, [60, 0, 90], [70, 5, 300], 5, 1),
    (256, 4, [30, 40], [90, 1500], 3, 0),
])
def test_rows_of_no_sequence_get_nothing(lam, D, G, rows, lens, before, after):
    c = Case(lam, D, 32, 1, G, "bf16", rows, lens, seed=D + after)
    n = sum(rows)
    q = torch.randn((before + n + after, G, D), device="cuda").to(torch.bfloat16)
    q[before:before + n] = c.q
    q[:before] = float("nan")
    starts = _i32([before + int(x) for x in c.starts])
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    w = torch.zeros((len(lens), 1, max(lens)), device="cuda")
    lam.kv_attend(q, c.pool, c.table, c.lengths, starts=starts, out=out, lse=lse, weights=w, window=50, sinks=3)
    mine = slice(before, before + n)
    c.check(out[mine], mask=_seen(c, 50, 3), lse=lse[mine], weights=w)
    for pad in (slice(0, before), slice(before + n, None)):
        assert not out[pad].any() and torch.isneginf(lse[pad]).all()


@pytest.mark.parametrize("D,G,rows,lens,cols", [
    (128, 4, [3, 3], [100, 50], 2), (128, 2, [8, 4], [5000, 300], 90), (64, 2, [70, 40], [100, 70], 2),
])
def test_a_window_goes_by_the_length_not_the_table(lam, D, G, rows, lens, cols):
    """Tokens past the table's columns, or the caller's bound, are as if masked; the windows of the last rows
    may lie there whole."""
    for window, sinks in ((30, 5), (60, 0), (5000, 1)):
        c = Case(lam, D, 32, 2, G, "bf16", rows, lens, seed=D + cols)
        cut = [[(np.arange(n) < 32 * cols)] for n in lens]
        lse = torch.empty(c.q.shape[:2], device="cuda")
        w = torch.zeros((2, 2, max(lens)), device="cuda")
        whole = c.table
        out = c.call(lse=lse, max_length=32 * cols, window=window, sinks=sinks)
        c.check(out, mask=_seen(c, window, sinks, cut), lse=lse)
        c.table = whole[:, :cols].contiguous()
        out = c.call(lse=lse, weights=w, window=window, sinks=sinks)
        c.check(out, mask=_seen(c, window, sinks, cut), lse=lse, weights=w)


@pytest.mark.parametrize("n,G", [(1, 4), (3, 2), (90, 2)])    # single tokens; scores kept; chunks
@pytest.mark.parametrize("length", [(1 << 31) - 1, (1 << 31) - 4097, 1 << 30, 5000])
def test_windows_far_past_the_table(lam, n, G, length):
    """Lengths that count tokens without a place, to the largest an int32 holds: of 200 tokens with one,
    rows at the length's end see the first alone, or nothing."""
    c = Case(lam, 64, 32, 2, G, "bf16", [n] * 2, [200, 200], seed=n)
    c.lengths = _i32([length, 200])
    for window, sinks in ((64, 3), (100, 0), (3000, 40)):
        seen = [[kv.in_window(n, 200, 1 << 40, 0) & (np.arange(200) < sinks)[None]], [kv.in_window(n, 200, window, sinks)]]
        for causal in (True, False):
            lse = torch.full(c.q.shape[:2], float("nan"), device="cuda")
            w = torch.zeros((2, 2, 200), device="cuda")
            out = c.call(causal=causal, lse=lse, weights=w, window=window, sinks=sinks)
            for b in range(2):
                one = Case.__new__(Case)
                one.D, one.Hk, one.G, one.dt, one.rows, one.lens = c.D, c.Hk, c.G, c.dt, [n], [200]
                at = slice(b * n, b * n + n)
                one.q, one.starts, one.k, one.v = c.q[at], [0, n], c.k[b:b + 1], c.v[b:b + 1]
                one.check(out[at], causal=causal and b == 1, mask=[seen[b]], lse=lse[at], weights=w[b:b + 1])


def test_a_window_of_everything_is_none(lam):
    for rows, lens in (([1, 1], [4000, 77]), ([200, 3], [1500, 90]), ([4, 4], [300, 300])):
        c = Case(lam, 128, 64, 2, 4, "bf16", rows, lens, seed=5)
        want = c.call()
        for window in (max(lens), 1 << 31, (1 << 63) - 1):
            assert torch.equal(c.call(window=window), want)
            assert torch.equal(c.call(window=window, sinks=1 << 40), want)
        w, w2 = (torch.zeros((len(lens), 2, max(lens)), device="cuda") for _ in range(2))
        c.call(weights=w), c.call(weights=w2, window=max(lens))
        # sums of a token's p over the rows and heads of a group, in another order
        assert ((w - w2).abs() <= max(rows) * c.G * 2.0 ** -24 * w).all()


def test_weights_outside_the_window_stay(lam):
    for n in (2, 200):                                       # scores kept, and a second pass
        c = Case(lam, 64, 32, 2, 2, "f16", [n], [3000], seed=n)
        w = torch.rand((1, 2, 3000), device="cuda")
        before = w.clone()
        c.call(weights=w, window=100, sinks=4)
        assert torch.equal(w[..., 4:3000 - n - 99], before[..., 4:3000 - n - 99])
        assert (w[..., :4] > before[..., :4]).all() and (w[..., -99:] != before[..., -99:]).any()


@pytest.mark.parametrize("n", [2, 90])                             # scores kept, and a second pass
def test_weights_and_masks_of_fewer_columns_than_tokens(lam, n):
    c = Case(lam, 64, 32, 2, 2, "f16", [n], [700], seed=n)
    whole = torch.zeros((1, 2, 700), device="cuda")
    c.call(weights=whole, window=300, sinks=40)
    for cols in (0, 20, 500, 650):
        w = torch.full((1, 2, cols + 3), 7.0, device="cuda")
        c.call(weights=w[..., :cols], window=300, sinks=40)
        assert torch.equal(w[..., :cols] - 7 + 7, whole[..., :cols] + 7) and (w[..., cols:] == 7).all()
    mask = torch.ones((1, 1, 650), dtype=torch.bool, device="cuda")
    seen = [m & (np.arange(700) < 650)[None] for m in _seen(c, 300, 40)[0]]
    c.check(c.call(mask=mask, window=300, sinks=40), mask=[seen])


def test_a_graph_whose_lengths_grow(lam):
    c = Case(lam, 128, 64, 2, 4, "bf16", [1, 1], [5000, 300], seed=2)
    full = c.lengths.clone()
    s = torch.cuda.Stream()
    ctx = lam.Context(stream=s)
    w = torch.zeros((2, 2, 5000), device="cuda")
    c.call(weights=w, window=2500, sinks=4, max_length=5000, ctx=ctx)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = c.call(weights=w, window=2500, sinks=4, max_length=5000, ctx=ctx)
    for cut in (0, 250, 2600, 1, 299):
        c.lengths.copy_((full - cut).clamp(min=1))
        w.zero_()
        g.replay()
        torch.cuda.synchronize()
        w2 = torch.zeros_like(w)
        want = c.call(weights=w2, window=2500, sinks=4, max_length=5000)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(w, w2)


def test_refusals(lam):
    c = Case(lam, 64, 32, 1, 2, "bf16", [1], [50])
    for bad in (dict(window=0), dict(window=-1), dict(window=1 << 63), dict(sinks=1), dict(window=5, sinks=-1),
                dict(window=5, sinks=1 << 63)):
        with pytest.raises(ValueError):
            c.call(**bad)


def test_bounds_beyond_64_bits(lam):
    """A bound of lengths is refused rather than cut to its low bits, which would leave tokens out."""
    c = Case(lam, 64, 32, 1, 2, "bf16", [1], [50])
    want = c.call()
    for bound in ((1 << 63) - 1, 1 << 40, 50):
        assert torch.equal(c.call(max_length=bound), want)
        assert torch.equal(c.call(max_length=bound, window=1 << 40), want)
    for bound in (1 << 63, (1 << 64) + 5, -(1 << 63) - 1):
        for window in (None, 20):
            with pytest.raises(ValueError):
                c.call(max_length=bound, window=window)


def test_streaming(lam):
    """Tokens normed, turned and appended, attended to in a window, and the pages behind it
    taken away: the steps of a stream of any length in a fixed number of pages."""
    D, T, Hq, Hk, window, sinks, steps = 128, 32, 8, 2, 70, 4, (5, 60, 1, 1, 40, 1, 90, 1, 1, 1)
    per = sinks // T + 1 + (window + 90) // T + 2
    pool = lam.kv_pages(per, Hk, D, T)
    table = torch.full((1, 16), -1, dtype=torch.int32, device="cuda")
    free, length = list(range(per)), 0
    f, _ = lam.rotary_frequencies(64)
    gq, gk = (torch.rand(D, device="cuda") + 0.5 for _ in range(2))
    ks, vs = [], []
    g = torch.Generator(device="cuda").manual_seed(1)
    for n in steps:
        for col in range(length // T, -(-(length + n) // T)):
            if table[0, col] < 0:
                table[0, col] = free.pop()
        q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hk, Hk))
        length += n
        lengths = _i32([length])
        status = _i32([0, 0, 0])
        q = lam.kv_rotate_append(q, k, v, pool, table, lengths, f, q_norm=gq, k_norm=gk, status=status)
        out = lam.kv_attend(q, pool, table, lengths, window=window, sinks=sinks)
        assert not status.any()
        pos = list(range(length - n, length))
        exact, _ = kv.rotate(k.double().cpu().numpy(), pos, f.cpu().numpy(), gain=gk.double().cpu().numpy())
        ks.append(kv.rounded(exact)), vs.append(kv.rounded(v.double().cpu().numpy()))
        c = Case.__new__(Case)
        c.D, c.Hk, c.G, c.dt, c.rows, c.lens = D, Hk, Hq // Hk, "bf16", [n], [length]
        c.q, c.starts, c.k, c.v = q, [0, n], [np.concatenate(ks)], [np.concatenate(vs)]
        c.check(out, mask=_seen(c, window, sinks))
        for col in range(-(-sinks // T), max(0, length - window + 1) // T):      # behind every window to come
            if table[0, col] >= 0:
                free.append(int(table[0, col]))
                pool[free[-1]] = 255
                table[0, col] = -1
    assert length == sum(steps) and length > per * T - 90
