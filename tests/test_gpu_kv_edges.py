"""The 4-bit key/value cache on the GPU at the edges of its contract: evictions that
follow each other, weights added to large ones, rows of no sequence, lengths beyond
the table, and what is refused.  Against the binary64 oracle; tolerances as in
test_gpu_kv_attend where none are given.
"""
import numpy as np
import pytest
import torch

from oracle import kv
from test_gpu_kv_attend import Case, _np
from test_gpu_kv_cache import _evict_case, _i32, _scores

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ eviction
@pytest.mark.parametrize("L,cuts", [
    (100, (64, 32)), (2100, (2080, 2070, 300)), (5000, (4990, 1000)), (30000, (20000, 19990)), (40000, (30000, 7)),
    (66000, (65990, 65800, 400)),
])
def test_evictions_without_new_tokens_keep_the_newest(lam, L, cuts):
    """After an eviction the last slot holds any token; the newest positions stay all the same."""
    D, T, heads, recent, sinks = 64, 256, 2, 5, 2
    table = torch.arange(-(-L // T), dtype=torch.int32, device="cuda").view(1, -1)
    pool = lam.kv_pages(table.shape[1], heads, D, T)
    pos = torch.arange(L, dtype=torch.int32, device="cuda").expand(1, heads, L).contiguous()
    lengths = _i32([L])
    moved = False
    for i, budget in enumerate(cuts):
        w = _scores(L + i, 1, heads, pos.shape[-1], "random")
        want = [kv.evict(w[0, h].tolist(), pos[0, h].tolist(), budget, recent, sinks) for h in range(heads)]
        kept, _, pos, lengths = lam.kv_evict(pool, table, lengths, w, budget, D, recent=recent, sinks=sinks, positions=pos)
        assert kept[0].tolist() == want
        for h in range(heads):
            assert set(pos[0, h].tolist()) >= set(range(L - recent, L)) | set(range(sinks))
        moved |= bool((pos[0, :, -1] != L - 1).any())
    assert moved


@pytest.mark.parametrize("newest", [0, 17, 1023, 1500, 2999])
def test_the_newest_position_in_any_slot(lam, newest):
    """The largest position in a slot of its own choice, negative ones (below every sink) among the others."""
    L = 3000
    pos = torch.arange(-500, L - 500, dtype=torch.int32, device="cuda").flip(0).repeat(1, 2, 1)
    pos[:, :, newest] = (1 << 31) - 1
    pos[:, 1, newest] = 2600
    _evict_case(lam, 64, 32, 2, [L], 1000, 300, 0, _scores(newest, 1, 2, L, "random"), pos, False)


# ------------------------------------------------------------------ weights
@pytest.mark.parametrize("prior", [2048.0, 1e5])
@pytest.mark.parametrize("n", [1, 4, 5])                     # scores kept, a wave a token and four; a second pass
def test_small_weights_are_added_to_large_ones_once(lam, n, prior):
    """Flat rows over many tokens, whose every p is below the rounding of the total so far:
    the call's sum is added with one rounding (2^-24 of the total), and is itself right to
    the scores' errors (test_gpu_kv_attend) and 2^-20 for its additions."""
    L, G, D = 16384, 16, 64
    c = Case(lam, D, 64, 1, G, "f16", [n], [L], seed=n, spread=1e-2)
    g = torch.Generator(device="cuda").manual_seed(n)
    before = prior * (1 + torch.rand((1, 1, L), generator=g, device="cuda"))
    w = before.clone()
    c.call(causal=False, weights=w)
    want, tol = np.zeros(L), np.zeros(L)
    for j in range(G):
        r = kv.attend(_np(c.q)[:, j], c.k[0][:, 0], c.v[0][:, 0], D ** -0.5, False)
        want += r["p"].sum(0)
        tol += ((2 * (r["slack"] * (D + 8) * 2.0 ** -24) + 2.0 ** -19)[:, None] * r["p"]).sum(0)
    total = before[0, 0].cpu().numpy().astype(np.float64) + want
    got = w[0, 0].cpu().numpy().astype(np.float64)
    assert (np.abs(got - total) <= 2.0 ** -24 * total + tol).all()


# ------------------------------------------------------------------ rows and lengths
@pytest.mark.parametrize("D,G,rows,lens,before,after", [
    (128, 4, [1, 1, 1], [300, 0, 77], 2, 3),                 # single tokens, whole and in parts
    (128, 4, [1, 1], [5000, 40], 1, 700),
    (64, 2, [60, 0, 90], [70, 5, 300], 5, 1),                # chunks
    (64, 2, [70], [2500], 0, 2),
    (256, 4, [30, 40], [90, 1500], 3, 0),
    (64, 1, [1] * 900, [9] * 900, 1, 2),                     # many sequences
    (64, 3, [0, 0], [40, 50], 4, 1),                         # no row of any sequence
])
def test_rows_of_no_sequence_get_nothing(lam, D, G, rows, lens, before, after):
    """A batch padded to more rows than its sequences have."""
    c = Case(lam, D, 32, 1, G, "bf16", rows, lens, seed=D + after)
    n = sum(rows)
    q = torch.randn((before + n + after, G, D), device="cuda").to(torch.bfloat16)
    q[before:before + n] = c.q
    q[:before] = float("nan")
    starts = _i32([before + int(x) for x in c.starts])
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
    w = torch.zeros((len(lens), 1, max(lens)), device="cuda")
    lam.kv_attend(q, c.pool, c.table, c.lengths, starts=starts, out=out, lse=lse, weights=w)
    mine = slice(before, before + n)
    c.check(out[mine], lse=lse[mine], weights=w)
    for pad in (slice(0, before), slice(before + n, None)):
        assert not out[pad].any() and torch.isneginf(lse[pad]).all()
    again = lam.kv_attend(q, c.pool, c.table, c.lengths, starts=starts)
    assert torch.equal(again, out)


@pytest.mark.parametrize("D,G,rows,lens,cols", [
    (128, 4, [3, 3], [100, 50], 2),                          # single tokens
    (128, 2, [8, 4], [5000, 300], 90),                       # in parts
    (64, 2, [70, 40], [100, 70], 2),                         # chunks
    (64, 1, [400, 80], [3500, 900], 80),
    (256, 4, [30, 40], [90, 150], 2),
])
def test_a_causal_limit_goes_by_the_length_not_the_table(lam, D, G, rows, lens, cols):
    """Tokens past the table's columns are as if masked; the rows are still the length's last."""
    c = Case(lam, D, 32, 2, G, "bf16", rows, lens, seed=D + cols)
    c.table = c.table[:, :cols].contiguous()
    there = [(np.arange(n) < 32 * cols)[None] for n in lens]
    assert not all(m.all() for m in there)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    w = torch.zeros((2, 2, max(lens)), device="cuda")
    c.check(c.call(lse=lse, weights=w), mask=there, lse=lse, weights=w)
    c.check(c.call(max_length=max(lens)), mask=there)
    assert not w[..., 32 * cols:].any()


# ------------------------------------------------------------------ refusals
def test_launches_too_large_are_refused_before_anything_is_written(lam):
    """1,024 sequences of 8 heads of 256 channels with a table of 131,072 tokens and no bound of
    lengths: 2^24 workgroups of the weights' second pass, one too many."""
    B, H, D, T = 1024, 8, 256, 1024
    pool = lam.kv_pages(1, H, D, T)
    k, v = (torch.randn((1, H, D), device="cuda").half() for _ in range(2))
    lam.kv_append(k, v, pool, _i32([[0]]), _i32([1]))
    table = torch.zeros((B, 128), dtype=torch.int32, device="cuda")
    lengths = torch.ones(B, dtype=torch.int32, device="cuda")
    q = torch.randn((B, H, D), device="cuda").half()
    out, w = torch.full_like(q, 7.0), torch.full((B, H, 1), 3.0, device="cuda")
    lse = torch.full((B, H), 5.0, device="cuda")
    with pytest.raises(lam.LamError) as e:
        lam.kv_attend(q, pool, table, lengths, weights=w, out=out, lse=lse)
    assert e.value.name == "LAM_EINVAL" and "max_length" in str(e.value)
    assert (out == 7).all() and (w == 3).all() and (lse == 5).all()
    # one sequence less, or the bound given, and it runs: each token is all that its row sees
    lam.kv_attend(q[1:], pool, table[1:], lengths[1:], weights=w[1:], out=out[1:])
    lam.kv_attend(q, pool, table, lengths, weights=w, out=out, lse=lse, max_length=1)
    a, b = lam.kv_read(pool, _i32([[0]]), _i32([1]), 1, D, dtype=torch.float16)
    assert torch.equal(out, b.expand_as(out))
    assert torch.allclose(w[1:], torch.full_like(w[1:], 5.0)) and torch.allclose(w[0], torch.full_like(w[0], 4.0))
    # one row in a batch of 2^20 sequences of 512 heads
    n = 1 << 20
    empty, lengths = torch.empty((n, 0), dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    starts = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    none, k = lam.kv_pages(0, 512, D, 32), torch.zeros((1, 512, D), dtype=torch.float16, device="cuda")
    for call in (lambda: lam.kv_append(k, k, none, empty, lengths, starts=starts),
                 lambda: lam.kv_read(none, empty, lengths, 1, D, starts=starts)):
        with pytest.raises(lam.LamError) as e:
            call()
        assert e.value.name == "LAM_EINVAL"


def test_slots_that_overlap_are_refused(lam):
    """Two slots of one element would be written by two workgroups; any layout without is taken."""
    B, Hk, L = 3, 2, 40
    c = Case(lam, 64, 32, Hk, 2, "f16", [1] * B, [40, 25, 33], seed=1)
    k = torch.zeros((B, Hk, 64), dtype=torch.float16, device="cuda")

    def strided(seq, head, dtype=torch.float32):
        flat = torch.zeros(1 + (B - 1) * seq + (Hk - 1) * head + L, dtype=dtype, device="cuda")
        return flat[1:].as_strided((B, Hk, L), (seq, head, 1))

    pool = c.pool.clone()
    for seq, head in ((40, 40), (40, 60), (60, 90), (40, 80), (41, 82), (79, 40), (100, 139), (80, 199)):
        for call in (lambda: lam.kv_append(k, k, c.pool, c.table, c.lengths, weights=strided(seq, head)),
                     lambda: lam.kv_append(k, k, c.pool, c.table, c.lengths, first=c.lengths,
                                           positions=strided(seq, head, torch.int32)),
                     lambda: c.call(weights=strided(seq, head)),
                     lambda: lam.kv_evict(c.pool, c.table, c.lengths, torch.zeros((B, Hk, L), device="cuda"), 20, 64,
                                          out=(strided(seq, head), None, c.lengths))):
            with pytest.raises(lam.LamError) as e:
                call()
            assert e.value.name == "LAM_EINVAL"
    assert torch.equal(pool, c.pool) and c.lengths.tolist() == c.lens
    want = torch.zeros((B, Hk, L), device="cuda")
    c.call(weights=want)
    for seq, head in ((80, 40), (40, 120), (83, 41), (100, 50), (50, 200), (40, 1000), (100, 140), (80, 200)):
        w = strided(seq, head)
        c.call(weights=w)
        assert torch.equal(w, want)


def test_gradients_are_not_dropped_unseen(lam):
    """The operators have no gradient: tensors that require one are refused, but under no_grad."""
    c = Case(lam, 64, 32, 1, 2, "f16", [1], [40], seed=2)
    k, w = torch.zeros((1, 1, 64), dtype=torch.float16, device="cuda"), torch.zeros((1, 1, 40), device="cuda")
    out, lse = torch.zeros_like(c.q), torch.zeros((1, 2), device="cuda")
    want = c.call()

    def grad(t):
        return t.clone().requires_grad_()

    pool = c.pool.clone()
    for call in (lambda: lam.kv_attend(grad(c.q), c.pool, c.table, c.lengths),
                 lambda: lam.kv_attend(grad(c.q) * 2, c.pool, c.table, c.lengths),
                 lambda: c.call(weights=grad(w)), lambda: c.call(out=grad(out)), lambda: c.call(lse=grad(lse)),
                 lambda: lam.kv_append(grad(k), k, c.pool, c.table, c.lengths),
                 lambda: lam.kv_append(k, grad(k), c.pool, c.table, c.lengths),
                 lambda: lam.kv_evict(c.pool, c.table, c.lengths, grad(w), 20, 64)):
        with pytest.raises(ValueError, match="gradient"):
            call()
    assert torch.equal(pool, c.pool)
    with torch.no_grad():
        assert torch.equal(lam.kv_attend(grad(c.q), c.pool, c.table, c.lengths), want)
    with torch.inference_mode():
        assert torch.equal(lam.kv_attend(c.q, c.pool, c.table, c.lengths), want)


@pytest.mark.parametrize("n", [1, 90])
def test_results_in_place_of_the_queries(lam, n):
    """out may be q, but where a second pass takes the weights from the queries."""
    for lens in ([200], [3000]):
        c = Case(lam, 64, 32, 2, 4, "bf16", [n], lens, seed=n)
        w = torch.zeros((1, 2, lens[0]), device="cuda")
        want, q = c.call(weights=w), c.q.clone()
        again = torch.zeros_like(w)
        if n > 1:
            with pytest.raises(lam.LamError) as e:
                c.call(out=c.q, weights=again)
            assert e.value.name == "LAM_EINVAL" and torch.equal(c.q, q) and not again.any()
        else:
            assert torch.equal(c.call(out=c.q, weights=again), want) and torch.equal(again, w)
            c.q.copy_(q)
        assert torch.equal(c.call(out=c.q), want) and torch.equal(c.q, want)
        flat = torch.zeros((n + 1) * 512, dtype=torch.bfloat16, device="cuda")
        for at in (8, 256, 504):                             # parts of one buffer
            a, b = flat[at:at + n * 512].view(n, 8, 64), flat[:n * 512].view(n, 8, 64)
            for x, y in ((a, b), (b, a)):
                with pytest.raises(lam.LamError):
                    lam.kv_attend(x, c.pool, c.table, c.lengths, out=y)
        assert not flat.any()
        both = torch.cat([q, q])                             # next to each other
        lam.kv_attend(both[:n], c.pool, c.table, c.lengths, out=both[n:], weights=torch.zeros_like(w))
        assert torch.equal(both[n:], want) and torch.equal(both[:n], q)


def test_numbers_beyond_32_bits_are_refused(lam):
    """Not taken for their low 32 bits."""
    pool, table, lengths = lam.kv_pages(2, 1, 64, 32), _i32([[0, 1]]), _i32([40])
    w = torch.zeros((1, 1, 40), device="cuda")
    for bad in (dict(recent=(1 << 32) + 3), dict(sinks=1 << 32), dict(recent=-(1 << 32)), dict(recent=1 << 31)):
        with pytest.raises(ValueError):
            lam.kv_evict(pool, table, lengths, w, 20, 64, **bad)
    with pytest.raises(ValueError):
        lam.kv_evict(pool, table, lengths, w, (1 << 32) + 20, 64)
    with pytest.raises(lam.LamError):
        lam.kv_evict(pool, table, lengths, w, -5, 64)
    for bad in (dict(head_dim=(1 << 32) + 64), dict(head_dim=64, page_size=(1 << 32) + 32)):
        with pytest.raises(ValueError):
            lam.kv_pages(1, 1, **bad)
    assert lengths.tolist() == [40]


# ------------------------------------------------------------------ paths with no other test
@pytest.mark.parametrize("D", [64, 128, 256])
def test_read_gives_zeros_for_rows_of_no_sequence(lam, D):
    k, v = (torch.randn((5, 2, D), device="cuda").half() for _ in range(2))
    pool, table, lens = lam.kv_pages(2, 2, D, 32), _i32([[0], [1]]), _i32([3, 4])
    lam.kv_append(k, v, pool, table, lens, starts=_i32([0, 3, 5]))
    for fill in range(2):                                    # memory that another call has just filled
        full = lam.kv_read(pool, table, lens, 9, D, dtype=torch.float16, starts=_i32([2, 5, 7]))
        for x, y in zip(full, (k, v)):
            assert np.array_equal(_np(x[2:7]), kv.rounded(_np(y)))
            assert not x[:2].any() and not x[7:].any()
            x.fill_(float("nan"))
        del full, x
    a, b = lam.kv_read(pool, table, lens, 700, D, dtype=torch.float16, starts=_i32([700, 700, 700]))
    assert not a.any() and not b.any()


@pytest.mark.parametrize("n", [1, 90])                       # scores kept, a second pass
@pytest.mark.parametrize("length", [700, 3000])              # whole, in parts
def test_weights_and_log_sums_of_any_scale(lam, n, length):
    for spread, scale in ((30.0, None), (1e-3, None), (1.0, 3.0), (1.0, -0.5), (20.0, -0.1), (1.0, 0.0)):
        c = Case(lam, 128, 64, 1, 4, "bf16", [n], [length], seed=int(spread), spread=spread)
        lse = torch.empty(c.q.shape[:2], device="cuda")
        w = torch.zeros((1, 1, length), device="cuda")
        c.check(c.call(scale=scale, lse=lse, weights=w), scale=scale, lse=lse, weights=w)


@pytest.mark.parametrize("G,n", [(4, 1), (16, 4), (4, 40)])  # a wave a token, four, a second pass
@pytest.mark.parametrize("cols", [0, 1, 33, 130, 255, 1030])
def test_weights_of_fewer_columns_than_tokens(lam, G, n, cols):
    lens, Hk = [1200, 90], 2
    c = Case(lam, 64, 32, Hk, G, "f16", [n] * 2, lens, seed=n)
    full = torch.zeros((2, Hk, 1200), device="cuda")
    c.check(c.call(weights=full), weights=full)
    wide = torch.full((2, Hk, 1200), 9.0, device="cuda")
    wide[..., :cols] = 0
    c.call(weights=wide[..., :cols])
    assert torch.equal(wide[..., :cols], full[..., :cols]) and (wide[..., cols:] == 9).all()


@pytest.mark.parametrize("n", [2, 70])
@pytest.mark.parametrize("cap", [128, 2560])
def test_lengths_that_cannot_be(lam, n, cap):
    """A negative length is 0; the rows of one near 2^31 see every token that the table has."""
    c = Case(lam, 64, 32, 2, 2, "f16", [n] * 3, [cap, cap, cap], seed=n)
    c.lengths = _i32([-3, (1 << 31) - 1, -(1 << 31)])
    lse, w = torch.empty(c.q.shape[:2], device="cuda"), torch.zeros((3, 2, cap), device="cuda")
    out = c.call(lse=lse, weights=w)
    for s in (0, 2):
        rows = slice(s * n, s * n + n)
        assert not out[rows].any() and torch.isneginf(lse[rows]).all() and not w[s].any()
    want, want_w = torch.empty_like(out), torch.zeros_like(w)
    c.lengths = _i32([cap, cap, cap])
    c.call(causal=False, out=want, weights=want_w)
    assert torch.allclose(out[n:2 * n].float(), want[n:2 * n].float(), rtol=2.0 ** -9, atol=2.0 ** -11)
    assert torch.allclose(w[1], want_w[1], rtol=2.0 ** -18, atol=0)
    # nothing of the rows has a place, and nothing is written
    pool, k = c.pool.clone(), torch.randn((3 * n, 2, 64), device="cuda").half()
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    bad = _i32([-3, (1 << 31) - 1, -(1 << 31)])
    lam.kv_append(k, k, c.pool, c.table, bad, status=status)
    assert status.tolist() == [0, 0, 3 * n * 2] and torch.equal(c.pool, pool)
    assert not lam.kv_read(c.pool, c.table, bad, 3 * n, 64, dtype=torch.float16)[0].any()
    scores = torch.rand((3, 2, cap), device="cuda")
    kept, _, _, lo = lam.kv_evict(c.pool, c.table, bad, scores, 100, 64)
    assert lo.tolist() == [0, 100, 0] and (kept[0] == -1).all() and (kept[2] == -1).all()
    for h in range(2):
        assert kept[1, h].tolist() == kv.evict(scores[1, h].tolist(), list(range(cap)), 100, 0, 0)
