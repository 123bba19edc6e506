"""Attention over the 4-bit cache where lengths are cut into parts, where a call has
more sequences than a wave has lanes, and where the weights come by either way; eviction
at the sizes where its kernels change.  Tolerances as in test_gpu_kv_attend.
"""
import numpy as np
import pytest
import torch

from oracle import kv
from test_gpu_kv_attend import Case, _i32
from test_gpu_kv_cache import _evict_case, _scores

pytestmark = pytest.mark.gpu


def _all(c, causal=True, mask=None, **kw):
    """Outputs, log sums and weights of one call, and the output without them."""
    B, cols = len(c.lens), max(1, max(c.lens))
    lse = torch.empty(c.q.shape[:2], device="cuda")
    w = torch.zeros((B, c.Hk, cols), device="cuda")
    m = None if mask is None else torch.from_numpy(mask).cuda()
    cut = None if mask is None else [mask[b][:, : c.lens[b]] for b in range(B)]
    c.check(c.call(causal=causal, mask=m, lse=lse, weights=w, **kw), causal=causal, mask=cut, lse=lse, weights=w)
    c.check(c.call(causal=causal, mask=m, **kw), causal=causal, mask=cut)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D,T,Hk,G,rows,lens", [
    (128, 64, 2, 4, [1], [5000]),                            # few tiles, many parts
    (128, 32, 1, 1, [1], [13000]),
    (64, 32, 1, 16, [1, 1, 1], [9000, 2049, 0]),
    (128, 64, 1, 4, [4, 4, 4], [2100, 70, 6000]),
    (256, 64, 1, 2, [1, 3, 2], [4097, 3, 2600]),
    (64, 1024, 2, 3, [11, 0, 2], [3001, 500, 2500]),         # three tiles of a sequence
    (128, 64, 1, 8, [8], [3333]),                            # 64 pairs
])
def test_parts_of_single_tokens(lam, D, T, Hk, G, rows, lens, dt):
    c = Case(lam, D, T, Hk, G, dt, rows, lens, seed=sum(lens))
    _all(c)
    _all(c, causal=False)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D,T,Hk,G,rows,lens", [
    (128, 64, 1, 4, [20], [3000]),
    (64, 128, 2, 2, [90, 0, 70], [2600, 900, 1500]),
    (256, 32, 1, 8, [9, 30], [2000, 1100]),
    (64, 64, 1, 1, [65, 65], [1025, 2303]),
])
def test_parts_of_chunks(lam, D, T, Hk, G, rows, lens, dt):
    c = Case(lam, D, T, Hk, G, dt, rows, lens, seed=sum(lens))
    _all(c)
    _all(c, causal=False)


@pytest.mark.parametrize("n,G", [(1, 4), (6, 8), (40, 2)])
def test_parts_and_masks(lam, n, G):
    lens = [2900, 64, 4100]
    c = Case(lam, 64, 32, 1, G, "f16", [n] * 3, lens, seed=n)
    m = np.random.default_rng(n).random((3, 1, max(lens))) > 0.3
    m[0, 0, 640:1900] = False                                # parts of which nothing is left
    m[1] = False
    _all(c, mask=m)


@pytest.mark.parametrize("D,n,G", [(64, 1, 4), (128, 3, 8), (128, 40, 2), (256, 30, 4)])
def test_masks_of_whole_strips(lam, D, n, G):
    """Strips that a mask leaves whole or takes out, beside some that it cuts."""
    lens = [700, 333, 2500]
    c = Case(lam, D, 64, 2, G, "f16", [n] * 3, lens, seed=n)
    m = (np.random.default_rng(n).random((3, 2, 40)) > 0.4).repeat(64, axis=2)[..., : max(lens)]
    m[:, :, 300:310] ^= True
    m[1, 1] = True
    m[2, 0, 1024:] = False
    _all(c, mask=m)
    _all(c, causal=False, mask=m)
    c.table[0, 2] = -1                                       # and a page that is not there
    m[0, :, 128:192] = True
    left = m.copy()
    left[0, :, 128:192] = False
    c.check(c.call(mask=torch.from_numpy(m).cuda()), mask=[left[b][:, : lens[b]] for b in range(3)])


@pytest.mark.parametrize("longest", [60, 2700])
@pytest.mark.parametrize("B,rows", [
    (64, lambda s: 1), (65, lambda s: 1), (200, lambda s: 1),
    (64, lambda s: s % 3), (129, lambda s: (s * 7) % 4),
    (70, lambda s: 60 if s in (3, 66) else s % 2),
    (66, lambda s: 40),                                      # chunks
    (130, lambda s: 50 + s % 30),
])
def test_many_sequences(lam, B, rows, longest):
    rng = np.random.default_rng(B)
    n = [rows(s) for s in range(B)]
    lens = [max(n[s], int(x)) for s, x in enumerate(rng.integers(0, 50, B))]
    lens[B // 2] = lens[-1] = longest
    n = [min(a, b) for a, b in zip(n, lens)] if len(set(n)) > 1 else n
    c = Case(lam, 64, 32, 1, 2, "bf16", n, lens, seed=B)
    _all(c)


@pytest.mark.parametrize("longest", [70, 1500])
@pytest.mark.parametrize("B", [100, 60])                     # 256 channels: tiles of 48 rows, of 32
def test_chunks_of_wide_heads(lam, B, longest):
    lens = [25 + s % 40 for s in range(B)]
    lens[7] = lens[-1] = longest
    c = Case(lam, 256, 32, 1, 4, "f16", [24] * B, lens, seed=B)
    _all(c)
    if longest == 70:
        _all(Case(lam, 256, 32, 1, 4, "bf16", [24 + s % 2 for s in range(B)], lens, seed=B))


def test_wide_heads_over_two_rounds(lam):
    """A few more tiles of 256 channels than run at once: lengths are split all the same."""
    rng = np.random.default_rng(3)
    lens = [int(x) for x in rng.integers(0, 60, 300)]
    lens[5], lens[299] = 2500, 2100
    c = Case(lam, 256, 32, 1, 2, "bf16", [1] * 300, lens, seed=3)
    _all(c)


def test_sequences_beyond_one_step_of_the_chip(lam):
    """More tiles than run at once: nothing is split."""
    rng = np.random.default_rng(1)
    lens = [int(x) for x in rng.integers(0, 40, 1100)]
    for rows in ([1] * 1100, [min(l, s % 3) for s, l in enumerate(lens)]):
        c = Case(lam, 64, 32, 1, 1, "f16", rows, lens, seed=2)
        _all(c)


def test_weights_of_a_wide_table(lam):
    """Scores of every column would take over a GiB: the weights come from a second pass."""
    c = Case(lam, 64, 64, 1, 16, "f16", [4, 4], [300, 2500], seed=5)
    wide = torch.zeros((2, (1 << 15) + 1), dtype=torch.int32, device="cuda")
    wide[:, : c.table.shape[1]] = c.table
    c.table = wide
    _all(c)


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_second_pass_of_many_tiles(lam, D, dt):
    """Enough sequences and tokens that a workgroup of the second pass takes 128."""
    rng = np.random.default_rng(D)
    lens = [int(x) for x in rng.integers(35, 300, 40)]
    lens[3], lens[20] = 900, 129
    c = Case(lam, D, 64, 2, 2, dt, [35] * 40, lens, seed=D)
    _all(c)
    _all(c, causal=False, mask=rng.random((40, 2, 900)) > 0.3)


@pytest.mark.parametrize("Hk", [8, 16])
@pytest.mark.parametrize("rows,lens", [([40, 35], [130, 500]), ([33], [77])])
def test_second_pass_of_eight_heads(lam, Hk, rows, lens):
    c = Case(lam, 64, 32, Hk, 3, "bf16", rows, lens, seed=Hk)
    _all(c)


def test_weights_by_both_ways_agree(lam):
    """One row at a time (kept scores) and all rows at once (a second pass) add up to the same."""
    c = Case(lam, 128, 64, 2, 4, "bf16", [48], [1500], seed=6)
    w = torch.zeros((1, 2, 1500), device="cuda")
    out = c.call(causal=False, weights=w)
    one, q = torch.zeros_like(w), c.q
    for i in range(48):
        c.q = q[i:i + 1]
        got = c.call(causal=False, weights=one)
        # an output differs by its own rounding, and by that of the weights to float16
        assert torch.allclose(got[0].float(), out[i].float(), rtol=2.0 ** -7, atol=2.0 ** -9)
    # sums of 48 * 4 weights: each to 2^-20 of itself, and the additions' rounding
    assert ((one - w).abs() <= 2.0 ** -18 * (1 + w)).all()


def test_a_context_of_another_stream(lam):
    """Copies that a call makes of its arguments, and its outputs, are its context's stream's."""
    side = torch.cuda.Stream()
    ctx = lam.Context(stream=side)
    c = Case(lam, 64, 32, 2, 2, "f16", [1, 1], [300, 90], seed=8)
    wide = torch.zeros((2, 2 * c.table.shape[1]), dtype=torch.int32, device="cuda")
    wide[:, ::2] = c.table
    table, lengths = wide[:, ::2], torch.stack([c.lengths, c.lengths], 1)[:, 0]
    q = torch.stack([c.q, c.q], -1)[..., 0]                  # strided: copied
    k, v = torch.randn((2, 2, 2, 64), device="cuda").half()
    w = torch.zeros((2, 2, 600), device="cuda")[..., :300]
    scores = torch.rand((2, 300, 2), device="cuda").transpose(1, 2)
    want_out = c.call()
    busy = torch.randn((4096, 4096), device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):                                      # the current stream has work before it
        busy = busy @ busy * 1e-3
    out = lam.kv_attend(q, c.pool, table, lengths, weights=w, ctx=ctx)
    kept, so, po, lo = lam.kv_evict(c.pool, table, lengths, scores, 100, 64, ctx=ctx)
    lam.kv_append(k, v, c.pool, table, lengths, ctx=ctx)
    got = lam.kv_read(c.pool, table, lengths, 2, 64, torch.float16, ctx=ctx)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out, want_out) and lo.tolist() == [100, 90]
    assert np.array_equal(got[0].double().cpu().numpy(), kv.rounded(k.double().cpu().numpy()))
    assert np.array_equal(got[1].double().cpu().numpy(), kv.rounded(v.double().cpu().numpy()))


def test_starts_that_do_not_rise(lam):
    """Such rows get anything, but nothing outside the call's arrays is touched, and the next call is right."""
    c = Case(lam, 64, 32, 2, 4, "f16", [2, 2, 2, 2], [3000, 90, 2100, 5], seed=7)
    w = torch.zeros((4, 2, 3000), device="cuda")
    for starts in ([0, 8, 0, 8, 0], [8, 6, 4, 2, 0], [-5, 100, -(1 << 31), (1 << 31) - 1, 3]):
        out = lam.kv_attend(c.q, c.pool, c.table, c.lengths, starts=_i32(starts), weights=w)
        assert out.shape == c.q.shape
    torch.cuda.synchronize()
    _all(c)


@pytest.mark.parametrize("kind", ["random", "equal", "odd"])
@pytest.mark.parametrize("L", [2048, 2049, 8192, 8193, 32768, 32769, 65536, 65537])
def test_evict_where_kernels_change(lam, L, kind):
    budget = L - 3 if kind == "equal" else L // 3
    _evict_case(lam, 64, 1024, 1, [L, max(0, L - 1500)], budget, 10, 2, _scores(L, 2, 1, L, kind), None, False, seed=L)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("D,T", [(64, 32), (128, 64), (256, 256)])
@pytest.mark.parametrize("lens,budget", [
    ([1060, 1001, 1000, 3, 1037], 1000),
    ([1064, 1064], 1000),                                    # as many moves as a selection makes itself
    ([1065, 999], 1000),                                     # and one more
    ([70], 6), ([71], 6), ([64, 0, 1], 1), ([3000, 2999], 2990),
])
def test_evict_few(lam, lens, budget, D, T, in_place):
    """A cache a little over its budget, as after every decode step."""
    heads, L = 3, max(lens)
    g = torch.Generator(device="cuda").manual_seed(L + D)
    pos = torch.argsort(torch.rand((len(lens), heads, L), generator=g, device="cuda"), dim=-1).to(torch.int32)
    kind = "ties" if D == 128 else "random"
    _evict_case(lam, D, T, heads, lens, budget, budget // 10, min(2, budget - budget // 10),
                _scores(L, len(lens), heads, L, kind), pos, in_place, seed=L)


def test_evict_few_and_bad_pages(lam):
    pool = torch.randint(0, 256, (2, 1, kv.page_bytes(64, 32)), device="cuda", dtype=torch.int32).to(torch.uint8)
    before = pool.clone()
    w = torch.arange(64.0, device="cuda").view(1, 1, 64)
    kept, _, _, lo = lam.kv_evict(pool, _i32([[0, 99]]), _i32([64]), w, 63, 64)
    assert lo.tolist() == [63] and kept[0, 0].tolist() == [63] + list(range(1, 63)) and torch.equal(pool, before)
    lam.kv_evict(pool, _i32([[-1, 1]]), _i32([64]), w, 63, 64)
    assert torch.equal(pool, before)


@pytest.mark.parametrize("D,n,G", [(64, 1, 4), (128, 2, 7), (128, 40, 2), (256, 1, 2), (256, 30, 4)])
def test_masked_tokens_may_hold_anything(lam, D, n, G):
    """Slots that the mask takes out were never written: scales that are not numbers."""
    T, lens, Hk = 64, [500, 97, 2300], 2
    c = Case(lam, D, T, Hk, G, "bf16", [n] * 3, lens, seed=D + n)
    m = np.random.default_rng(n).random((3, Hk, max(lens))) > 0.3
    m[1, 0] = False
    table, blocks = c.table.cpu().numpy(), D // 32
    s, h, t = np.nonzero(~m & (np.arange(max(lens)) < np.array(lens)[:, None, None]))
    page, t = torch.from_numpy(table[s, t // T]).long().cuda(), t % T
    head, b = torch.from_numpy(h).cuda(), np.arange(blocks)
    at = np.concatenate([T * D + t[:, None] * blocks + b,
                         T * D + T * blocks + (t[:, None] // 4 * blocks + b) * 4 + t[:, None] % 4], axis=1)
    c.pool[page[:, None], head[:, None], torch.from_numpy(at).cuda()] = 255
    _all(c, mask=m)
    _all(c, causal=False, mask=m)


def test_a_graph_outlives_larger_scratch(lam):
    """A recorded call keeps its scratch where later calls of the context need more."""
    c = Case(lam, 128, 64, 2, 4, "bf16", [1, 1], [4100, 2900], seed=3)
    big = Case(lam, 128, 64, 2, 4, "bf16", [8] * 8, [9000] * 8, seed=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    w = torch.zeros((2, 2, 4100), device="cuda")
    with torch.cuda.stream(s):
        ctx = lam.Context(stream=s)
        want = c.call(weights=w, ctx=ctx)
        want_w = w.clone()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            out = c.call(weights=w, ctx=ctx)
        wide = torch.zeros((8, 2, 9000), device="cuda")
        big.check(big.call(weights=wide, ctx=ctx), weights=wide)
    junk = torch.full((1 << 24,), float("nan"), device="cuda")
    for _ in range(3):
        w.zero_()
        out.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(w, want_w)
        assert junk.isnan().all()
