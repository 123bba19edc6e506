"""The 4-bit key/value cache on the GPU against its oracle: codes and bytes of
kv_append, values of kv_read, selection and moves of kv_evict, all exact; what is
refused; and the long cache (offsets beyond 32 bits)."""
import math

import numpy as np
import pytest
import torch

from oracle import kv

pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
FILL = 0xA5


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _table(n_seqs, cols, spare, seed):
    """A table of distinct pages in an order of its own and the pool's size."""
    n = n_seqs * cols + spare
    perm = np.random.default_rng(seed).permutation(n)[: n_seqs * cols]
    return _i32(perm.reshape(n_seqs, cols).tolist()).reshape(n_seqs, cols), n


def _rows(seed, n, heads, D, dt):
    g = _gen(seed)
    x = torch.randn((n, heads, D), generator=g, device="cuda")
    return (x * torch.exp(1.5 * torch.randn((n, heads, 1), generator=g, device="cuda"))).to(dt)


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


def _expected_pool(pool, table, T, D, slots, k, v):
    """The pool after rows (seq, slot, row) were written into it."""
    pool, table = pool.copy(), table.cpu().numpy()
    (kc, ke), (vc, ve) = kv.encode(k), kv.encode(v)
    half, nb = T * D // 2, D // 32
    for s, slot, r in slots:
        page, t = table[s, slot // T], slot % T
        for h in range(k.shape[1]):
            one = np.zeros((T, D), np.uint8)
            # the bytes of token t in a page that holds it alone, and which bytes those are
            a, b = one.copy(), one.copy()
            a[t], b[t] = kc[r, h], vc[r, h]
            ea, eb = np.full((T, nb), -127), np.full((T, nb), -127)
            ea[t], eb[t] = ke[r, h], ve[r, h]
            run = D // 32
            at = np.concatenate([t * (D // 2) + np.arange(D // 2),
                                 half + ((((t // 4) * 16 + np.arange(16)) * 4 + t % 4)[:, None] * run + np.arange(run)).reshape(-1),
                                 2 * half + t * nb + np.arange(nb),
                                 2 * half + T * nb + ((t // 4) * nb + np.arange(nb)) * 4 + t % 4])
            pool[page, h, at] = kv.pack_page(a, ea, b, eb)[at]
    return pool


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("D,T,heads,rows,lens", [
    (64, 32, 3, [1], [1]),
    (128, 64, 2, [1, 0, 3], [64, 5, 66]),
    (128, 32, 1, [33, 2], [33, 32]),
    (256, 32, 2, [5, 1], [37, 31]),
    (64, 128, 2, [7, 4], [130, 9]),
])
def test_append_bytes(lam, D, T, heads, rows, lens, dt):
    total, B = sum(rows), len(rows)
    table, n = _table(B, -(-max(lens) // T), 2, D + T)
    pool = torch.full((n, heads, kv.page_bytes(D, T)), FILL, dtype=torch.uint8, device="cuda")
    k, v = _rows(1, total, heads, D, DT[dt]), _rows(2, total, heads, D, DT[dt])
    starts = np.concatenate([[0], np.cumsum(rows)])
    lam.kv_append(k, v, pool, table, _i32(lens), starts=_i32(starts.tolist()))
    slots = [(s, lens[s] - rows[s] + i, starts[s] + i) for s in range(B) for i in range(rows[s])]
    want = _expected_pool(np.full(pool.shape, FILL, np.uint8), table, T, D, slots, _np(k), _np(v))
    got = pool.cpu().numpy()
    # the sign of a zero code is free
    def canon(x):
        lo, hi = x & 15, x >> 4
        return np.where(lo == 8, 0, lo) | (np.where(hi == 8, 0, hi) << 4)
    codes = T * D
    assert np.array_equal(canon(got[..., :codes]), canon(want[..., :codes]))
    assert np.array_equal(got[..., codes:], want[..., codes:])
    rk, rv = lam.kv_read(pool, table, _i32(lens), total, D, dtype=DT[dt], starts=_i32(starts.tolist()))
    assert np.array_equal(_np(rk), kv.rounded(_np(k))) and np.array_equal(_np(rv), kv.rounded(_np(v)))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_every_float16_rounds_as_defined(lam, D):
    bits = torch.arange(0, 65536, dtype=torch.int32, device="cuda").to(torch.int16).view(torch.float16)
    bits = bits[torch.isfinite(bits)]
    g = _gen(D)
    x = bits[torch.randperm(bits.numel(), generator=g, device="cuda")]
    x = x[: x.numel() // (2 * D) * 2 * D].view(-1, 2, D)
    # blocks whose values are near each other, so that every code of a scale occurs
    y = bits[bits.float().abs().argsort()][: x.numel()].view(-1, 2, D)
    n = x.shape[0]
    pool = lam.kv_pages(-(-n // 32), 2, D, 32)
    table = torch.arange(pool.shape[0], dtype=torch.int32, device="cuda").view(1, -1)
    lam.kv_append(x, y, pool, table, _i32([n]))
    a, b = lam.kv_read(pool, table, _i32([n]), n, D, dtype=torch.float16)
    assert np.array_equal(_np(a), kv.rounded(_np(x))) and np.array_equal(_np(b), kv.rounded(_np(y)))


def test_append_strided_and_unaligned_rows(lam):
    D, T, heads, n = 128, 64, 4, 29
    g = _gen(5)
    flat = torch.randn(n * (3 * heads) * D + 8, generator=g, device="cuda").to(torch.bfloat16)
    for off in (0, 1, 3):                                   # parts of one projection, at any element
        qkv = flat[off: off + n * 3 * heads * D].view(n, 3 * heads, D)
        k, v = qkv[:, heads:2 * heads], qkv[:, 2 * heads:]
        pool = lam.kv_pages(2, heads, D, T)
        table = _i32([[1, 0]])
        lam.kv_append(k, v, pool, table, _i32([n + 40]))
        a, b = lam.kv_read(pool, table, _i32([n + 40]), n, D)
        assert np.array_equal(_np(a), kv.rounded(_np(k))) and np.array_equal(_np(b), kv.rounded(_np(v)))
    # channels that are not contiguous, heads first, one row for all
    kt = torch.randn((D, heads, n), generator=g, device="cuda").to(torch.bfloat16).permute(2, 1, 0)
    vt = torch.randn((1, heads, D), generator=g, device="cuda").to(torch.bfloat16).expand(n, heads, D)
    lam.kv_append(kt, vt, pool, table, _i32([n]))
    a, b = lam.kv_read(pool, table, _i32([n]), n, D)
    assert np.array_equal(_np(a), kv.rounded(_np(kt))) and np.array_equal(_np(b), kv.rounded(_np(vt)))


def test_append_status_and_side_arrays(lam):
    D, T, heads = 64, 32, 2
    k, v = _rows(3, 6, heads, D, torch.bfloat16), _rows(4, 6, heads, D, torch.bfloat16)
    pool = lam.kv_pages(4, heads, D, T)
    table = _i32([[0, 1], [2, 3]])
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    w = torch.full((2, heads, 50), 7.0, device="cuda")
    pos = torch.full((2, heads, 50), -5, dtype=torch.int32, device="cuda")
    lam.kv_append(k, v, pool, table, _i32([40, 12]), weights=w, positions=pos, first=_i32([100, 200]), status=status)
    assert status.tolist() == [0, 0, 0]
    w, pos = w.cpu().numpy(), pos.cpu().numpy()
    for s, length, first in ((0, 40, 100), (1, 12, 200)):
        new = np.zeros(50, bool)
        new[length - 3: length] = True
        assert (w[s][:, new] == 0).all() and (w[s][:, ~new] == 7).all()
        assert (pos[s][:, new] == first + np.arange(3)).all() and (pos[s][:, ~new] == -5).all()
    k2 = k.clone()
    k2[0, 0, 3], k2[1, 1, 40], k2[2, 0, 5] = math.nan, math.inf, 1e30
    lam.kv_append(k2, v, pool, table, _i32([40, 12]), status=status)
    got = status.tolist()
    assert got[0] == 2 and got[1] == 4 and got[2] == 0       # four lanes share the block that is over
    assert np.array_equal(_np(lam.kv_read(pool, table, _i32([40, 12]), 6, D)[0]), kv.rounded(_np(k2)))
    # tokens without a place: past the table, before the first slot, pages outside the pool
    before = pool.clone()
    status.zero_()
    lam.kv_append(k, v, pool, table, _i32([67, 2]), status=status)
    assert status[2].item() == (3 + 1) * heads
    after = pool.clone()
    status.zero_()
    lam.kv_append(k, v, pool, _i32([[-1, -7], [4, 1 << 30]]), _i32([40, 12]), status=status)
    assert status[2].item() == 6 * heads and torch.equal(pool, after)
    assert torch.equal(before[0], after[0])
    a, _ = lam.kv_read(pool, _i32([[-1, -7], [4, 1 << 30]]), _i32([40, 12]), 6, D)
    assert not a.any()


def test_append_rows_of_no_sequence(lam):
    D, T = 128, 32
    k, v = _rows(5, 9, 1, D, torch.float16), _rows(6, 9, 1, D, torch.float16)
    pool = lam.kv_pages(2, 1, D, T)
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    lam.kv_append(k, v, pool, _i32([[0], [1]]), _i32([3, 4]), starts=_i32([2, 5, 7]), status=status)
    assert status.tolist() == [0, 0, 4]                     # rows 0, 1, 7, 8
    a, _ = lam.kv_read(pool, _i32([[0], [1]]), _i32([3, 4]), 5, D, dtype=torch.float16, starts=_i32([0, 3, 5]))
    assert np.array_equal(_np(a), kv.rounded(_np(k[2:7])))


def test_long_pool_offsets(lam):
    """Pages whose bytes lie beyond 2^32 and 2^33."""
    D, T, heads = 128, 64, 8
    size = kv.page_bytes(D, T)
    n = (9 << 30) // (heads * size)
    pool = torch.empty((n, heads, size), dtype=torch.uint8, device="cuda")
    table = _i32([[n - 1, (5 << 30) // (heads * size), 0]])
    k, v = _rows(7, 150, heads, D, torch.bfloat16), _rows(8, 150, heads, D, torch.bfloat16)
    lam.kv_append(k, v, pool, table, _i32([150]))
    a, b = lam.kv_read(pool, table, _i32([150]), 150, D)
    ra, rb = kv.rounded(_np(k)), kv.rounded(_np(v))
    assert np.array_equal(_np(a), ra) and np.array_equal(_np(b), rb)
    q = _rows(9, 1, heads, D, torch.bfloat16)
    o = _np(lam.kv_attend(q, pool, table, _i32([150])))
    for h in range(heads):
        r = kv.attend(_np(q)[:, h], ra[:, h], rb[:, h], D ** -0.5)
        assert np.all(np.abs(o[:, h] - r["out"]) <= 2.0 ** -8 * np.abs(r["out"]) + 2.0 ** -9 * r["mean"] + 2.0 ** -32 * r["total"])
    kept, *_ = lam.kv_evict(pool, table, _i32([150]), torch.arange(150.0, device="cuda").expand(1, heads, 150).contiguous(), 60, D)
    a, b = lam.kv_read(pool, table, _i32([60]), 60, D)
    old = kept[0, 0].cpu().numpy()
    assert np.array_equal(np.sort(old), np.arange(90, 150))
    assert np.array_equal(_np(a), ra[old]) and np.array_equal(_np(b), rb[old])


# ------------------------------------------------------------------ eviction
def _evict_case(lam, D, T, heads, lens, budget, recent, sinks, scores, positions, in_place, seed=0, cols=None):
    B, L = len(lens), max(max(lens), 1)
    table, n = _table(B, -(-L // T), 1, seed)
    g = _gen(seed)
    pool = torch.randint(0, 256, (n, heads, kv.page_bytes(D, T)), generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
    view = dict(rows=B * L, head_dim=D, dtype=torch.bfloat16)
    # scale bytes that stand for something
    pool[..., T * D:] = 100 + pool[..., T * D:] % 40
    before = [_np(x).reshape(B, L, heads, D) for x in lam.kv_read(pool, table, _i32([L] * B), **view)]
    s, p = scores.clone(), None if positions is None else positions.clone()
    lengths = _i32(lens)
    out = (s, p, lengths) if in_place else None
    kept, so, po, lo = lam.kv_evict(pool, table, lengths, s, budget, D, recent=recent, sinks=sinks, positions=p, out=out)
    after = [_np(x).reshape(B, L, heads, D) for x in lam.kv_read(pool, table, _i32([L] * B), **view)]
    sc = scores.cpu().numpy()
    ps = np.broadcast_to(np.arange(sc.shape[2]), sc.shape) if positions is None else positions.cpu().numpy()
    kept, so, lo = kept.cpu().numpy(), so.cpu().numpy(), lo.cpu().numpy()
    po = None if po is None else po.cpu().numpy()
    for b in range(B):
        length = min(lens[b], sc.shape[2])
        assert lo[b] == min(length, budget)
        for h in range(heads):
            want = kv.evict(sc[b, h, :length], ps[b, h, :length], budget, recent, sinks)
            assert kept[b, h].tolist() == want, (b, h)
            m = min(length, budget)
            old = np.array(want[:m], dtype=int)
            assert np.array_equal(so[b, h, :m], sc[b, h, old], equal_nan=True)
            assert (so[b, h, m:budget] == 0).all()
            if po is not None:
                assert np.array_equal(po[b, h, :m], ps[b, h, old]) and (po[b, h, m:budget] == -1).all()
            for x, y in zip(before, after):
                assert np.array_equal(y[b, :m, h], x[b, old, h])
                assert np.array_equal(y[b, budget:, h], x[b, budget:, h])   # sources are left


def _scores(seed, B, heads, cols, kind):
    g = _gen(seed)
    w = torch.rand((B, heads, cols), generator=g, device="cuda")
    if kind == "ties":
        w = (w * 4).floor()
    if kind == "equal":
        w = torch.ones_like(w)
    if kind == "odd":                                        # NaN, infinities, both zeros, negatives
        pick = torch.randint(0, 6, w.shape, generator=g, device="cuda")
        for i, v in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0)):
            w = torch.where(pick == i, torch.full_like(w, v), w)
        w = torch.where(pick == 5, -w, w)
    return w


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lens,budget,recent,sinks", [
    ([33, 32, 31, 0, 1], 32, 0, 0),
    ([100, 257, 64], 64, 16, 4),
    ([1500, 1025, 2049], 1024, 0, 1),
    ([2500, 90], 7, 3, 4),
    ([70, 2], 1, 1, 0),
])
def test_evict(lam, lens, budget, recent, sinks, kind, in_place):
    _evict_case(lam, 64, 32, 2, lens, budget, recent, sinks, _scores(budget, len(lens), 2, max(max(lens), budget), kind),
                None, in_place and kind != "odd", seed=budget)


@pytest.mark.parametrize("D,T", [(64, 128), (128, 64), (256, 32)])
def test_evict_positions(lam, D, T):
    lens, heads = [700, 300, 450], 3
    g = _gen(D)
    pos = torch.argsort(torch.rand((3, heads, 700), generator=g, device="cuda"), dim=-1).to(torch.int32)
    for in_place in (False, True):
        _evict_case(lam, D, T, heads, lens, 300, 50, 5, _scores(D, 3, heads, 700, "ties"), pos, in_place, seed=D)


def test_evict_columns_bound_lengths_and_bad_pages_stay(lam):
    _evict_case(lam, 64, 32, 1, [200], 40, 0, 0, _scores(1, 1, 1, 150, "random"), None, False)
    pool = lam.kv_pages(2, 1, 64, 32)
    w = torch.arange(64.0, device="cuda").view(1, 1, 64)
    kept, so, po, lo = lam.kv_evict(pool, _i32([[0, 99]]), _i32([64]), w, 32, 64)
    assert not pool.any() and lo.tolist() == [32] and kept[0, 0].tolist() == list(range(32, 64))


@pytest.mark.parametrize("L", [40000, 70001])
def test_evict_long(lam, L):
    _evict_case(lam, 64, 256, 1, [L, L - 777], 9001, 100, 4, _scores(L, 2, 1, L, "ties"), None, True, seed=L)


# ------------------------------------------------------------------ refusals
def test_refusals(lam):
    pool = lam.kv_pages(4, 2, 64, 32)
    table, lens = _i32([[0, 1], [2, 3]]), _i32([10, 20])
    k = torch.zeros((4, 2, 64), dtype=torch.float16, device="cuda")
    for bad in (dict(head_dim=96), dict(head_dim=64, page_size=48), dict(head_dim=64, page_size=16)):
        with pytest.raises(ValueError):
            lam.kv_pages(4, 2, **bad)
    with pytest.raises(TypeError):
        lam.kv_append(k.float(), k.float(), pool, table, lens)
    with pytest.raises(ValueError):
        lam.kv_append(k, k[:2], pool, table, lens)
    with pytest.raises(ValueError):
        lam.kv_append(k[:3], k[:3], pool, table, lens)        # three rows, two sequences, no starts
    with pytest.raises(ValueError):
        lam.kv_append(k[:, :1], k[:, :1], pool, table, lens)  # another number of heads
    with pytest.raises(ValueError):
        lam.kv_append(torch.cat([k, k], 2), torch.cat([k, k], 2), pool, table, lens)   # another head size
    with pytest.raises(ValueError):
        lam.kv_append(k, k, pool, table[:1], lens)
    with pytest.raises(ValueError):
        lam.kv_append(k, k, pool, table, lens, starts=lens)
    with pytest.raises(TypeError):
        lam.kv_append(k, k, pool, table.long(), lens)
    with pytest.raises(TypeError):
        lam.kv_append(k.cpu(), k.cpu(), pool, table, lens)
    with pytest.raises(lam.LamError) as e:
        lam.kv_append(k, k, pool, table, lens, positions=torch.zeros((2, 2, 64), dtype=torch.int32, device="cuda"))
    assert e.value.name == "LAM_EINVAL"
    with pytest.raises(ValueError):
        lam.kv_append(k, k, pool, table, lens, status=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(lam.LamError):
        lam.kv_attend(torch.zeros((4, 3, 64), dtype=torch.float16, device="cuda"), pool, table, lens)
    with pytest.raises(lam.LamError):
        lam.kv_attend(k, pool, table, lens, scale=math.nan)
    with pytest.raises(ValueError):
        lam.kv_attend(k, pool, table, lens, mask=torch.ones((2, 3, 40), dtype=torch.bool, device="cuda"))
    with pytest.raises(TypeError):
        lam.kv_attend(k, pool, table, lens, weights=torch.zeros((2, 2, 40), dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        lam.kv_attend(k, pool, table, lens, weights=torch.zeros((2, 40, 2), device="cuda").transpose(1, 2))
    with pytest.raises(ValueError):
        lam.kv_attend(k, pool, table, lens, out=torch.zeros((4, 2, 128), dtype=torch.float16, device="cuda"))
    with pytest.raises(lam.LamError):                         # one row of weights for every head
        lam.kv_attend(k, pool, table, lens, weights=torch.zeros((2, 1, 40), device="cuda").expand(2, 2, 40))
    w = torch.zeros((2, 2, 40), device="cuda")
    for bad in (dict(budget=0), dict(budget=4, recent=3, sinks=2), dict(budget=4, recent=-1)):
        with pytest.raises(lam.LamError):
            lam.kv_evict(pool, table, lens, w, head_dim=64, **bad)
    with pytest.raises(lam.LamError):                         # outputs shorter than the budget
        lam.kv_evict(pool, table, lens, w, 41, 64, out=(w, None, lens))
    assert not pool.any() and lens.tolist() == [10, 20]


def test_empty_calls(lam):
    pool = lam.kv_pages(2, 2, 64, 32)
    none = torch.empty((0, 2, 64), dtype=torch.float16, device="cuda")
    table, lens = torch.empty((0, 0), dtype=torch.int32, device="cuda"), _i32([])
    lam.kv_append(none, none, pool, table, lens)
    assert lam.kv_attend(none, pool, table, lens).shape == (0, 2, 64)
    assert lam.kv_read(pool, table, lens, 0, 64)[0].shape == (0, 2, 64)
    kept, *_ = lam.kv_evict(pool, table, lens, torch.empty((0, 2, 8), device="cuda"), 4, 64)
    assert kept.shape == (0, 2, 4)
    # sequences without rows or tokens
    table, lens = _i32([[0], [1]]), _i32([0, 0])
    lam.kv_append(none, none, pool, table, lens)
    q = torch.ones((2, 4, 64), dtype=torch.float16, device="cuda")
    lse = torch.empty((2, 4), device="cuda")
    assert not lam.kv_attend(q, pool, table, lens, lse=lse).any() and torch.isneginf(lse).all()
    assert not pool.any()
