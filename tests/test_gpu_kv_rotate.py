"""Norms and rotations of heads on the GPU, on their own and on the way into the 4-bit
cache, against the binary64 oracle.

Tolerances, per element: half a unit in the last place of the output's type (2^-8 of
bfloat16's and 2^-11 of float16's value; 2^-25, half of float16's smallest step, below its
normal numbers), and the roundings of float32 before it: 16 of 2^-24 of the sum of the sizes
of the pair's two terms (sine and cosine 4, gain and amplitude 4, the products and their sum
3, the norm's factor 3, and its product).  Keys in the cache are codes of the binary64
value: equal to the oracle's, of which no code is within 1e-9 of being another.
"""
import numpy as np
import pytest
import torch

from oracle import kv

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
ULP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}

pytestmark = pytest.mark.gpu


def _np(x):
    return x.float().cpu().numpy().astype(np.float64)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _freq(f):
    return torch.tensor(f, dtype=torch.float64, device="cuda")


def _rows(seed, n, heads, D, dt, real=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((n, heads, D), generator=g, device="cuda") * torch.exp(torch.randn((heads, D), generator=g, device="cuda"))
    if real is not None:
        x[..., real:] = 0
    return x.to(DT[dt])


def _gain(seed, D, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    return (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(dtype)


def _check(got, x, pos, f, layout, amplitude, gain, eps, norm_dim, dt):
    want, size = kv.rotate(_np(x), pos, f, layout, amplitude, None if gain is None else _np(gain), eps, norm_dim)
    tol = ULP[dt] * np.abs(want) + 16 * 2.0 ** -24 * size + (2.0 ** -25 if dt == "f16" else 0.0)
    assert (np.abs(_np(got) - want) <= tol).all()


# ------------------------------------------------------------------ rows on their own
@pytest.mark.parametrize("D,real", [(64, 64), (128, 128), (256, 256), (8, 8), (40, 40), (80, 80), (96, 96), (192, 192), (128, 80)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dt,norm", [("bf16", True), ("f16", False), ("f16", True)])
def test_rotate(lam, D, real, layout, dt, norm):
    for pairs in sorted({0, 1, real // 8, real // 4, real // 2 - 1, real // 2}):
        f, amplitude = kv.frequencies(pairs, 10000.0) if pairs else ([], 1.0)
        amplitude = 1.1 if pairs % 2 else 1.0
        n, Hq, Hk = 7, 5, 2
        q, k = _rows(D + pairs, n, Hq, D, dt, real), _rows(D + pairs + 1, n, Hk, D, dt, real)
        gq, gk = (_gain(1, D), _gain(2, D, DT[dt])) if norm else (None, None)
        pos = [0, 1, 2, 1000, 65537, -5, 1 << 20]
        got = lam.kv_rotate(q, _freq(f), _i32(pos), k=k, layout=layout, amplitude=amplitude, q_norm=gq, k_norm=gk,
                            eps=1e-5, norm_dim=real)
        _check(got[0], q, pos, f, layout, amplitude, gq, 1e-5, real, dt)
        _check(got[1], k, pos, f, layout, amplitude, gk, 1e-5, real, dt)
        if real < D:
            assert not got[0][..., real:].any()


@pytest.mark.parametrize("rows,Hq,Hk", [(1, 1, 0), (1, 32, 8), (3, 7, 1), (65, 12, 12), (1025, 40, 8), (5000, 3, 3), (2, 129, 65)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_rotate_sizes(lam, rows, Hq, Hk, D):
    f, _ = kv.frequencies(D // 2)
    q = _rows(rows, rows, Hq, D, "bf16")
    k = _rows(rows + 1, rows, Hk, D, "bf16") if Hk else None
    pos = torch.arange(rows, dtype=torch.int32, device="cuda") * 37
    g = _gain(0, D)
    got = lam.kv_rotate(q, _freq(f), pos, k=k, q_norm=g, k_norm=g)
    got = got if Hk else (got,)
    pick = sorted({0, rows // 2, rows - 1})
    for y, x in zip(got, (q, k)):
        _check(y[pick], x[pick], [p * 37 for p in pick], f, "half", 1.0, g, 1e-6, None, "bf16")
    if rows > 100:
        a = pos.double()[:, None, None] * _freq(f)
        u = x.double()
        u = u * torch.rsqrt(u.square().mean(-1, keepdim=True) + 1e-6) * g
        u, v = u.chunk(2, -1)
        want = torch.cat([u * a.cos() - v * a.sin(), u * a.sin() + v * a.cos()], -1)
        assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()


@pytest.mark.parametrize("D,Hq,Hk,layout,pairs", [
    (64, 4, 1, "half", 32), (64, 3, 2, "half", 21), (40, 5, 0, "interleaved", 20), (64, 24, 16, "interleaved", 8),
    (128, 4, 1, "half", 64), (128, 7, 2, "half", 33), (96, 1, 1, "interleaved", 16), (128, 16, 2, "half", 0),
])
def test_few_heads_of_many_rows(lam, D, Hq, Hk, layout, pairs):
    """Waves of four rows each: against waves of one (calls of fewer rows), whose results are the same but
    for the order of a product's factors, and against the oracle at both ends."""
    n = 40961
    f = _freq(kv.frequencies(pairs)[0] if pairs else [])
    q, k = _rows(D, n, Hq, D, "bf16"), _rows(D + 1, n, Hk, D, "bf16") if Hk else None
    pos = (torch.arange(n, dtype=torch.int32, device="cuda") * 7919) % 100003 - 50
    g = _gain(D, D)
    call = dict(layout=layout, amplitude=1.125, q_norm=g, k_norm=g)
    whole = lam.kv_rotate(q, f, pos, k=k, **call)
    whole = whole if Hk else (whole,)
    for x, y in zip((q, k), whole):
        for a in range(0, n, 4099):
            part = lam.kv_rotate(x[a:a + 4099], f, pos[a:a + 4099], layout=layout, amplitude=1.125, q_norm=g)
            got = y[a:a + 4099]
            assert ((got.float() - part.float()).abs() <= 2.0 ** -7 * part.abs().float() + 2.0 ** -19 * x[a:a + 4099].abs().amax()).all()
        ends = [0, 1, 2, 3, 4, n - 2, n - 1]
        _check(y[ends], x[ends], pos[ends].tolist(), f.tolist(), layout, 1.125, g, 1e-6, None, "bf16")
    lam.kv_rotate(q, f, pos, k=k, out=(q, k) if Hk else q, **call)
    assert torch.equal(q, whole[0]) and (not Hk or torch.equal(k, whole[1]))


@pytest.mark.parametrize("pos", [(1 << 31) - 1, -(1 << 31), (1 << 30) + 12345, 999999937])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_positions(lam, pos, layout):
    """Angles of 2^31 radians are as exact as those of one."""
    f, _ = kv.frequencies(64)
    f[1] = 1.0 - 2.0 ** -50
    q = _rows(3, 1, 4, 128, "f16")
    got = lam.kv_rotate(q, _freq(f), _i32([pos]), layout=layout)
    _check(got, q, [pos], f, layout, 1.0, None, 1e-6, None, "f16")


def test_strides_and_in_place(lam):
    """Parts of one product's rows, transposed heads, odd strides and offsets: the same as contiguous ones."""
    for D, layout, pairs in ((64, "half", 32), (128, "interleaved", 40), (128, "half", 37), (256, "half", 128), (80, "half", 20)):
        n, Hq, Hk = 9, 6, 3
        f, _ = kv.frequencies(pairs)
        f, pos, g = _freq(f), _i32(list(range(100, 100 + n))), _gain(D, D)
        q, k = _rows(1, n, Hq, D, "bf16"), _rows(2, n, Hk, D, "bf16")
        call = dict(layout=layout, q_norm=g, k_norm=g)
        want = lam.kv_rotate(q, f, pos, k=k, **call)
        for pad in (0, 8, 3):                                      # rows of one product, 16-byte aligned or not
            whole = torch.zeros((n, (Hq + 2 * Hk) * D + pad), dtype=q.dtype, device="cuda")
            parts = whole[:, : (Hq + 2 * Hk) * D].view(n, Hq + 2 * Hk, D) if pad == 0 else \
                whole.as_strided((n, Hq + 2 * Hk, D), (whole.shape[1], D, 1), pad)[:, :, :]
            a, b = parts[:, :Hq], parts[:, Hq:Hq + Hk]
            a.copy_(q), b.copy_(k)
            rest = parts[:, Hq + Hk:].clone()
            got = lam.kv_rotate(a, f, pos, k=b, **call)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            lam.kv_rotate(a, f, pos, k=b, out=(a, b), **call)
            assert torch.equal(a, want[0]) and torch.equal(b, want[1]) and torch.equal(parts[:, Hq + Hk:], rest)
        qt = q.transpose(0, 1).contiguous().transpose(0, 1)
        assert torch.equal(lam.kv_rotate(qt, f, pos, **{**call, "k_norm": None}), want[0])
        out = torch.zeros((Hq, n, D + 1), dtype=q.dtype, device="cuda").transpose(0, 1)
        lam.kv_rotate(q, f, pos, layout=layout, q_norm=g, out=out[..., :D])
        assert torch.equal(out[..., :D], want[0]) and not out[..., D].any()
        cols = q.transpose(1, 2).contiguous().transpose(1, 2)      # channels apart: copied
        assert torch.equal(lam.kv_rotate(cols, f, pos, layout=layout, q_norm=g), want[0])
        odd = torch.zeros(D + 1, device="cuda")[1:].copy_(g)       # gains that begin anywhere
        assert torch.equal(lam.kv_rotate(q, f, pos, layout=layout, q_norm=odd), want[0])
        one = q[:1].expand(n, Hq, D)                               # one row for all positions
        assert torch.equal(lam.kv_rotate(one, f, pos, layout=layout, q_norm=g),
                           lam.kv_rotate(one.contiguous(), f, pos, layout=layout, q_norm=g))


@pytest.mark.parametrize("layout,pairs", [("half", 32), ("interleaved", 32), ("half", 33)])
def test_what_is_not_finite_stays_in_its_pair_or_head(lam, layout, pairs):
    D = 128
    f, _ = kv.frequencies(pairs)
    x = _rows(5, 4, 3, D, "bf16")
    clean = lam.kv_rotate(x, _freq(f), _i32([1, 2, 3, 4]), layout=layout)
    y = x.clone()
    y[1, 1, 3], y[2, 0, 100], y[3, 2, 127] = float("nan"), float("inf"), float("-inf")
    got = lam.kv_rotate(y, _freq(f), _i32([1, 2, 3, 4]), layout=layout)
    other = 3 + pairs if layout == "half" else 2
    changed = {(1, 1, 3), (1, 1, other), (2, 0, 100), (3, 2, 127)}
    same = torch.ones_like(x, dtype=torch.bool)
    for c in changed:
        same[c] = False
    assert torch.equal(got[same], clean[same])
    assert got[1, 1, 3].isnan() and got[1, 1, other].isnan() and got[2, 0, 100] == float("inf") and got[3, 2, 127] == float("-inf")
    g = torch.ones(D, device="cuda")
    clean = lam.kv_rotate(x, _freq(f), _i32([1, 2, 3, 4]), layout=layout, q_norm=g)
    got = lam.kv_rotate(y, _freq(f), _i32([1, 2, 3, 4]), layout=layout, q_norm=g)
    for r in range(4):
        for h in range(3):
            assert torch.equal(got[r, h], clean[r, h]) != ((r, h) in {(1, 1), (2, 0), (3, 2)})


def test_norms_of_extreme_rows(lam):
    """Rows of zeros, of the type's largest and smallest values."""
    D = 64
    x = torch.zeros((4, 1, D), dtype=torch.bfloat16, device="cuda")
    x[1] = 3.0e38
    x[2] = 1.0e-30
    x[3, 0, 5] = -3.0e38
    y = lam.kv_rotate(x, None, q_norm=torch.ones(D, device="cuda"), eps=1e-6)
    assert not y[0].any() and (y[1] == 1).all()
    assert torch.allclose(y[2].float(), torch.full((D,), 1.0e-27, device="cuda"), rtol=2.0 ** -7, atol=0)
    assert y[3, 0, 5] == -8 and y[3].abs().sum() == 8


@pytest.mark.parametrize("D,Hq,n", [(64, 3, 6), (64, 2, 8200), (128, 1, 8200), (128, 5, 7), (256, 2, 6), (80, 3, 6)])
@pytest.mark.parametrize("layout,pairs", [("half", None), ("half", 5), ("interleaved", 12), ("half", 0)])
def test_norms_of_extreme_rows_with_gains_and_rotations(lam, D, Hq, n, layout, pairs):
    """Rows at both ends of bfloat16's range: what is normed is in the range of its gains, however it is computed
    (the tolerance counts float32's roundings, not its range, and 2^-134, half of bfloat16's smallest step); on the way
    into the cache as well."""
    def check(got, x, pos, gain, eps):
        want, size = kv.rotate(_np(x), pos, f, layout, 1.25, _np(gain), eps)
        assert (np.abs(_np(got) - want) <= 2.0 ** -8 * np.abs(want) + 16 * 2.0 ** -24 * size + 2.0 ** -134).all()

    pairs = D // 2 if pairs is None else pairs
    f = kv.frequencies(pairs)[0] if pairs else []
    sizes = [3.3e38, 1e38, 1e20, 1.0, 1e-30, 2e-38]
    x = (_rows(D, n, Hq, D, "f16").float().sign() * torch.tensor([sizes[i % 6] for i in range(n)], device="cuda")[:, None, None])
    x = (x * (1 - 0.2 * torch.rand(x.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda"))).bfloat16()
    pos = [7 * i + 1 for i in range(n)]
    pick = list(range(6)) + [n - 1]
    for gain, eps in ((4 * _gain(1, D), 1e-6), (_gain(2, D, torch.bfloat16), 1e-80), (1e-3 * _gain(3, D), 1e40)):
        call = dict(layout=layout, amplitude=1.25, q_norm=gain, eps=eps)
        got = lam.kv_rotate(x, _freq(f), _i32(pos), **call)
        assert got.isfinite().all()
        check(got[pick], x[pick], [pos[i] for i in pick], gain, eps)
        if D != 80:
            cols = -(-n // 64)
            pool, table = lam.kv_pages(cols, 1, D, 64), torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
            got = lam.kv_rotate_append(x, x[:, :1], x[:, :1], pool, table, _i32([n]), _freq(f), k_norm=gain, **call)
            check(got[pick], x[pick], pick, gain, eps)
            k, _ = lam.kv_read(pool, table, _i32([n]), n, D)
            exact, _ = kv.rotate(_np(x[pick, :1]), pick, f, layout, 1.25, _np(gain), eps)
            assert np.array_equal(_np(k[pick]), kv.rounded(exact))


@pytest.mark.parametrize("n", [5, 8200])
def test_rotations_of_the_largest_values(lam, n):
    """Without a norm a result that the type holds is found, also where its two terms are beyond it."""
    D, layout, f = 64, "half", kv.frequencies(32)[0]
    x = _rows(4, n, 2, D, "f16").float().sign() * 3.3e38
    x = (x * torch.rand(x.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")).bfloat16()
    got = lam.kv_rotate(x, _freq(f), _i32(list(range(n))), amplitude=1.375)
    pick = list(range(5)) + [n - 1]
    want, size = kv.rotate(_np(x[pick]), pick, f, layout, 1.375)
    y, most = _np(got[pick]), (2 - 2.0 ** -7) * 2.0 ** 127
    err = 2.0 ** -8 * np.abs(want) + 16 * 2.0 ** -24 * size
    fits, over = np.abs(want) + err <= most, np.abs(want) > (2 - 2.0 ** -8) * 2.0 ** 127 + 16 * 2.0 ** -24 * size
    assert fits.sum() > 100 and over.sum() > 10
    assert (np.abs(y - want)[fits] <= err[fits]).all()
    assert np.array_equal(y[over], np.sign(want[over]) * np.inf)


@pytest.mark.parametrize("n", [12, 8200])
@pytest.mark.parametrize("layout,pairs", [("half", 32), ("interleaved", 20), ("half", 13)])
def test_amplitudes_and_gains_at_their_limits(lam, n, layout, pairs):
    """An amplitude of 4 without a norm, and with gains of 2^60 for rows of every size."""
    D, f = 64, kv.frequencies(pairs)[0]
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.rand((n, 2, D), generator=g, device="cuda") * 2 - 1
    pick = list(range(11)) + [n - 1]
    big = (x * 3.3e38).bfloat16()
    got = _np(lam.kv_rotate(big, _freq(f), _i32(list(range(n))), layout=layout, amplitude=4.0)[pick])
    want, size = kv.rotate(_np(big[pick]), pick, f, layout, 4.0)
    most, err = (2 - 2.0 ** -7) * 2.0 ** 127, 2.0 ** -8 * np.abs(want) + 16 * 2.0 ** -24 * size
    fits, over = np.abs(want) + err <= most, np.abs(want) > (2 - 2.0 ** -8) * 2.0 ** 127 + 16 * 2.0 ** -24 * size
    assert fits.sum() > 100 and over.sum() > 100
    assert (np.abs(got - want)[fits] <= err[fits]).all() and np.array_equal(got[over], np.sign(want[over]) * np.inf)
    sizes = torch.tensor([10.0 ** (i % 12 * 7 - 37) for i in range(n)], dtype=torch.float64, device="cuda").clamp(max=3.3e38)
    y = (x.double() * sizes[:, None, None]).bfloat16()            # 1e-37, 1e-30, ... 3e38
    gain = _gain(1, D) * 2.0 ** 59
    got = lam.kv_rotate(y, _freq(f), _i32(list(range(n))), layout=layout, amplitude=4.0, q_norm=gain, eps=1e-76)
    _check(got[pick], y[pick], pick, f, layout, 4.0, gain, 1e-76, None, "bf16")


@pytest.mark.parametrize("eps", [1e-6, 1e-80, 1e-300, 5e-324, 1e300])
@pytest.mark.parametrize("n", [3, 8200])
@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_norms_of_rows_of_zeros(lam, eps, n, dt):
    D = 128
    x = torch.zeros((n, 1, D), dtype=DT[dt], device="cuda")
    g, f = _gain(1, D), _freq(kv.frequencies(64)[0])
    assert not lam.kv_rotate(x, f, _i32(list(range(n))), q_norm=g, eps=eps).any()
    cols = -(-n // 64)
    pool, status = lam.kv_pages(cols, 1, D, 64), _i32([0, 0, 0])
    table = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    assert not lam.kv_rotate_append(x, x, x, pool, table, _i32([n]), f, q_norm=g, k_norm=g, eps=eps, status=status).any()
    assert status.tolist() == [0, 0, 0] and not lam.kv_read(pool, table, _i32([n]), n, D)[0].any()


def test_rotations_add(lam):
    """A key turned to one position and then by a distance is the key at the other (f16: two roundings)."""
    f, _ = kv.frequencies(64)
    k = _rows(9, 3, 2, 128, "f16").clamp(-8, 8)
    a = lam.kv_rotate(lam.kv_rotate(k, _freq(f), _i32([5000, 70, 3])), _freq(f), _i32([-4000, 30, 0]))
    b = lam.kv_rotate(k, _freq(f), _i32([1000, 100, 3]))
    assert ((a.float() - b.float()).abs() <= 4 * 2.0 ** -11 * 16).all()


# ------------------------------------------------------------------ into the cache
def _append_case(lam, D, T, Hq, Hk, dt, rows, lens, layout="half", pairs=None, norm=True, first=None, before=0, after=0,
                 seed=0, packed=False, real=None):
    """Sequences' rows into pages that hold other bytes; everything that the call should write is
    compared, and everything else has to stay."""
    pairs = D // 2 if pairs is None else pairs
    B, n = len(lens), sum(rows)
    total = before + n + after
    cols = max(1, max(-(-x // T) for x in lens))
    perm = np.random.default_rng(seed).permutation(B * cols + 2)[: B * cols].reshape(B, cols)
    pool = torch.full((B * cols + 2, Hk, kv.page_bytes(D, T)), 0xA5, dtype=torch.uint8, device="cuda")
    if packed:
        whole = _rows(seed, total, Hq + 2 * Hk, D, dt, real)
        q, k, v = whole[:, :Hq], whole[:, Hq:Hq + Hk], whole[:, Hq + Hk:]
    else:
        q, k, v = (_rows(seed + i, total, h, D, dt, real) for i, h in enumerate((Hq, Hk, Hk)))
    f, _ = kv.frequencies(pairs) if pairs else ([], 1.0)
    gq, gk = (_gain(seed, D), _gain(seed + 1, D)) if norm else (None, None)
    equal = before == after == 0 and len(set(rows)) == 1
    starts = None if equal else _i32([before + sum(rows[:b]) for b in range(B + 1)])
    w = torch.full((B, Hk, max(lens)), 7.0, device="cuda")
    p = torch.full((B, Hk, max(lens)), -9, dtype=torch.int32, device="cuda")
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    args = (pool, _i32(perm.tolist()), _i32(lens), _freq(f))
    got = lam.kv_rotate_append(q, k, v, *args, starts=starts, first=None if first is None else _i32(first), layout=layout,
                               amplitude=1.0625, q_norm=gq, k_norm=gk, norm_dim=real, weights=w, positions=p, status=status)
    kk, vv = lam.kv_read(pool, args[1], args[2], total, D, dtype=DT[dt], starts=starts)
    assert status.tolist() == [0, 0, (before + after) * Hk]
    at = before
    for b, (r, length) in enumerate(zip(rows, lens)):
        mine, p0 = slice(at, at + r), first[b] if first is not None else length - r
        pos = list(range(p0, p0 + r))
        if r:
            _check(got[mine], q[mine], pos, f, layout, 1.0625, gq, 1e-6, real, dt)
            exact, _ = kv.rotate(_np(k[mine]), pos, f, layout, 1.0625, None if gk is None else _np(gk), 1e-6, real)
            assert np.array_equal(_np(kk[mine]), kv.rounded(exact))
            assert np.array_equal(_np(vv[mine]), kv.rounded(_np(v[mine])))
        new = torch.arange(max(lens), device="cuda")
        new = (new >= length - r) & (new < length)
        assert (w[b][:, new] == 0).all() and (w[b][:, ~new] == 7).all()
        assert (p[b][:, new] == _i32(pos)).all() and (p[b][:, ~new] == -9).all()
        at += r
    assert not got[:before].any() and not got[at:].any()
    # bytes of no new token stay as they were: the same call into pages of other bytes differs there alone
    other = torch.full_like(pool, 0x5A)
    lam.kv_rotate_append(None, k, v, other, *args[1:], starts=starts, first=None if first is None else _i32(first),
                         layout=layout, amplitude=1.0625, k_norm=gk, norm_dim=real)
    assert int((pool == other).sum()) == n * Hk * (D + D // 16)
    return got


@pytest.mark.parametrize("D,T,Hq,Hk,dt,rows,lens", [
    (128, 64, 32, 8, "bf16", [1, 1, 1, 1], [1, 64, 65, 1000]),
    (128, 64, 32, 8, "bf16", [1], [47]),
    (64, 32, 12, 12, "f16", [3, 3], [3, 35]),
    (64, 32, 7, 1, "f16", [33, 1, 0, 70], [33, 129, 5, 71]),
    (256, 64, 4, 2, "bf16", [5, 6], [70, 6]),
    (256, 128, 16, 1, "f16", [200], [200]),
    (128, 1024, 28, 4, "f16", [130, 61, 2], [130, 400, 1025]),
    (64, 64, 3, 2, "bf16", [1] * 70, [1 + 3 * i for i in range(70)]),
    (128, 32, 1, 1, "bf16", [2] * 67, [40] * 67),
])
@pytest.mark.parametrize("layout,norm", [("half", True), ("interleaved", False)])
def test_rotate_append(lam, D, T, Hq, Hk, dt, rows, lens, layout, norm):
    _append_case(lam, D, T, Hq, Hk, dt, rows, lens, layout, norm=norm, seed=D + Hq)
    _append_case(lam, D, T, Hq, Hk, dt, rows, lens, layout, pairs=D // 8, norm=not norm,
                 first=[100000 * b + 17 for b in range(len(lens))], seed=D + Hq + 1, packed=True)


@pytest.mark.parametrize("D,layout,pairs", [(64, "half", 0), (64, "half", 1), (64, "half", 31), (64, "interleaved", 31),
                                            (128, "half", 20), (128, "interleaved", 3), (256, "half", 127), (256, "half", 8)])
def test_rotate_append_parts(lam, D, layout, pairs):
    _append_case(lam, D, 32, 6, 3, "bf16", [9, 2], [40, 2], layout, pairs=pairs, seed=pairs)
    _append_case(lam, D, 32, 6, 3, "f16", [9, 2], [40, 2], layout, pairs=pairs, seed=pairs, packed=True, norm=False, first=[-7, 0])


@pytest.mark.parametrize("D,Hq,Hk,layout,pairs,norm", [
    (64, 4, 1, "half", 32, True), (64, 2, 3, "half", 21, False), (64, 0, 2, "interleaved", 20, True),
    (128, 4, 1, "half", 64, True), (128, 3, 2, "half", 33, True), (128, 1, 1, "interleaved", 16, False),
])
def test_few_heads_of_many_rows_into_the_cache(lam, D, Hq, Hk, layout, pairs, norm):
    """Waves of four rows each, ragged, with rows of no sequence and tokens without a place: the codes
    and the queries of calls of fewer rows."""
    rows, T = [9001, 0, 3, 12345, 1], 64
    lens = [9001, 7, 100, 12600, 1]
    before, after = 2, 6
    n = sum(rows) + before + after
    f = _freq(kv.frequencies(pairs)[0])
    q = _rows(D, n, Hq, D, "f16") if Hq else None
    k, v = _rows(D + 1, n, Hk, D, "f16"), _rows(D + 2, n, Hk, D, "f16")
    g = _gain(D, D) if norm else None
    cols = -(-max(lens) // T)
    table = torch.arange(5 * cols, dtype=torch.int32, device="cuda").view(5, cols).flip(1).contiguous()
    table[3, 190] = -1
    first = _i32([0, 5, 100000, -40, 9])
    starts = np.cumsum([before] + rows)
    call = dict(layout=layout, amplitude=1.125, q_norm=g if Hq else None, k_norm=g)
    pool, status = lam.kv_pages(5 * cols, Hk, D, T), _i32([0, 0, 0])
    got = lam.kv_rotate_append(q, k, v, pool, table, _i32(lens), f, starts=_i32(starts.tolist()), first=first, status=status, **call)
    lost = min(max(0, 191 * T - (12600 - 12345)), 12345) - max(0, 190 * T - (12600 - 12345))
    assert status.tolist() == [0, 0, (before + after + lost) * Hk]
    want_pool = lam.kv_pages(5 * cols, Hk, D, T)
    for b in range(5):
        for a in range(0, rows[b], 1000):                         # the same tokens, a thousand at a time
            m = min(1000, rows[b] - a)
            at = slice(starts[b] + a, starts[b] + a + m)
            length = _i32([lens[b] - rows[b] + a + m])
            part = lam.kv_rotate_append(None if q is None else q[at], k[at], v[at], want_pool, table[b:b + 1], length, f,
                                        first=first[b:b + 1] + a, **call)
            if Hq:
                tol = 2.0 ** -10 * part.float().abs() + 2.0 ** -19 * q[at].float().abs().amax() + 2.0 ** -24
                assert ((got[at].float() - part.float()).abs() <= tol).all()
    assert torch.equal(pool, want_pool)
    if Hq:
        assert not got[:before].any() and not got[-after:].any()


def test_rotate_append_of_padded_heads_and_rows(lam):
    _append_case(lam, 128, 64, 8, 4, "bf16", [3, 40], [9, 64], real=80, pairs=40, before=2, after=5, seed=4)
    _append_case(lam, 64, 64, 8, 4, "f16", [1, 1, 1], [9, 64, 1], real=40, pairs=20, layout="interleaved", after=300, seed=5)
    _append_case(lam, 64, 64, 2, 1, "f16", [0, 0], [9, 64], before=1, after=2, seed=6)


@pytest.mark.parametrize("n", [40, 9000])                         # a wave a part of a row; four rows
def test_rotate_append_in_place(lam, n):
    """Queries turned in place beside their keys and values, as one product leaves all three."""
    D, Hq, Hk, T = 64, 3, 1, 64
    whole = _rows(n, n, Hq + 2 * Hk, D, "bf16")
    q, k, v = whole.split((Hq, Hk, Hk), dim=1)
    table = torch.arange(-(-n // T), dtype=torch.int32, device="cuda").view(1, -1)
    f, g = _freq(kv.frequencies(32)[0]), _gain(1, D)
    a, b = (lam.kv_pages(table.numel(), Hk, D, T) for _ in range(2))
    want = lam.kv_rotate_append(q, k, v, a, table, _i32([n]), f, q_norm=g, k_norm=g)
    rest = whole[:, Hq:].clone()
    got = lam.kv_rotate_append(q, k, v, b, table, _i32([n]), f, q_norm=g, k_norm=g, out=q)
    assert got is q and torch.equal(q, want) and torch.equal(a, b) and torch.equal(whole[:, Hq:], rest)


def test_without_norm_and_rotation_it_is_an_append(lam):
    D, T, Hk = 128, 64, 4
    k, v = _rows(1, 37, Hk, D, "f16"), _rows(2, 37, Hk, D, "f16")
    table, lengths = _i32([[1, 0]]), _i32([100])
    a, b = lam.kv_pages(2, Hk, D, T), lam.kv_pages(2, Hk, D, T)
    lam.kv_append(k, v, a, table, lengths)
    assert lam.kv_rotate_append(None, k, v, b, table, lengths, None) is None
    assert torch.equal(a, b)


def test_borders_of_the_codes_are_decided_exactly(lam):
    """Keys whose value lies a relative 1e-9 to either side of a border between codes: float32
    would put half of them on it, and the tie to the even code."""
    D, Hk = 64, 1
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    x = torch.zeros((14, Hk, D), dtype=torch.float16, device="cuda")
    x[:, 0, 0] = 6.0                                              # the block's largest: a scale of 1
    amplitudes, want = [], []
    for i in range(14):
        x[i, 0, 1:8] = torch.tensor(mids, dtype=torch.float16, device="cuda")
    for side, up in ((1 - 1e-9, False), (1 + 1e-9, True)):
        pool = lam.kv_pages(1, Hk, D, 64)
        # a rotation by no angle whose amplitude is the factor
        x6 = x.clone()
        x6[:, 0, 0] = 5.5
        lam.kv_rotate_append(None, x6, x6, pool, _i32([[0]]), _i32([14]), torch.zeros(32, dtype=torch.float64, device="cuda"),
                             amplitude=side)
        k, v = lam.kv_read(pool, _i32([[0]]), _i32([14]), 14, D, dtype=torch.float16)
        m = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        assert k[0, 0, 1:8].tolist() == [m[i + 1] if up else m[i] for i in range(7)]
        assert v[0, 0, 1:8].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0]      # values: ties to the even code
    # the scale's own border: 6 (1 + 1e-9) needs the next one
    for side, e in ((1.0, 0), (1 - 1e-9, 0), (1 + 1e-9, 1)):
        pool = lam.kv_pages(1, Hk, D, 64)
        lam.kv_rotate_append(None, x[:1], x[:1], pool, _i32([[0]]), _i32([1]), torch.zeros(32, dtype=torch.float64, device="cuda"),
                             amplitude=side)
        assert pool[0, 0, 64 * D].item() - 127 == e


def test_counts_of_what_cannot_be_held(lam):
    D, Hk = 64, 2
    k, v = (torch.ones((6, Hk, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[0, 0, 3], v[1, 1, 5], k[2, 1, 40] = float("nan"), float("inf"), 60000.0
    status = torch.zeros(3, dtype=torch.int32, device="cuda")
    pool = lam.kv_pages(2, Hk, D, 32)
    table, lengths = _i32([[0, 9], [1, -1]]), _i32([3, 34])       # a page outside the pool
    q = _rows(1, 6, 3, D, "bf16")
    f = _freq(kv.frequencies(32)[0])
    got = lam.kv_rotate_append(q, k, v, pool, table, lengths, f, status=status)
    # the second sequence's rows are tokens 31, 32 and 33: two have no place
    assert status.tolist()[0] >= 2 and status.tolist()[1] >= 1 and status.tolist()[2] == 2 * Hk
    _check(got, q, [0, 1, 2, 31, 32, 33], kv.frequencies(32)[0], "half", 1.0, None, 1e-6, None, "bf16")
    kk, vv = lam.kv_read(pool, table, lengths, 6, D)
    assert kk[0, 0, 3] == 0 and kk[0, 0, 35] == 0 and vv[1, 1, 5] == 0 and not kk[4:].any()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,pairs,Hq,Hk,n", [
    (64, 0, 0, 2, 5), (64, 3, 2, 3, 40), (128, 16, 4, 2, 5), (128, 33, 0, 5, 12), (256, 20, 1, 2, 9),
    (64, 8, 1, 2, 8200), (64, 5, 0, 1, 8200), (128, 0, 1, 1, 8200), (128, 24, 0, 2, 8200),     # waves of four rows
])
def test_what_is_not_finite_stays_in_its_pair_on_the_way_into_the_cache(lam, D, pairs, Hq, Hk, n, layout):
    """Channels that are not turned have no other one to spoil, and each is counted by the one thread that holds it."""
    T = 64
    q = _rows(1, n, Hq, D, "bf16") if Hq else None
    k, v = _rows(2, n, Hk, D, "bf16"), _rows(3, n, Hk, D, "bf16")
    f = kv.frequencies(pairs)[0] if pairs else []
    exact, _ = kv.rotate(_np(k), range(n), f, layout, 1.0625)
    # one element a row, so that no thread meets two: channels past the pairs, their neighbours, a turned one
    spoiled, places = 0, [2 * pairs, 2 * pairs + 1, D - 1, D - 2, 2 * pairs + 6] + ([pairs] if pairs else [])
    rows = np.linspace(0, n - 1, min(n, 60)).astype(int) // (4 if n > 1000 else 1) * (4 if n > 1000 else 1)
    for i, r in enumerate(sorted(set(rows.tolist()))):
        c, h = places[i % len(places)], i % Hk
        k[r, h, c] = (float("nan"), float("inf"), float("-inf"))[i % 3]
        other = c
        if c < 2 * pairs:
            other = c ^ 1 if layout == "interleaved" else c + pairs if c < pairs else c - pairs
        exact[r, h, [c, other]] = np.nan
        spoiled += 1 if c // 8 == other // 8 else 2
    cols = -(-n // T)
    pool, status = lam.kv_pages(cols, Hk, D, T), _i32([0, 0, 0])
    table = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    lam.kv_rotate_append(q, k, v, pool, table, _i32([n]), _freq(f), layout=layout, amplitude=1.0625, status=status)
    got, _ = lam.kv_read(pool, table, _i32([n]), n, D, dtype=torch.bfloat16)
    assert np.array_equal(_np(got), kv.rounded(exact))
    assert status.tolist() == [spoiled, 0, 0]
    if pairs == 0:                                                # as they are: lam_kv_append's bytes
        plain = lam.kv_pages(cols, Hk, D, T)
        lam.kv_rotate_append(None, k, v, pool.zero_(), table, _i32([n]), _freq(f), layout=layout)
        lam.kv_append(k, v, plain, table, _i32([n]))
        assert torch.equal(pool, plain)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("D,Hq,Hk,n,layout", [
    (64, 3, 1, 48, "half"), (64, 0, 5, 48, "interleaved"), (128, 2, 3, 48, "half"), (128, 8, 6, 5000, "interleaved"), (256, 1, 2, 48, "half"),
    (64, 4, 1, 8200, "half"), (64, 0, 3, 8200, "interleaved"), (128, 1, 2, 8200, "half"),       # waves of four rows
])
def test_counts_are_of_the_threads_that_met_them(lam, D, Hq, Hk, n, layout, norm):
    """A thread holds eight channels of a token and head, four hold a block: one element that is not finite is met
    by the one that holds it and by that of its pair's other channel, with a norm by all of its head;
    a block out of range by its four.  Lanes that repeat a head or a row and waves that share one count nothing twice."""
    pairs, T, seen = D // 4, 32, [0, 0]
    q = _rows(1, n, Hq, D, "bf16") if Hq else None
    k, v = _rows(2, n, Hk, D, "bf16").clamp(-8, 8), _rows(3, n, Hk, D, "bf16").clamp(-8, 8)
    cols = -(-n // T)
    last = (cols - 1) * T
    k[last:], v[last:] = float("nan"), 60000.0                    # without a place: not counted but as such
    for i, r in enumerate(range(1, last - 6, max(12, n // 50 // 4 * 4))):   # rows apart, so that no thread meets two
        h, c = (i * 7) % Hk, (i * 13) % D
        k[r, h, c] = (float("nan"), float("inf"), float("-inf"))[i % 3]
        other = c if c >= 2 * pairs else c ^ 1 if layout == "interleaved" else (c + pairs) % (2 * pairs)
        seen[0] += D // 8 if norm else len({c // 8, other // 8})
        v[r + 4, h, (i * 5) % D] = float("nan")
        v[r + 4, h, D - 1 - (i * 5) % D] = 60000.0                # another block of the same head
        seen[0] += 1
        seen[1] += 4
        if not norm:
            k[r + 6, h, 2 * pairs + (i * 3) % (D - 2 * pairs)] = -50000.0
            seen[1] += 4
    table = torch.arange(cols, dtype=torch.int32, device="cuda").view(1, cols)
    table[0, cols - 1] = -1
    status, pool, f = _i32([0, 0, 0]), lam.kv_pages(cols, Hk, D, T), _freq(kv.frequencies(pairs)[0])
    for times in (1, 2):                                          # added to
        lam.kv_rotate_append(q, k, v, pool, table, _i32([n]), f, layout=layout, k_norm=torch.ones(D, device="cuda") if norm else None,
                             status=status)
        assert status.tolist() == [times * seen[0], times * seen[1], times * (n - last) * Hk]


# ------------------------------------------------------------------ streams, graphs, refusals
def test_another_stream_and_a_graph(lam):
    D, Hq, Hk, B = 128, 8, 2, 3
    f, g = _freq(kv.frequencies(64)[0]), _gain(3, D)
    q, k, v = (_rows(i, B, h, D, "bf16") for i, h in enumerate((Hq, Hk, Hk)))
    table, lengths, first = _i32([[0], [1], [2]]), _i32([5, 9, 64]), _i32([4, 8, 63])

    def step(pool, q, out, ctx=None):
        lam.kv_rotate_append(q, k, v, pool, table, lengths, f, first=first, q_norm=g, k_norm=g, out=out, ctx=ctx)
        return lam.kv_rotate(out, f, first, ctx=ctx)

    want_pool, want = lam.kv_pages(3, Hk, D, 64), torch.empty_like(q)
    want_again = step(want_pool, q, want)
    side = torch.cuda.Stream()
    ctx = lam.Context(stream=side)
    pool, out = lam.kv_pages(3, Hk, D, 64), torch.empty_like(q)
    torch.cuda.synchronize()
    again = step(pool, q, out, ctx)
    side.synchronize()
    assert torch.equal(pool, want_pool) and torch.equal(out, want) and torch.equal(again, want_again)

    graph = torch.cuda.CUDAGraph()
    q2 = q.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        again = step(pool, q2, out, ctx)
    for i in range(4):
        q2.copy_(_rows(50 + i, B, Hq, D, "bf16"))
        first += 10
        pool.zero_()
        graph.replay()
        eager_pool, eager = lam.kv_pages(3, Hk, D, 64), torch.empty_like(q)
        eager_again = step(eager_pool, q2, eager)
        torch.cuda.synchronize()
        assert torch.equal(pool, eager_pool) and torch.equal(out, eager) and torch.equal(again, eager_again)


def test_binding_refusals(lam):
    D, Hq, Hk = 64, 4, 2
    q, k = _rows(1, 6, Hq, D, "bf16"), _rows(2, 6, Hk, D, "bf16")
    f, pos, g = _freq(kv.frequencies(32)[0]), _i32([0] * 6), _gain(1, D)
    ok = dict(q=q, frequencies=f, positions=pos, k=k, q_norm=g)

    def bad(error, **change):
        with pytest.raises(error):
            lam.kv_rotate(**{**ok, **change})

    bad(TypeError, q=q.float())
    bad(TypeError, q=q.cpu())
    bad(ValueError, q=q[0])
    bad(TypeError, frequencies=f.float())
    bad(lam.LamError, frequencies=torch.cat([f, f]))
    bad(TypeError, positions=pos.long())
    bad(ValueError, positions=pos[:5])
    bad(ValueError, positions=None)
    bad(ValueError, k=k[:5])
    bad(ValueError, k=k.half())
    bad(ValueError, layout="other")
    bad(lam.LamError, amplitude=float("inf"))
    bad(TypeError, q_norm=g.double())
    bad(TypeError, q_norm=g.half())
    bad(ValueError, q_norm=g[:60])
    bad(lam.LamError, eps=0.0)
    bad(ValueError, norm_dim=0)
    bad(lam.LamError, norm_dim=65)
    bad(ValueError, out=(torch.empty_like(q)[:5], torch.empty_like(k)))
    bad(TypeError, out=(torch.empty_like(q).half(), torch.empty_like(k)))
    bad(lam.LamError, out=(torch.empty_like(q), torch.empty_like(q)[:, :1].expand(6, Hk, D)))
    bad(lam.LamError, out=(k.new_empty(0).set_(k.untyped_storage(), 0, (6, Hq, D), (Hk * D, 0, 1)), torch.empty_like(k)))
    for name, t in (("q", q), ("k", k), ("q_norm", g), ("frequencies", f)):
        bad(ValueError, **{name: t.clone().requires_grad_()})
    with torch.no_grad():
        lam.kv_rotate(q.clone().requires_grad_(), f, pos)
    with pytest.raises(lam.LamError):
        lam.kv_rotate(_rows(1, 2, 1, 264, "bf16"), None)
    assert lam.kv_rotate(q[:0], f, pos[:0]).shape == (0, Hq, D)

    pool, table, lengths = lam.kv_pages(2, Hk, D, 32), _i32([[0], [1]]), _i32([3, 3])
    ok = dict(q=q, k=k, v=k.clone(), pages=pool, table=table, lengths=lengths, frequencies=f)

    def bad_append(error, **change):
        with pytest.raises(error):
            lam.kv_rotate_append(**{**ok, **change})

    bad_append(ValueError, q=q[:5])
    bad_append(ValueError, k=q, v=q)
    bad_append(ValueError, v=q)
    bad_append(ValueError, q=None, out=q)
    bad_append(ValueError, first=_i32([1]))
    bad_append(TypeError, first=torch.zeros(2, device="cuda"))
    bad_append(ValueError, status=_i32([0, 0]))
    bad_append(lam.LamError, out=k.new_empty(0).set_(k.untyped_storage(), 0, (6, Hq, D), (Hk * D // 2, 1, 1)))
    bad_append(ValueError, k=k.clone().requires_grad_())
    assert not pool.any()
