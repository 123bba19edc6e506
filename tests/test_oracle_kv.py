"""Pins of the 4-bit cache's oracle (CPU): the block format against its
definition in rationals, its error bound, the page layout, softmax attention on
closed forms, eviction against hand-worked lists."""
import math

import numpy as np
import pytest

from oracle import kv


def test_values_of_every_code():
    codes = np.arange(16, dtype=np.uint8).repeat(2)
    for e in (kv.E_LO, -3, 0, kv.E_HI):
        want = [m * 2.0 ** e for m in kv.MAGNITUDES] + [-m * 2.0 ** e for m in kv.MAGNITUDES]
        got = kv.decode(codes, np.array([e]))
        assert np.array_equal(got, np.repeat(want, 2))
        assert np.array_equal(got.astype(np.float16).astype(np.float64), got)   # exact in 16 bits


@pytest.mark.parametrize("amax,e", [(0.0, -23), (6.0, 0), (6.0000001, 1), (3.0, -1), (3.01, 0), (49152.0, 13), (1e9, 13),
                                    (1e-12, -23)])
def test_exponent(amax, e):
    assert kv.exponent(amax) == e
    x = np.zeros(32)
    x[7] = -amax
    assert kv.encode(x)[1][0] == e


def test_codes_match_the_definition():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((40, 32)) * 2.0 ** rng.integers(-20, 14, (40, 1))
    # halfway cases at every gap, on a block whose scale is 1
    x[0, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0]
    x[0, 16:] = 0.0
    codes, e = kv.encode(x)
    assert e[0, 0] == 0
    assert list(codes[0, :8]) == [0, 2, 2, 4, 4, 6, 6, 7]
    for i in range(x.shape[0]):
        assert e[i, 0] == kv.exponent(np.abs(x[i]).max())
        assert [int(c) for c in codes[i]] == [kv.code_exact(v, int(e[i, 0])) for v in x[i]]


def test_error_bound():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((500, 64)) * 2.0 ** rng.uniform(-18, 12, (500, 1))
    x = np.clip(x, -49152, 49152)
    codes, e = kv.encode(x)
    err = np.abs(x - kv.decode(codes, e)).reshape(500, 2, 32)
    assert (err <= 2.0 ** e[..., None]).all()
    amax = np.abs(x).reshape(500, 2, 32).max(-1)
    assert (err <= np.where(e > kv.E_LO, amax / 3.0, 2.0 ** kv.E_LO)[..., None]).all()
    assert np.array_equal(kv.rounded(kv.rounded(x)), kv.rounded(x))


def test_nonfinite_is_zero_and_large_saturates():
    x = np.ones(32)
    x[:4] = [math.nan, math.inf, -math.inf, 1e9]
    r = kv.rounded(x)
    assert list(r[:3]) == [0.0, 0.0, 0.0] and r[3] == 49152.0


@pytest.mark.parametrize("D", [64, 128, 256])
def test_page_holds_every_code_once(D):
    T = 32
    rng = np.random.default_rng(D)
    kc, vc = rng.integers(0, 16, (2, T, D), dtype=np.uint8)
    ke, ve = rng.integers(kv.E_LO, kv.E_HI + 1, (2, T, D // 32))
    page = kv.pack_page(kc, ke, vc, ve)
    assert page.size == T * D * 17 // 16
    half = T * D // 2
    nib = np.stack([page & 15, page >> 4], 1).reshape(-1)
    assert np.array_equal(nib[: T * D].reshape(T, D), kc)
    v = nib[T * D: 2 * T * D].reshape(T // 4, 16, 4, D // 16).transpose(0, 2, 1, 3).reshape(T, D)
    assert np.array_equal(v, vc)
    ks = page[2 * half: 2 * half + T * D // 32].reshape(T, -1)
    vs = page[2 * half + T * D // 32:].reshape(T // 4, -1, 4).transpose(0, 2, 1).reshape(T, -1)
    assert np.array_equal(ks, ke + 127) and np.array_equal(vs, ve + 127)


def test_attention_closed_forms():
    v = np.arange(12.0).reshape(6, 2)
    q = np.zeros((2, 2))
    r = kv.attend(q, np.ones((6, 2)), v, 1.0)                    # equal scores: means of what is seen
    assert np.allclose(r["out"], [v[:5].mean(0), v.mean(0)]) and np.allclose(r["lse"], np.log([5, 6]))
    r = kv.attend(q, np.ones((6, 2)), v, 1.0, causal=False, mask=[0, 0, 1, 0, 0, 0])
    assert np.array_equal(r["out"], [v[2], v[2]])
    r = kv.attend(q, np.ones((6, 2)), v, 1.0, mask=np.zeros(6))
    assert np.array_equal(r["out"], np.zeros((2, 2))) and np.all(r["lse"] == -math.inf)
    k = np.zeros((6, 2))
    k[4, 0] = 200.0                                              # one score far above: its value
    assert np.allclose(kv.attend(np.ones((1, 2)), k, v, 1.0)["out"], v[4])
    assert kv.attend(np.ones((3, 2)), np.ones((1, 2)), v[:1], 1.0)["p"].sum(1).tolist() == [0.0, 0.0, 1.0]


def test_eviction_by_hand():
    w = [5.0, 1.0, 4.0, 0.5, 3.0, 9.0, 2.0]
    pos = list(range(7))
    # the four largest are slots 0, 2, 4, 5: holes 1 and 3 take 4 and 5
    assert kv.evict(w, pos, 4, 0, 0) == [0, 4, 2, 5]
    # the newest two and the first one stay
    assert kv.evict(w, pos, 4, 2, 1) == [0, 5, 2, 6]
    # equal scores: the lowest slots
    assert kv.evict([1.0] * 6, pos[:6], 3, 0, 0) == [0, 1, 2]
    assert kv.evict([math.nan, 1.0, -2.0, -0.0, 0.0], pos[:5], 2, 0, 0) == [3, 1]
    assert kv.evict([1.0, 2.0], pos[:2], 4, 1, 1) == [0, 1, -1, -1]
    assert kv.evict([1.0, 2.0, 3.0, 4.0], [9, 3, 7, 10], 2, 2, 0) == [0, 3]


def test_eviction_twice_keeps_the_newest():
    """An eviction puts tokens of the tail into holes, so the last slot then holds an older
    one; the next eviction protects the newest positions all the same."""
    # token 4 takes the place of token 0; then it is the newest, in slot 0
    assert kv.evict([0.0, 5.0, 5.0, 5.0, 1.0], list(range(5)), 4, 1, 0) == [4, 1, 2, 3]
    assert kv.evict([0.0, 1.0, 2.0, 3.0], [4, 1, 2, 3], 2, 1, 0) == [0, 3]
    assert kv.evict([9.0, 1.0, 8.0, 7.0], [9, 8, 2, 1], 2, 2, 0) == [0, 1]
    rng = np.random.default_rng(0)
    moved = 0
    for _ in range(50):
        n, mid, budget, recent, sinks = 100, 64, 32, 16, 2
        w = rng.random(n)
        first = kv.evict(w, list(range(n)), mid, recent, sinks)
        moved += first[-1] != n - 1
        w2 = rng.random(mid)
        second = kv.evict(w2, first, budget, recent, sinks)
        kept = {first[t] for t in second}
        assert set(range(n - recent, n)) <= kept and set(range(sinks)) <= kept
    assert moved > 0
