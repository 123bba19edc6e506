"""Norms and rotations of heads: the oracle against complex products and hand-made cases, the
library's frequencies, and what its calls refuse before they touch a device (CPU)."""
import ctypes
import math
import os
from fractions import Fraction

import numpy as np
import pytest

from oracle import kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_32256_amd", "liblam.so")
needs_lib = pytest.mark.skipif(not os.path.exists(LIB), reason="liblam.so not built")


# ------------------------------------------------------------------ oracle
def test_angles_are_exact_products():
    assert kv.angle(0, 0.3) == 0.0
    assert kv.angle(7, 0.125) == 0.875
    assert kv.angle(-7, 0.125) == -0.875
    big = kv.angle(2 ** 31 - 1, 1.0)
    a = Fraction(2 ** 31 - 1)
    turn = 2 * kv.PI
    assert abs(Fraction(big) - (a - turn * round(a / turn))) < Fraction(1, 2 ** 52)
    assert abs(float(kv.PI) - math.pi) == 0.0


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_is_a_complex_product(layout):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 40))
    f, _ = kv.frequencies(12)
    pos = [0, 1, 17, 1000, -3]
    y, size = kv.rotate(x, pos, f, layout, 1.25)
    i = np.arange(12)
    a, b = (i, i + 12) if layout == "half" else (2 * i, 2 * i + 1)
    z = (x[..., a] + 1j * x[..., b]) * (1.25 * np.exp(1j * np.array(pos)[:, None] * np.array(f)))[:, None, :]
    assert np.allclose(y[..., a], z.real, atol=1e-12) and np.allclose(y[..., b], z.imag, atol=1e-12)
    assert (y[..., 24:] == x[..., 24:]).all()
    assert (np.abs(y) <= size + 1e-12).all()


def test_norm_of_a_padded_head():
    x = np.zeros((1, 1, 64))
    x[..., :40] = 3.0
    y, _ = kv.rotate(x, [5], [], gain=np.full(64, 2.0), eps=1e-12, norm_dim=40)
    assert np.allclose(y[..., :40], 2.0, atol=1e-9) and (y[..., 40:] == 0).all()


def test_rotations_of_positions_add():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 1, 64))
    f, _ = kv.frequencies(32)
    once, _ = kv.rotate(x, [123], f)
    back, _ = kv.rotate(once, [-100], f)
    assert np.allclose(back, kv.rotate(x, [23], f)[0], atol=1e-12)


def test_windows_by_hand():
    w = kv.in_window(2, 6, 2, 1)
    assert w.tolist() == [[True, False, False, True, True, True], [True, False, False, False, True, True]]
    assert kv.in_window(1, 3, 1, 0).tolist() == [[False, False, True]]
    assert kv.in_window(3, 2, 5, 0).all()


# ------------------------------------------------------------------ frequencies
@needs_lib
@pytest.mark.parametrize("pairs", [1, 2, 20, 64, 128])
@pytest.mark.parametrize("scaling,args", [
    (None, {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
    ("parts", dict(factor=8.0, length=8192.0)), ("parts", dict(factor=32.0, length=100.0, low=1.0, high=4.0)),
])
def test_frequencies(pairs, scaling, args):
    import paper_2609_32256_amd as lam
    if scaling == "base" and pairs == 1:
        with pytest.raises(lam.LamError):
            lam.rotary_frequencies(2, scaling="base", device="cpu", **args)
        return
    for base in (10000.0, 500000.0, 2.0):
        got, amplitude = lam.rotary_frequencies(2 * pairs, base, scaling, device="cpu", **args)
        want, want_amplitude = kv.frequencies(pairs, base, scaling, **args)
        assert got.shape == (pairs,)
        assert np.allclose(got.numpy(), want, rtol=1e-12, atol=0)
        assert math.isclose(amplitude, want_amplitude, rel_tol=1e-14)
    if scaling == "base":
        f, _ = lam.rotary_frequencies(2 * pairs, 10000.0, device="cpu")
        s, _ = lam.rotary_frequencies(2 * pairs, 10000.0, scaling, device="cpu", **args)
        assert s[0] == f[0] and math.isclose(s[-1], f[-1] / 8.0, rel_tol=1e-12)


@needs_lib
def test_frequencies_refused():
    import paper_2609_32256_amd as lam
    for bad in (dict(base=0.0), dict(base=float("nan")), dict(scaling="linear", factor=0.5),
                dict(scaling="linear", factor=float("inf")), dict(scaling="parts", factor=2.0),
                dict(scaling="parts", factor=2.0, length=100.0, low=2.0, high=2.0)):
        with pytest.raises(lam.LamError) as e:
            lam.rotary_frequencies(64, device="cpu", **bad)
        assert e.value.name == "LAM_EINVAL"
    for bad in (dict(rotary_dim=3), dict(rotary_dim=-2), dict(rotary_dim=8, scaling="other"), dict(rotary_dim=1 << 40)):
        with pytest.raises(ValueError):
            lam.rotary_frequencies(device="cpu", **bad)
    assert lam.rotary_frequencies(0, device="cpu")[0].shape == (0,)


@needs_lib
def test_device_0_is_not_the_current_one(monkeypatch):
    """An index of a device is taken as it is, 0 as well (no device is touched)."""
    import torch

    import paper_2609_32256_amd as lam
    asked, make = [], torch.tensor
    monkeypatch.setattr(torch, "tensor", lambda *a, device, **kw: (asked.append(device), make(*a, **kw))[1])
    for device in (0, 1, None, "cpu"):
        lam.rotary_frequencies(8, device=device)
    assert asked == [0, 1, "cuda", "cpu"]
    asked.clear()
    empty = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, device, **kw: (asked.append(device), empty(*a, **kw))[1])
    for device in (0, 1, None, "cpu"):
        lam.kv_pages(2, 1, 64, device=device)
    assert asked == [0, 1, "cuda", "cpu"]


# ------------------------------------------------------------------ refusals, with addresses that nothing touches
A = 1 << 40                      # 16-byte aligned addresses, far apart
CTX = ctypes.c_void_p(A)         # a refused call does not look into its context


def _heads(lam, x=A, row=512, head=64, y=A + (1 << 30), y_row=512, y_head=64, gain=0, gain_type=2, heads=8):
    return lam._HEADS.pack(x, row, head, y, y_row, y_head, gain, gain_type, heads)


def _rotary(lam, freq=A + 64, pairs=32, layout=0, amplitude=1.0):
    return lam._ROTARY.pack(freq, pairs, layout, amplitude)


def _rotate(lam, q=None, k=None, rotary=None, rows=10, dim=64, dtype=1, positions=A + (1 << 35), eps=1e-6, norm_dim=0):
    q = _heads(lam) if q is None else q
    rotary = _rotary(lam) if rotary is None else rotary
    return lam._lib.lam_kv_rotate(CTX, rotary, q, k, rows, dim, dtype, positions, eps, norm_dim)


@needs_lib
def test_rotate_refusals():
    import paper_2609_32256_amd as lam
    far = A + (1 << 33)
    bad = [
        dict(dim=0), dict(dim=260), dict(dim=12), dict(dim=-8), dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=1 << 31),
        dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=-1.0), dict(norm_dim=-1), dict(norm_dim=65),
        dict(positions=None), dict(positions=A + 2),
        dict(rotary=_rotary(lam, pairs=33)), dict(rotary=_rotary(lam, pairs=-1)), dict(rotary=_rotary(lam, layout=2)),
        dict(rotary=_rotary(lam, freq=0)), dict(rotary=_rotary(lam, freq=A + 4)),
        dict(rotary=_rotary(lam, amplitude=float("nan"))), dict(rotary=_rotary(lam, amplitude=1e300)),
        dict(q=_heads(lam, x=0)), dict(q=_heads(lam, y=0)), dict(q=_heads(lam, x=A + 1)), dict(q=_heads(lam, y=far + 1)),
        dict(q=_heads(lam, row=-1)), dict(q=_heads(lam, y_head=-64)), dict(q=_heads(lam, heads=-1)),
        dict(q=_heads(lam, gain=A, gain_type=0)), dict(q=_heads(lam, gain=A + 2)), dict(q=_heads(lam, gain=A, gain_type=7)),
        dict(q=_heads(lam, y_head=32)), dict(q=_heads(lam, y_row=500)), dict(q=_heads(lam, y_row=0)),     # results overlap
        dict(q=_heads(lam, y=A + 64)), dict(q=_heads(lam, y=A, y_row=1024)),                              # in part the rows
        dict(k=_heads(lam, x=far, y=A)), dict(k=_heads(lam, x=A + (1 << 30), y=far)),                     # one's result, the other's rows
        dict(k=_heads(lam, x=far, y=A + (1 << 30) + 128)),                                                # both results
    ]
    for case in bad:
        assert _rotate(lam, **case) == 1, case
        assert lam._lib.lam_last_error()
    assert lam._lib.lam_kv_rotate(None, _rotary(lam), _heads(lam), None, 1, 64, 1, A, 1e-6, 0) == 1
    assert lam._lib.lam_kv_rotate(CTX, None, _heads(lam), None, 1, 64, 1, A, 1e-6, 0) == 1
    assert lam._lib.lam_kv_rotate(CTX, _rotary(lam), None, None, 1, 64, 1, A, 1e-6, 0) == 1
    assert _rotate(lam, rows=0) == 0
    assert _rotate(lam, q=_heads(lam, heads=0, x=0, y=0)) == 0


@needs_lib
def test_rows_in_turn_are_apart():
    """Parts of one product's rows: queries turned in place beside their keys and values are not
    refused for where they lie (but for the positions, so that nothing runs), moved ones are."""
    import paper_2609_32256_amd as lam

    def why(q, k):
        assert _rotate(lam, q=q, k=k, positions=None) == 1
        return lam._lib.lam_last_error().decode()

    row = 12 * 64
    q = dict(x=A, row=row, y=A, y_row=row)
    k = dict(x=A + 2 * 512, row=row, y=A + 2 * 512, y_row=row, heads=2)
    assert "positions" in why(_heads(lam, **q), _heads(lam, **k))
    assert "overlaps" in why(_heads(lam, **q), _heads(lam, **{**k, "x": A + 2 * 448, "y": A + 2 * 448}))
    assert "overlaps" in why(_heads(lam, **q), _heads(lam, **{**k, "x": A + 2 * 700, "y": A + 2 * 700}))
    assert "overlaps" in why(_heads(lam, **q), _heads(lam, **{**k, "row": row + 64, "y_row": row + 64}))
    # results whose heads are the outer axis
    assert "positions" in why(_heads(lam, y_row=64, y_head=640), None)
    assert "overlap" in why(_heads(lam, y_row=64, y_head=639), None)


@needs_lib
def test_append_refusals():
    import paper_2609_32256_amd as lam
    far = A + (1 << 33)

    def view(rows=10, heads=8, dim=64, page=64, starts=0):
        return lam._KV_VIEW.pack(A + (1 << 36), 100, A + (1 << 37), 4, A + (1 << 38), starts, rows, 2, 4, heads, dim, page, 1)

    def call(v=None, rotary=None, q=None, k=None, vals=far, first=None, eps=1e-6, norm_dim=0, status=None, row=512, head=64):
        return lam._lib.lam_kv_rotate_append(CTX, v or view(), rotary or _rotary(lam), q,
                                             _heads(lam, y=0) if k is None else k, vals, row, head, None, None, first, eps,
                                             norm_dim, status)

    bad = [
        dict(v=view(rows=11)), dict(v=view(dim=80)), dict(v=view(page=48)), dict(v=view(heads=0)),
        dict(k=_heads(lam, heads=4)), dict(k=_heads(lam, x=0)), dict(k=_heads(lam, row=-1)), dict(vals=None), dict(vals=far + 1),
        dict(row=-1), dict(head=-1), dict(first=A + 2), dict(status=A + 1), dict(eps=0.0), dict(norm_dim=70),
        dict(rotary=_rotary(lam, pairs=40)),
        dict(q=_heads(lam, x=far, y=A)), dict(q=_heads(lam, y=far)), dict(q=_heads(lam, y=0)),
    ]
    for case in bad:
        assert call(**case) == 1, case
    assert call(v=view(rows=0)) == 0
    # the queries' result beside keys and values of the same rows (refused for the status alone)
    row = 24 * 64
    mine = _heads(lam, x=A, row=row, y=A, y_row=row)
    assert call(q=mine, k=_heads(lam, x=A + 1024, row=row, y=0), vals=A + 2048, row=row, status=A + 1) == 1
    assert "status" in lam._lib.lam_last_error().decode()


@needs_lib
def test_append_results_beside_keys_and_values():
    """Queries turned in place beside the keys and values of one product are found to lie apart from them (the
    call is then refused for its status, so that nothing runs), and moved onto either they are not."""
    import paper_2609_32256_amd as lam
    view = lam._KV_VIEW.pack(A + (1 << 36), 100, A + (1 << 37), 4, A + (1 << 38), 0, 10, 2, 4, 8, 64, 64, 1)
    row = 24 * 64

    def why(at=0, row_q=row, k=A + 1024, v=A + 2048, rows=view):
        q = _heads(lam, x=A + at, row=row_q, y=A + at, y_row=row_q)
        assert lam._lib.lam_kv_rotate_append(CTX, rows, _rotary(lam), q, _heads(lam, x=k, row=row, y=0), v, row, 64, None, None,
                                             None, 1e-6, 0, A + 1) == 1
        return lam._lib.lam_last_error().decode()

    assert "status" in why()
    assert "status" in why(k=A + 2048, v=A + 1024)
    assert "status" in why(at=10 * 2 * row, k=A, v=A + 1024)         # behind the last row
    for at in (2, 128, 1024, 2048, 3070, 2 * row - 2, 2 * row + 1022):
        assert "overlaps" in why(at=at), at
    assert "overlaps" in why(row_q=row + 8) and "overlaps" in why(k=A) and "overlaps" in why(v=A)
    assert "overlaps" in why(k=A + (1 << 30), v=A + 1022)
    empty = lam._KV_VIEW.pack(A + (1 << 36), 100, A + (1 << 37), 4, A + (1 << 38), 0, 0, 2, 4, 8, 64, 64, 1)
    assert "status" in why(rows=empty)


@needs_lib
def test_window_refusals():
    import paper_2609_32256_amd as lam
    view = lam._KV_VIEW.pack(A + (1 << 36), 100, A + (1 << 37), 4, A + (1 << 38), 0, 10, 2, 4, 8, 64, 64, 1)
    empty = lam._KV_VIEW.pack(A + (1 << 36), 100, A + (1 << 37), 4, A + (1 << 38), 0, 0, 2, 4, 8, 64, 64, 1)

    def call(window, sinks, v=view, heads=8, out=A + (1 << 30)):
        return lam._lib.lam_kv_attend_window(CTX, v, A, 512, 64, heads, 0.125, 1, 0, window, sinks, None, None, out, None)

    for window, sinks in ((-1, 0), (0, 1), (5, -1), (-(1 << 63), 0), (0, 1 << 62)):
        assert call(window, sinks) == 1
        assert "window" in lam._lib.lam_last_error().decode()
    assert call(5, 1, heads=12) == 1 and call(5, 1, out=None) == 1
    assert call(5, 1, v=empty) == 0 and call((1 << 63) - 1, (1 << 63) - 1, v=empty) == 0
