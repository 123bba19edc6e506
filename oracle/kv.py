"""Oracle of the 4-bit key/value cache -- test infrastructure only.

Plain binary64 NumPy, sequence by sequence and head by head: the block format
(code by code, from its definition), the layout of a page, norms and rotations of
heads, attention over the values the cache stands for, and eviction as a sort.
"""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

BLOCK = 32
E_LO, E_HI = -23, 13
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ format
def exponent(amax: float) -> int:
    """Smallest integer e with 6 * 2^e >= amax, held to [E_LO, E_HI]."""
    e = E_LO
    while e < E_HI and 6.0 * 2.0 ** e < amax:
        e += 1
    return e


def code_exact(x: float, e: int) -> int:
    """The code of one value, in rationals: nearest magnitude, halfway to the even one."""
    y = abs(Fraction(float(x))) / Fraction(2) ** e
    m = [Fraction(v) for v in MAGNITUDES]
    best = min(range(8), key=lambda i: (abs(y - m[i]), i % 2))
    return best | (8 if x < 0 else 0)


def encode(x):
    """(codes, exponents) of an array whose last axis is a multiple of 32.  NaN and
    Inf count as 0."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isfinite(x), x, 0.0)
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK, BLOCK))
    amax = np.abs(b).max(axis=-1)
    e = np.full(amax.shape, E_LO)
    for k in range(E_LO, E_HI):
        e = np.where(amax > 6.0 * 2.0 ** k, k + 1, e)
    y = np.minimum(np.abs(b) / 2.0 ** e[..., None], 6.0)   # beyond the largest: the largest
    d = np.abs(y[..., None] - np.array(MAGNITUDES))
    # halfway: the even code; argmin takes the first, so even codes are put first
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmin(d[..., order], axis=-1)]
    return (code + 8 * (b < 0)).reshape(x.shape).astype(np.uint8), e


def decode(codes, e):
    m = np.array(MAGNITUDES)[codes & 7] * np.where(codes >= 8, -1.0, 1.0)
    return (m.reshape(e.shape + (BLOCK,)) * 2.0 ** e[..., None]).reshape(codes.shape)


def rounded(x):
    return decode(*encode(x))


def page_bytes(head_dim: int, page_size: int) -> int:
    return page_size * head_dim + page_size * head_dim // 16


def pack_page(kc, ke, vc, ve):
    """Bytes of one head's part of a page from codes [T][D] and exponents [T][D/32]."""
    T, D = kc.shape
    out = np.zeros(page_bytes(D, T), dtype=np.uint8)
    half, run = T * D // 2, D // 16
    for t in range(T):
        for d in range(0, D, 2):
            out[t * (D // 2) + d // 2] = kc[t, d] | (kc[t, d + 1] << 4)
            at = (((t // 4) * 16 + d // run) * 4 + t % 4) * (D // 32) + (d % run) // 2
            out[half + at] = vc[t, d] | (vc[t, d + 1] << 4)
        for b in range(D // BLOCK):
            out[2 * half + t * (D // 32) + b] = ke[t, b] + 127
            out[2 * half + T * (D // 32) + ((t // 4) * (D // 32) + b) * 4 + t % 4] = ve[t, b] + 127
    return out


# ------------------------------------------------------------------ norm and rotation
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628621,
              10 ** 77)


def angle(position: int, frequency: float) -> float:
    """position * frequency modulo a turn, from the exact product."""
    a = int(position) * Fraction(float(frequency))
    return float(a - 2 * PI * round(a / (2 * PI)))


def frequencies(pairs, base=10000.0, scaling=None, factor=1.0, length=0.0, low=1.0, high=32.0):
    """Radians a position of each pair, and the amplitude."""
    if scaling == "base":
        base = base * factor ** (pairs / (pairs - 1))
    f = [base ** (-i / pairs) for i in range(pairs)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        for i, x in enumerate(f):
            turns = length * x / (2 * math.pi)
            f[i] = x if turns >= high else x / factor if turns <= low else \
                x / factor + (x - x / factor) * (turns - low) / (high - low)
    return f, 0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0


def rotate(x, positions, freq, layout="half", amplitude=1.0, gain=None, eps=1e-6, norm_dim=None):
    """Rows x [n, heads, D] normed and turned: (result, size), size being what the errors of
    the result scale with: the sum of the sizes of the terms of each element."""
    y = np.array(x, dtype=np.float64)
    if gain is not None:
        mean = (y * y).sum(-1, keepdims=True) / (norm_dim or y.shape[-1])
        y = y / np.sqrt(mean + eps) * np.asarray(gain, dtype=np.float64)
    out, size = y.copy(), np.abs(y)
    n = len(freq)
    for i, f in enumerate(freq):
        a, b = (i, i + n) if layout == "half" else (2 * i, 2 * i + 1)
        t = np.array([angle(p, f) for p in positions])[:, None]
        u, v = y[..., a], y[..., b]
        out[..., a] = amplitude * (u * np.cos(t) - v * np.sin(t))
        out[..., b] = amplitude * (u * np.sin(t) + v * np.cos(t))
        size[..., a] = size[..., b] = abs(amplitude) * (np.abs(u) + np.abs(v))
    return out, size


# ------------------------------------------------------------------ attention
def in_window(n, length, window, sinks):
    """Which tokens [n, length] the last n tokens' rows have in a window that ends with
    themselves, or among the first."""
    t, at = np.arange(length)[None, :], (length - n + np.arange(n))[:, None]
    return (t > at - window) | (t < sinks)


def attend(q, k, v, scale, causal=True, mask=None):
    """Rows q [n, D] (one head) over values k, v [len, D]: dict of
    out [n, D], p [n, len], lse [n], and what rounding errors scale with: mean
    (sum p |v|), total (sum |v| over the tokens seen) and slack, the largest
    scale * sum_d |q_d k_d| a row has."""
    n, length = q.shape[0], k.shape[0]
    q, k, v = (np.asarray(a, dtype=np.float64) for a in (q, k, v))
    s = scale * (q @ k.T)
    seen = np.ones((n, length), dtype=bool)
    if causal:
        seen &= np.arange(length)[None, :] <= length - n + np.arange(n)[:, None]
    if mask is not None:   # of the tokens, or of each row's
        m = np.asarray(mask, dtype=bool)
        seen &= m if m.ndim == 2 else m[None, :]
    p, lse = np.zeros((n, length)), np.full(n, -math.inf)
    for i in range(n):
        if seen[i].any():
            x = s[i, seen[i]]
            top = x.max()
            ex = np.exp(x - top)
            p[i, seen[i]] = ex / ex.sum()
            lse[i] = top + math.log(ex.sum())
    slack = np.abs(scale) * (np.abs(q) @ np.abs(k).T)
    slack = np.where(seen, slack, 0.0).max(axis=1) if length else np.zeros(n)
    return dict(out=p @ v, p=p, lse=lse, mean=p @ np.abs(v), total=seen.astype(float) @ np.abs(v),
                slack=slack)


# ------------------------------------------------------------------ eviction
def evict(scores, positions, budget, recent, sinks):
    """The old slot of each new one, for one head: scores and positions of its tokens.
    The newest is the largest position, whichever slot has it."""
    n = len(scores)
    if n <= budget:
        return list(range(n)) + [-1] * (budget - n)
    newest = max(int(p) for p in positions)

    def rank(t):
        safe = positions[t] < sinks or positions[t] > newest - recent
        s = float(scores[t])
        return (0 if safe else 1, 0.0 if safe else (math.inf if math.isnan(s) else -s),
                1 if math.isnan(s) and not safe else 0, t)

    chosen = set(sorted(range(n), key=rank)[:budget])
    late = [t for t in range(budget, n) if t in chosen]
    kept = []
    for t in range(budget):
        kept.append(t if t in chosen else late.pop(0))
    assert not late
    return kept
