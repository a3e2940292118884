"""Plain 64-bit references of the context-free operators, for their tests."""
import math

import numpy as np

PAGE = 64


def bf16(x):
    """float64 values rounded to bf16, as uint16 bits (nearest even)."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32)
    r = ((b.astype(np.uint64) + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(np.asarray(x, dtype=np.float32)), np.uint16(0x7FC0), r)


def bf16_value(bits):
    return (np.asarray(bits, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def e4m3_value(codes):
    c = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    e, m = (c & 127) >> 3, c & 7
    v = np.where(e > 0, (1 + m / 8) * np.exp2(e - 7.0), m / 8 * 2.0 ** -6)
    v = np.where((c & 127) == 127, math.nan, v)
    return np.where(c & 128, -v, v)


def page_scale(x):
    """x: the values of one page and head."""
    a = np.abs(x[np.isfinite(x)])
    a = a.max() if a.size else 0.0
    if a == 0:
        return 1.0
    e = math.ceil(math.log2(a / 448)) + 1
    while e > -126 and a <= 448 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** max(e, -126)


def e4m3_round(y):
    """Values |y| <= 448 rounded to the nearest e4m3 number, ties to even; infinities are NaN."""
    a = np.abs(y)
    e = np.where(a > 0, np.floor(np.log2(np.where(a > 0, a, 1))), -6)
    step = np.exp2(np.maximum(e, -6) - 3)
    r = np.copysign(np.rint(a / step) * step, y)
    return np.where(np.isfinite(y), r, math.nan)


def attention(q, k, v, vis, scale):
    """One row: q [D], k, v [slots, D]; returns out, lse and the terms of the error bounds: sum p |v|, max sum |q||k|,
    sum of e^(s - max), max |v|."""
    if vis == 0:
        return np.zeros(v.shape[1]), -math.inf, np.zeros(v.shape[1]), 0.0, 1.0, 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        k, v = k[:vis], v[:vis]
        s = k @ q * scale
        m = s.max()
        e = np.exp(s - m)
        l = e.sum()
        return (e @ v / l, m + math.log(l) if l > 0 else math.nan, e @ np.abs(v) / l,
                float(np.nanmax(np.abs(k) @ np.abs(q)) * abs(scale)), l, float(np.abs(v[np.isfinite(v)]).max(initial=0)))


def scores(x, given, top):
    """One row of logits [V] (float64): log probabilities of given, entropy, top indices, their log probabilities, and
    Z's terms (sum below the maximum, times the maximum occurs, sum of e d)."""
    V = x.size
    order = np.lexsort((np.arange(V), -np.where(np.isnan(x), -math.inf, x)))[:top]
    with np.errstate(invalid="ignore"):
        M = x.max()
        if not np.isfinite(M):
            nan = math.nan
            return np.full(len(given), nan), nan, order, np.full(top, nan), (nan, 1.0, nan)
        d = x - M
        e = np.exp(d)
        S, N = e[d < 0].sum(), float((d == 0).sum())
        T = np.where(e > 0, e * np.where(e > 0, d, 0), 0).sum()
        Z = math.log1p(N - 1 + S)
        lp = d - Z
        g = np.array([lp[t] if 0 <= t < V else math.nan for t in given])
        return g, Z - T / (N + S), order, lp[order], (S, N, T)
