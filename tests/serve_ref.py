"""Definitions of the 8-bit serving operators in numpy, 64 bits where they are
not fp32 by definition, with the error bounds their arithmetic allows."""
import numpy as np

import workloads as wl

TOP = {"i8": np.float32(127.0), "e4m3": np.float32(448.0)}
LEAST = np.float32(1e-5)
U = 2.0 ** -24            # fp32: half a step, relative
UB = 2.0 ** -8            # bf16: half a step, relative


def e4m3_table():
    """The 256 values of the 8-bit float with 4 exponent bits, bias 7, no infinity."""
    out = np.zeros(256)
    for c in range(256):
        s, e, m = -1.0 if c & 0x80 else 1.0, (c >> 3) & 15, c & 7
        out[c] = s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        if e == 15 and m == 7:
            out[c] = np.nan
    return out


E4M3 = e4m3_table()


def to_e4m3(x):
    """Nearest code of every value (|x| <= 448 up to rounding), ties to the even code."""
    pos = E4M3[:127]                                   # 0 .. 448, increasing
    a = np.abs(x.astype(np.float64))
    hi = np.clip(np.searchsorted(pos, a), 1, 126)
    lo = hi - 1
    down, up = a - pos[lo], pos[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(a >= 448.0, 126, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def quantise(x, kind):
    """(codes as stored, r) of rows x [..., hd] float32; fp32 by definition."""
    x = np.asarray(x, np.float32)
    a = np.abs(x).max(-1) if x.shape[-1] else np.zeros(x.shape[:-1], np.float32)
    bad = ~np.isfinite(x).all(-1)
    r = np.maximum(np.where(bad, np.float32(1), a), LEAST).astype(np.float32)
    y = np.where(bad[..., None], np.float32(0), x) * (TOP[kind] / r)[..., None]
    code = np.rint(y).astype(np.int8) if kind == "i8" else to_e4m3(y)
    return code, np.where(bad, np.float32(np.nan), r)


def code_values(code, kind):
    return code.astype(np.float64) if kind == "i8" else E4M3[code.view(np.uint8)]


def rounded(x, elem):
    """float32 values as elem holds them."""
    return wl.round_bf16(x) if elem == "bf16" else np.asarray(x, np.float32)


def attention(q, k, v, pos, scale, causal, window):
    """Rows of one request and one K/V head in float64: q [m][hd], k, v [L][hd],
    pos [m] -> o, lse, and for the bounds sum p|v| / l and the largest sum |q||k| scale."""
    L = k.shape[0]
    row = np.arange(L)[None]
    see = np.ones((len(pos), L), bool)
    if causal:
        see &= row <= pos[:, None]
    if window:
        see &= row > pos[:, None] - window
    o = np.zeros((len(pos), v.shape[1]))
    lse = np.full(len(pos), -np.inf)
    mag = np.zeros_like(o)
    big = np.zeros(len(pos))
    for i in range(len(pos)):
        s = see[i]
        if not s.any():
            continue
        z = scale * (k[s] @ q[i])
        top = z.max()
        if np.isnan(z).any():
            o[i], lse[i] = np.nan, np.nan
            continue
        p = np.exp(z - top)
        with np.errstate(invalid="ignore"):
            o[i] = p @ v[s] / p.sum()
            mag[i] = p @ np.abs(v[s]) / p.sum()
        lse[i] = top + np.log(p.sum())
        big[i] = abs(scale) * (np.abs(k[s]) @ np.abs(q[i])).max()
    return o, lse, mag, big
