"""Oracle for 8-bit KV rows, rotary positions and decode-step attention.

TEST INFRASTRUCTURE ONLY (see the package docstring).  Plain float64 numpy
from the definitions in the public header:

* an 8-bit row of one token and KV head: scale s = max(a / T rounded up to a
  bf16, 2^-126), code = nearest code to x / s (ties to even), one step lower
  where code * s would round to infinity in the element type, a row with a
  NaN or an infinity has s = NaN and codes 0;
* rotary positions: pairs of a head turn by position * theta_i, theta_i
  optionally scaled for long contexts;
* a decode step's rows attend to the shared keys and to their own sequence's
  keys up to their position.

Pins (tests/test_oracle_decode.py): e4m3 decoding against torch's cast of all
256 bytes and encoding against nearest-value search over the code table; the
scale against a search over all bf16; rotation by 2x2 matrices, its inverse
and the shift invariance of q . k; attention against a per-row softmax of the
concatenated keys.
"""

import math

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}
LARGEST = {"bf16": 255.0 * 2.0**120, "f16": 65504.0}
# Magnitudes from here on round to infinity (nearest even).
OVERFLOW = {"bf16": 255.5 * 2.0**120, "f16": 65520.0}


def e4m3_values():
    """The 256 values of the 8-bit format with 3 mantissa bits (NaN at 0x7f and 0xff)."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, (b & 7).astype(np.float64)
    v = np.where(e == 0, m * 2.0**-9, (8 + m) * 2.0**(e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b > 127, -v, v)


def code_values(codes, fmt):
    """Values of code bytes (uint8)."""
    if fmt == "int8":
        return codes.view(np.int8).astype(np.float64)
    return e4m3_values()[codes]


def bf16_up(x):
    """Smallest bf16 (as float64) not below positive x."""
    m, e = np.frexp(x)
    return np.ldexp(np.ceil(m * 256.0), e - 8)


def quantise(x, fmt, dtype):
    """Code bytes (uint8, shape of x) and scales (float64, last axis dropped) of rows x[..., d] (float64)."""
    a = np.abs(x).max(axis=-1)
    finite = np.isfinite(a)
    s = np.maximum(bf16_up(np.where(finite, a, 0.0) / TOP[fmt]), 2.0**-126)
    y = np.where(finite[..., None], x, 0.0) / s[..., None]
    if fmt == "int8":
        c = np.rint(y)
        c = np.where(np.abs(c * s[..., None]) >= OVERFLOW[dtype], c - np.sign(c), c)
        codes = c.astype(np.int8).view(np.uint8)
    else:
        _, e = np.frexp(y)
        unit = np.ldexp(1.0, np.maximum(e - 4, -9))
        v = np.abs(np.rint(y / unit) * unit)
        table = e4m3_values()[:127]
        mag = np.searchsorted(table, v)
        assert np.array_equal(table[mag], v)
        mag = np.where(table[mag] * s[..., None] >= OVERFLOW[dtype], mag - 1, mag)
        codes = (mag + np.where(y < 0, 128, 0)).astype(np.uint8)     # a zero has code 0
    return codes, np.where(finite, s, np.nan)


def dequantise(codes, scales, fmt):
    return code_values(codes, fmt) * scales[..., None]


def frequencies(rotary_dim, base, scaling="plain", factor=1.0, original_len=0.0, low=0.0, high=0.0):
    i = np.arange(rotary_dim // 2, dtype=np.float64)
    theta = base ** (-2.0 * i / rotary_dim)
    if scaling == "plain":
        return theta
    if scaling == "linear":
        return theta / factor
    if scaling == "banded":
        out = []
        for t in theta:
            turns = original_len * t / (2 * math.pi)
            if turns >= high:
                out.append(t)
            elif turns <= low:
                out.append(t / factor)
            else:
                w = (turns - low) / (high - low)
                out.append((1 - w) * t / factor + w * t)
        return np.array(out)
    c = lambda n: rotary_dim * math.log(original_len / (2 * math.pi * n)) / (2 * math.log(base))
    lo, hi = max(0, math.floor(c(high))), min(rotary_dim - 1, math.ceil(c(low)))
    w = np.clip((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
    return (1 - w) * theta + w * theta / factor


def rotate(x, positions, theta, layout, amplitude=1.0):
    """x [t][heads][d] (float64) turned to positions [t]."""
    r = 2 * len(theta)
    y = x.copy()
    f = np.asarray(positions, dtype=np.float64)[:, None, None] * theta
    c, s = np.cos(f) * amplitude, np.sin(f) * amplitude
    i0, i1 = (np.arange(0, r // 2), np.arange(r // 2, r)) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


def attend(q, k, v, limits, scale=None):
    """q [n][hq][d], k and v [t][hkv][d] (float64); row i sees keys below limits[i].  Returns out, lse [hq][n] and,
    for error bounds, sum_j p_j |v_j| and max_j scale * sum_d |q_d k_d| per row (both [n][hq]...)."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out, absv = np.zeros_like(q), np.zeros_like(q)
    lse = np.full((hq, n), -np.inf)
    mag = np.zeros((n, hq))
    for i in range(n):
        t = max(0, int(limits[i]))
        if t == 0:
            continue
        for h in range(hq):
            kh, vh = k[:t, h // g], v[:t, h // g]
            s = scale * (kh @ q[i, h])
            top = s.max()
            e = np.exp(s - top)
            out[i, h] = e @ vh / e.sum()
            absv[i, h] = e @ np.abs(vh) / e.sum()
            lse[h, i] = top + math.log(e.sum())
            mag[i, h] = scale * (np.abs(kh) @ np.abs(q[i, h])).max()
    return out, lse, absv, mag
