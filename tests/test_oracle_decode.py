"""Pins of oracle.decode: 8-bit rows, rotary positions, decode attention."""

import math

import numpy as np
import pytest

from oracle import decode as od


def test_e4m3_values_match_torch():
    import torch
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = od.e4m3_values()
    assert np.array_equal(np.isnan(t), np.isnan(v)) and np.array_equal(t[~np.isnan(t)], v[~np.isnan(v)])


def test_scale_is_the_next_bf16_up():
    bits = np.arange(0x0080, 0x7f80, dtype=np.uint32) << 16
    all_bf16 = bits.view(np.float32).astype(np.float64)
    rng = np.random.default_rng(5)
    x = np.exp(rng.uniform(-60, 60, 2000))
    assert np.array_equal(od.bf16_up(x), all_bf16[np.searchsorted(all_bf16, x)])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_codes_are_nearest(fmt, dtype):
    rng = np.random.default_rng(7)
    x = rng.standard_normal((50, 64)) * np.exp(rng.uniform(-8, 8, (50, 1)))
    x[0] = 0.0
    codes, s = od.quantise(x, fmt, dtype)
    table = np.arange(-127, 128, dtype=np.float64) if fmt == "int8" else od.e4m3_values()[~np.isnan(od.e4m3_values())]
    best = np.abs(table[None, None] * s[:, None, None] - x[..., None]).min(-1)
    got = np.abs(od.dequantise(codes, s, fmt) - x)
    assert np.all(got <= best * (1 + 1e-12) + 1e-300)
    assert np.all(np.abs(x).max(-1) <= od.TOP[fmt] * s)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_extremes_stay_finite_and_bad_rows_read_as_nan(fmt):
    for dtype in ("bf16", "f16"):
        big = od.LARGEST[dtype]
        x = np.full((1, 64), big)
        x[0, ::2] = -big
        codes, s = od.quantise(x, fmt, dtype)
        v = od.dequantise(codes, s, fmt)
        assert np.all(np.abs(v) < od.OVERFLOW[dtype]) and np.all(np.sign(v) == np.sign(x))
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones((1, 64))
        x[0, 3] = bad
        codes, s = od.quantise(x, fmt, "bf16")
        assert np.isnan(s).all() and not codes.any()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_turns_pairs_and_keeps_relative_scores(layout):
    rng = np.random.default_rng(3)
    theta = od.frequencies(32, 10000.0)
    x = rng.standard_normal((5, 2, 64))
    pos = rng.integers(0, 1000, 5)
    y = od.rotate(x, pos, theta, layout)
    assert np.array_equal(y[..., 32:], x[..., 32:])
    for t in range(5):
        for i in range(16):
            a, b = (i, i + 16) if layout == "half" else (2 * i, 2 * i + 1)
            f = pos[t] * theta[i]
            m = np.array([[math.cos(f), -math.sin(f)], [math.sin(f), math.cos(f)]])
            assert np.allclose(y[t][:, [a, b]], x[t][:, [a, b]] @ m.T, atol=1e-12)
    assert np.allclose(od.rotate(y, -pos, theta, layout), x, atol=1e-12)
    # q at p + 7 against k at p: the same for every p
    q, k = rng.standard_normal((1, 1, 64)), rng.standard_normal((1, 1, 64))
    dots = [float((od.rotate(q, [p + 7], theta, layout) * od.rotate(k, [p], theta, layout)).sum()) for p in (0, 5, 900)]
    assert np.allclose(dots, dots[0], atol=1e-10)


def test_scaled_frequencies_end_where_they_should():
    plain = od.frequencies(128, 500000.0)
    banded = od.frequencies(128, 500000.0, "banded", 8.0, 8192.0, 1.0, 4.0)
    turns = 8192.0 * plain / (2 * math.pi)
    assert np.array_equal(banded[turns >= 4], plain[turns >= 4])
    assert np.allclose(banded[turns <= 1], plain[turns <= 1] / 8)
    ramp = od.frequencies(128, 500000.0, "ramp", 16.0, 4096.0, 1.0, 32.0)
    assert ramp[0] == plain[0] and np.isclose(ramp[-1], plain[-1] / 16)
    for f in (banded, ramp):
        assert np.all(np.diff(f) < 0) and np.all(f <= plain) and np.all(f >= plain / 16 * (1 - 1e-12))


def test_attention_rows():
    rng = np.random.default_rng(9)
    q, k, v = (rng.standard_normal(s) for s in ((3, 4, 16), (20, 2, 16), (20, 2, 16)))
    out, lse, absv, mag = od.attend(q, k, v, [0, 7, 20])
    assert not out[0].any() and np.all(lse[:, 0] == -np.inf)
    s = k[:7, 1] @ q[1, 2] / 4.0
    p = np.exp(s) / np.exp(s).sum()
    assert np.allclose(out[1, 2], p @ v[:7, 1]) and np.isclose(lse[2, 1], np.log(np.exp(s).sum()))
    assert np.all(absv[1:] >= np.abs(out[1:]) - 1e-12) and np.all(mag[1:] > 0)
