"""Rotary positions against the 64-bit oracle."""

import numpy as np
import pytest

from oracle import decode as od

pytestmark = pytest.mark.gpu

SCALINGS = {
    "plain": {}, "linear": dict(factor=4.0), "banded": dict(factor=8.0, original_len=8192.0, low=1.0, high=4.0),
    "ramp": dict(factor=16.0, original_len=4096.0, low=1.0, high=32.0),
}


@pytest.fixture(scope="module")
def sc():
    from _gpu_util import require_gpu
    return require_gpu()


def bound(x, y, theta, layout, dtype, amp, pos):
    """One rounding of the result; sine and cosine in fp32 (of an angle
    reduced in 64 bits: 4 ulp of 1 and the fp32 turn fraction, 2 pi 2^-25)
    and two fp32 products; on both sides the angle itself, pos * theta with
    up to four 64-bit roundings (power, scaling, turns, product)."""
    from _decode_util import HALF_STEP, TINY
    r = 2 * len(theta)
    pair = np.abs(x).copy()
    i0, i1 = (np.arange(r // 2), np.arange(r // 2, r)) if layout == "half" else (np.arange(0, r, 2), np.arange(1, r, 2))
    pair[..., i0] = pair[..., i1] = np.abs(x[..., i0]) + np.abs(x[..., i1])
    pair[..., r:] = 0.0
    angle = 8 * 2.0**-53 * np.abs(np.asarray(pos, dtype=np.float64))[:, None, None]
    fp32 = (4 * 2.0**-24 + 2 * np.pi * 2.0**-25 + 3 * 2.0**-24 + angle) * amp * pair
    return HALF_STEP[dtype] * (np.abs(y) + fp32) + fp32 + TINY[dtype]


CASES = [
    # tokens, q heads, KV heads, head_dim, rotary_dim, layout, scaling, type
    (1, 8, 2, 64, 64, "half", "plain", "bf16"),
    (1, 32, 8, 128, 128, "interleaved", "plain", "f16"),
    (5, 7, 7, 64, 16, "half", "linear", "f16"),
    (3, 3, 1, 128, 48, "half", "banded", "bf16"),
    (1023, 4, 4, 128, 112, "interleaved", "ramp", "bf16"),
    (1025, 5, 1, 128, 128, "half", "ramp", "f16"),
    (1026, 1, 3, 64, 32, "interleaved", "banded", "bf16"),
    (4099, 2, 2, 64, 48, "half", "linear", "bf16"),
]


@pytest.mark.parametrize("t,hq,hkv,d,rot,layout,scaling,dtype", CASES)
@pytest.mark.parametrize("form", ["apart", "strided", "in place"])
def test_rotation(sc, t, hq, hkv, d, rot, layout, scaling, dtype, form):
    import torch
    from _decode_util import TD, device16, host64, rand16
    print("[rope]", t, hq, hkv, d, rot, layout, scaling, dtype, form, flush=True)
    rng = np.random.default_rng(t * 131 + rot)
    kw = SCALINGS[scaling]
    rope = sc.sc_rope_create(d, rot, sc.ROPE_LAYOUTS[layout], base=500000.0, scaling=sc.ROPE_SCALINGS[scaling], **kw)
    theta = od.frequencies(rot, 500000.0, scaling, **kw)
    assert np.allclose(sc.sc_rope_frequencies(rope), theta, rtol=1e-13, atol=0)
    amp = 0.1 * np.log(16.0) + 1.0 if scaling == "ramp" else 1.0
    pos = rng.integers(0, 200000, t)
    pos[0] = 2**31 - 1
    if t > 2:
        pos[1], pos[2] = 0, -77
    q, k = rand16(rng, (t, hq, d), dtype), rand16(rng, (t, hkv, d), dtype)
    p = torch.tensor(pos, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    code = sc.DTYPE_CODES[dtype]
    if form == "strided":      # slices of one projection's rows, padded output rows
        row = torch.full((t, hq + 2 * hkv, d), 3.0, dtype=TD[dtype], device="cuda")
        row[:, :hq], row[:, hq:hq + hkv] = device16(q, dtype), device16(k, dtype)
        qo = torch.full((t, hq * d + 24), 5.0, dtype=TD[dtype], device="cuda")
        ko = torch.full((t, hkv * d + 8), 6.0, dtype=TD[dtype], device="cuda")
        kd = row[:, hq:]
        sc.sc_rope_apply(rope, code, t, p.data_ptr(), row.data_ptr(), row.stride(0), hq, qo.data_ptr(), qo.stride(0),
                         kd.data_ptr(), row.stride(0), hkv, ko.data_ptr(), ko.stride(0), stream)
        torch.cuda.synchronize()
        assert torch.all(qo[:, hq * d:] == 5.0) and torch.all(ko[:, hkv * d:] == 6.0)
        assert torch.all(row[:, hq + hkv:] == 3.0)
        got = [host64(qo[:, :hq * d].reshape(t, hq, d)), host64(ko[:, :hkv * d].reshape(t, hkv, d))]
    else:
        qd, kd = device16(q, dtype), device16(k, dtype)
        qo, ko = (qd, kd) if form == "in place" else (torch.zeros_like(qd), torch.zeros_like(kd))
        sc.sc_rope_apply(rope, code, t, p.data_ptr(), qd.data_ptr(), hq * d, hq, qo.data_ptr(), hq * d, kd.data_ptr(),
                         hkv * d, hkv, ko.data_ptr(), hkv * d, stream)
        torch.cuda.synchronize()
        got = [host64(qo), host64(ko)]
    sc.sc_rope_destroy(rope)
    for x, y in zip((q, k), got):
        ref = od.rotate(x, pos, theta, layout, amp)
        err = np.abs(y - ref)
        b = bound(x, ref, theta, layout, dtype, amp, pos)
        assert np.all(err <= b), (float((err / b).max()), np.unravel_index((err / b).argmax(), err.shape))
        assert np.array_equal(y[..., rot:], x[..., rot:])


def test_counts_of_zero_and_refusals(sc):
    import torch
    x = torch.full((2, 4, 64), 2.0, dtype=torch.bfloat16, device="cuda")
    y = torch.full_like(x, 9.0)
    p = torch.zeros(2, dtype=torch.int32, device="cuda")
    rope = sc.sc_rope_create(64, 64)
    call = sc.sc_rope_apply
    X, Y, P = x.data_ptr(), y.data_ptr(), p.data_ptr()
    call(rope, 0, 0, 0, 0, 0, 4, 0, 0, 0, 0, 4, 0, 0)              # no token: nothing is looked at
    call(rope, 0, 2, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)              # no head
    call(rope, 0, 2, P, 0, 0, 0, 0, 0, X, 256, 4, Y, 256)          # k only, position 0
    torch.cuda.synchronize()
    assert torch.equal(x, y)
    bad = [
        (2, 2, P, X, 256, 4, Y, 256), (0, -1, P, X, 256, 4, Y, 256), (0, 2, P, X, 256, -4, Y, 256),
        (0, 2, 0, X, 256, 4, Y, 256), (0, 2, P + 2, X, 256, 4, Y, 256), (0, 2, P, 0, 256, 4, Y, 256),
        (0, 2, P, X, 256, 4, 0, 256), (0, 2, P, X + 8, 256, 4, Y, 256), (0, 2, P, X, 248, 4, Y, 256),
        (0, 2, P, X, 260, 4, Y, 256), (0, 2, P, X, 256, 4, Y, 128), (0, 2, P, X, 256, 4, X, 264),
    ]
    for dtype, n, pos, q, qs, heads, out, outs in bad:
        with pytest.raises(sc.SwiftCacheError) as e:
            call(rope, dtype, n, pos, q, qs, heads, out, outs, 0, 0, 0, 0, 0)
        assert e.value.status == sc.SC_ERR_INVALID
    with pytest.raises(sc.SwiftCacheError) as e:
        call(rope, 0, 2**31, P, X, 256, 4, Y, 256, 0, 0, 0, 0, 0)
    assert e.value.status == sc.SC_ERR_RANGE
    sc.sc_rope_destroy(rope)
    with pytest.raises(sc.SwiftCacheError):
        sc.sc_rope_create(64, 64, device=4096)


def test_nan_and_infinity_stay_in_their_pair(sc):
    import torch
    rope = sc.sc_rope_create(64, 64)
    x = torch.ones((1, 1, 64), dtype=torch.float16, device="cuda")
    x[0, 0, 5], x[0, 0, 40] = float("nan"), float("inf")
    y, p = torch.zeros_like(x), torch.tensor([3], dtype=torch.int32, device="cuda")
    sc.sc_rope_apply(rope, 1, 1, p.data_ptr(), x.data_ptr(), 64, 1, y.data_ptr(), 64, 0, 0, 0, 0, 0)
    torch.cuda.synchronize()
    bad = sorted(torch.nonzero(~torch.isfinite(y[0, 0])).flatten().tolist())
    assert bad == [5, 8, 37, 40]
    sc.sc_rope_destroy(rope)


def test_more_tokens_than_one_launch_takes(sc):
    """2^26 + 9 tokens in place (8.6 GB), checked around the launches' ends."""
    import torch
    from _decode_util import device16, host64, rand16
    t = 2**26 + 9
    rng = np.random.default_rng(1)
    rope = sc.sc_rope_create(64, 64)
    x = torch.zeros((t, 1, 64), dtype=torch.bfloat16, device="cuda")
    p = torch.arange(t, dtype=torch.int32, device="cuda")
    at = np.concatenate([np.arange(a - 9, a + 9) for a in (9, 2**24, 2**25, 2**26)])
    rows = rand16(rng, (len(at), 1, 64), "bf16")
    x[torch.from_numpy(at).cuda()] = device16(rows, "bf16")
    torch.cuda.synchronize()
    sc.sc_rope_apply(rope, 0, t, p.data_ptr(), 0, 0, 0, 0, 0, x.data_ptr(), 64, 1, x.data_ptr(), 64,
                     torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    sc.sc_rope_destroy(rope)
    theta = od.frequencies(64, 10000.0)
    ref = od.rotate(rows, at, theta, "half")
    y = host64(x[torch.from_numpy(at).cuda()])
    assert np.all(np.abs(y - ref) <= bound(rows, ref, theta, "half", "bf16", 1.0, at))
    assert torch.count_nonzero(x[2**25 + 9:2**26 - 9]) == 0
