"""Pools of 8-bit blocks: stored bytes, fetched values and stacks against the
64-bit oracle."""

import numpy as np
import pytest

from oracle import attention as oa
from oracle import decode as od

pytestmark = pytest.mark.gpu
FORMATS = ["int8", "e4m3"]
DTYPES = ["bf16", "f16"]


@pytest.fixture(scope="module")
def sc():
    from _gpu_util import require_gpu
    return require_gpu()


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def place(rng, lens, block, blocks):
    per = [-(-x // block) for x in lens]
    ids = rng.permutation(blocks)[:sum(per)]
    cu = np.concatenate([[0], np.cumsum(per)])
    return ids, cu


def store_and_compare(sc, pool, ids, cu, p, n, k, v, layer):
    """Stores rows k, v; every byte of the table's blocks must be the oracle's."""
    import torch
    from _decode_util import device16
    lists = [ids[a:b] for a, b in zip(cu[:-1], cu[1:])]
    before = {(int(i), h): pool.bytes_of(i, layer, h) for i in ids for h in (0, 1)}
    other = {(int(i), h): pool.bytes_of(i, 1 - layer, h) for i in ids for h in (0, 1)}
    t = pool.table(ids, cu, p, n)
    kd, vd = device16(k, pool.dtype), device16(v, pool.dtype)
    sc.sc_store_layer_kv(pool.handle, t, layer, kd.data_ptr(), vd.data_ptr(), stream())
    torch.cuda.synchronize()
    row, off = pool.heads * pool.d, pool.block * pool.heads * pool.d
    at = 0
    from _decode_util import scale_bits
    for b, (pp, nn) in enumerate(zip(p, n)):
        for h, x in ((0, k), (1, v)):
            codes, s = od.quantise(x[at:at + nn], pool.fmt, pool.dtype)
            sb = scale_bits(s)
            for i in range(nn):
                blk, r = divmod(pp + i, pool.block)
                want = before[(int(lists[b][blk]), h)]
                want[r * row:(r + 1) * row] = codes[i].reshape(-1)
                want[off + 2 * r * pool.heads:off + 2 * (r + 1) * pool.heads] = sb[i].view(np.uint8)
        at += nn
    for (i, h), want in before.items():
        got = pool.bytes_of(i, layer, h)
        assert np.array_equal(got, want), (i, h, np.nonzero(got != want)[0][:8])
        assert np.array_equal(pool.bytes_of(i, 1 - layer, h), other[(i, h)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,d,block,p,n", [
    (8, 128, 16, [5, 0, 32, 31], [40, 1, 16, 0]), (3, 64, 7, [3, 6], [1, 20]), (1, 64, 1, [2], [3]),
    (2, 128, 256, [200], [300]),
])
def test_stored_bytes(sc, fmt, dtype, heads, d, block, p, n):
    from _decode_util import Pool, rand16
    print("[store]", fmt, dtype, heads, d, block, flush=True)
    rng = np.random.default_rng(d + block)
    ids, cu = place(rng, [a + b for a, b in zip(p, n)], block, 2000 // block + 8)
    pool = Pool(sc, fmt, dtype, 2, heads, d, block, 2000 // block + 8)
    try:
        shape = (sum(n), heads, d)
        k = rand16(rng, shape, dtype) * np.exp2(np.round(rng.uniform(-6, 6, shape[:2] + (1,))))
        store_and_compare(sc, pool, ids, cu, p, n, k, rand16(rng, shape, dtype), 1)
    finally:
        pool.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_every_value_and_every_tie(sc, fmt, dtype):
    """Rows over all magnitudes of the type, subnormals and the largest ones
    included, rows of halves and quarters of their maximum (ties), zeros and
    rows with a NaN or an infinity."""
    from _decode_util import Pool, round16, to64
    rng = np.random.default_rng(11)
    heads, d, n = 8, 64, 1024
    bits = rng.integers(0, 1 << 16, (n, heads, d)).astype(np.uint16)
    x = to64(bits, dtype)
    top = np.nanmax(np.abs(np.where(np.isfinite(x), x, 0)))
    x = np.where(np.isfinite(x), x, 1.0)
    exp = rng.integers(-20, 8, (n, heads, 1))            # rows of one magnitude and what rounds against it
    mant = np.floor(rng.uniform(128, 256, (n, heads, d))) * 2.0**-8
    near = mant * np.exp2(exp.astype(np.float64)) * np.where(rng.random((n, heads, d)) < 0.5, -1, 1)
    if dtype == "f16":
        near *= 2.0**-2
    near *= np.exp2(-np.floor(rng.uniform(0, 9, (n, heads, d))))
    near = to64(round16(near, dtype), dtype)
    near[..., 1] = near[..., 0] / 2
    near[..., 2] = near[..., 0] / 4
    near = to64(round16(near, dtype), dtype)
    x[::2] = near[::2]
    x[0, 0] = 0.0
    x[0, 1] = -0.0
    x[0, 2, :] = top
    x[0, 3, ::2] = -top
    x[0, 4, 7] = np.nan
    x[0, 5, 63] = np.inf
    x[0, 6, 0] = -np.inf
    x[0, 7] = to64(np.full(d, 1, np.uint16), dtype)      # the smallest subnormal
    pool = Pool(sc, fmt, dtype, 2, heads, d, 16, n // 16)
    try:
        ids, cu = place(rng, [n], 16, n // 16)
        store_and_compare(sc, pool, ids, cu, [0], [n], x, x[::-1].copy(), 0)
    finally:
        pool.close()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,d,block,host", [(8, 128, 16, 0), (2, 64, 16, 12), (3, 128, 5, 0), (1, 64, 256, 2)])
def test_fetched_values(sc, fmt, dtype, heads, d, block, host):
    """Every code with many scales, NaN codes and scales among them: one
    rounding of code * scale, bit for bit; rows of new tokens untouched."""
    import torch
    from _decode_util import TD, Pool, round16, to64
    from _gpu_util import to_u16
    print("[fetch]", fmt, dtype, heads, d, block, host, flush=True)
    rng = np.random.default_rng(block)
    p, n = [3 * block + 1, 0, 1, 2 * block], [2, 3, 0, 1]
    per = sum(-(-(a + b) // block) for a, b in zip(p, n))
    blocks = 2 * per + 3
    pool = Pool(sc, fmt, dtype, 2, heads, d, block, blocks - host, host)
    try:
        ids = rng.permutation(blocks)[:per]
        cu = np.concatenate([[0], np.cumsum([-(-(a + b) // block) for a, b in zip(p, n)])])
        for i in ids:
            for h in (0, 1):
                b = rng.integers(0, 256, pool.half).astype(np.uint8)
                c = block * heads
                s = round16(np.exp2(rng.uniform(-24, 6, c)), "bf16")
                s[rng.random(c) < 0.05] = 0x7fc0
                b[c * d:c * d + 2 * c] = s.view(np.uint8)
                pool._slice(i, 1, h).copy_(torch.from_numpy(b))
        torch.cuda.synchronize()
        t = pool.table(ids, cu, p, n)
        total = sum(p) + sum(n)
        k = torch.full((total + 5, heads, d), 7.0, dtype=TD[dtype], device="cuda")
        v = torch.full_like(k, 7.0)
        sc.sc_fetch_layer_kv(pool.handle, t, 1, sc.active(k.data_ptr(), v.data_ptr(), total + 5), stream())
        torch.cuda.synchronize()
        at = 0
        seven = round16(np.full(1, 7.0), dtype)[0]
        for b, (pp, nn) in enumerate(zip(p, n)):
            want = pool.read(ids[cu[b]:cu[b + 1]], 1, pp)
            for got, w in zip((k, v), want):
                g = to_u16(got[at:at + pp + nn])
                wb = round16(w, dtype)
                nan = np.isnan(w)
                assert np.array_equal(np.isnan(to64(g[:pp], dtype)), nan)
                assert np.array_equal(g[:pp][~nan], wb[~nan])
                assert np.all(g[pp:] == seven)
            at += pp + nn
        assert torch.all(k[total:] == 7.0)
    finally:
        pool.close()


@pytest.mark.parametrize("mode", ["overlap", "serial", "chunked", "events", "host"])
@pytest.mark.parametrize("fmt,dtype,d", [("int8", "bf16", 128), ("e4m3", "f16", 64), ("e4m3", "bf16", 128)])
def test_stack(sc, mode, fmt, dtype, d):
    """Whole stacks over 8-bit blocks: attention over the prefix as the pool
    holds it and the new turn as given; the turn stored as the oracle's
    bytes; then the next turn's fetch returns them."""
    import torch
    from _decode_util import TD, Pool, device16, host64, rand16, round16, to64
    from _gpu_util import compare_attention, to_u16
    print("[stack]", mode, fmt, dtype, d, flush=True)
    rng = np.random.default_rng(17)
    layers, hq, heads, block = 4, 8, 2, 16
    p, n = [333, 0, 64], [45, 17, 1]
    per = [-(-(a + b) // block) for a, b in zip(p, n)]
    blocks = sum(per) + 9
    host = 12 if mode == "host" else 0
    pool = Pool(sc, fmt, dtype, layers, heads, d, block, blocks - host, host)
    try:
        ids = rng.permutation(blocks)[:sum(per)]
        cu = np.concatenate([[0], np.cumsum(per)])
        kept = [[pool.write(ids[cu[b]:cu[b + 1]][:-(-p[b] // block)], l, rand16(rng, (p[b], heads, d), dtype),
                            rand16(rng, (p[b], heads, d), dtype)) for b in range(3)] for l in range(layers)]
        t = pool.table(ids, cu, p, n)
        total, new = sum(p) + sum(n), sum(n)
        q = [rand16(rng, (new, hq, d), dtype) for _ in range(layers)]
        kn = [rand16(rng, (new, heads, d), dtype) for _ in range(layers)]
        vn = [rand16(rng, (new, heads, d), dtype) for _ in range(layers)]
        dev = [[device16(x, dtype) for x in xs] for xs in (q, kn, vn)]
        out = [torch.full((new, hq, d), float("nan"), dtype=TD[dtype], device="cuda") for _ in range(layers)]
        slots = [[torch.full((total, heads, d), float("nan"), dtype=TD[dtype], device="cuda") for _ in range(2)]
                 for _ in range(2)]
        active = [sc.active(a.data_ptr(), b.data_ptr(), total) for a, b in slots]
        ptrs = [[x.data_ptr() for x in xs] for xs in dev + [out]]
        copy = torch.cuda.Stream()
        flags = {"serial": sc.SC_STACK_SERIAL, "events": sc.SC_STACK_EVENT_WAIT}.get(mode, sc.SC_STACK_OVERLAP)
        torch.cuda.synchronize()
        if mode == "chunked":
            sc.sc_prefill_stack_chunked(pool.handle, t, *ptrs, active, hq, 16, flags | sc.SC_STACK_DEBUG_POISON,
                                        compute_stream=stream(), copy_stream=copy.cuda_stream)
        else:
            sc.sc_prefill_stack(pool.handle, t, *ptrs, active, hq, flags, compute_stream=stream(),
                                copy_stream=copy.cuda_stream)
        torch.cuda.synchronize()
        assert not sc.sc_table_stack_status(t)
        nxt = pool.table(ids, cu, [a + b for a, b in zip(p, n)], [0, 0, 0])
        for l in range(layers):
            at = new_at = 0
            ks, vs = [], []
            for b in range(3):
                rows = slice(new_at, new_at + n[b])
                for xs, held, fresh in ((ks, kept[l][b][0], kn[l][rows]), (vs, kept[l][b][1], vn[l][rows])):
                    xs += [to64(round16(held, dtype), dtype), fresh]
                new_at += n[b]
            ref, _ = oa.attention(q[l], np.concatenate(ks), np.concatenate(vs), p, n)
            compare_attention(to_u16(out[l]), ref, f"layer {l}", dtype)
            k, v = slots[0]
            sc.sc_fetch_layer_kv(pool.handle, nxt, l, active[0], stream())
            torch.cuda.synchronize()
            new_at = 0
            for b in range(3):
                for got, held, fresh in ((k, kept[l][b][0], kn[l]), (v, kept[l][b][1], vn[l])):
                    codes, s = od.quantise(fresh[new_at:new_at + n[b]], fmt, dtype)
                    want = np.concatenate([held, od.dequantise(codes, s, fmt)])
                    assert np.array_equal(round16(host64(got[at:at + p[b] + n[b]]), dtype), round16(want, dtype))
                at, new_at = at + p[b] + n[b], new_at + n[b]
    finally:
        pool.close()


def test_slot_timeouts_still_show_over_byte_sized_blocks(sc):
    """The forced time-outs of both slot waits: NaN rows, and the status says so."""
    import torch
    from _decode_util import Pool, device16, rand16
    rng = np.random.default_rng(2)
    pool = Pool(sc, "int8", "bf16", 4, 2, 64, 16, 8)
    try:
        pool_ids = list(range(5))
        for l in range(4):
            pool.write(pool_ids[:4], l, rand16(rng, (64, 2, 64), "bf16"), rand16(rng, (64, 2, 64), "bf16"))
        t = pool.table(pool_ids, [0, 5], [64], [9])
        q = [device16(rand16(rng, (9, 4, 64), "bf16"), "bf16") for _ in range(4)]
        kn = [device16(rand16(rng, (9, 2, 64), "bf16"), "bf16") for _ in range(4)]
        slots = [[torch.zeros((73, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
        active = [sc.active(a.data_ptr(), b.data_ptr(), 73) for a, b in slots]
        copy = torch.cuda.Stream()
        for flag in (sc.SC_STACK_TEST_NEVER_READY, sc.SC_STACK_TEST_NEVER_FREE):
            out = [torch.zeros_like(x) for x in q]
            ptrs = [[x.data_ptr() for x in xs] for xs in (q, kn, kn, out)]
            sc.sc_prefill_stack(pool.handle, t, *ptrs, active, 4, flag, compute_stream=stream(),
                                copy_stream=copy.cuda_stream)
            torch.cuda.synchronize()
            assert sc.sc_table_stack_status(t, clear=True)
            assert torch.isnan(out[3]).all()
    finally:
        pool.close()


def test_library_owned_tier_and_refused_copies(sc):
    """A chunk-mapped tier of 8-bit blocks keeps its blocks over a resize; the copy engines' fetch refuses."""
    import torch
    from _decode_util import device16, host64, rand16, round16
    rng = np.random.default_rng(4)
    pool = sc.sc_pool_create_quant(sc.SC_KV_E4M3, 3, 2, 64, 16, 40)
    t = sc.sc_table_create(pool, [1, 7], [0, 2], [0], [20], stream())
    nxt = sc.sc_table_create(pool, [1, 7], [0, 2], [20], [0], stream())
    x = rand16(rng, (20, 2, 64), "bf16")
    xd = device16(x, "bf16")
    k, v = (torch.zeros((20, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    sc.sc_store_layer_kv(pool, t, 2, xd.data_ptr(), xd.data_ptr(), stream())
    torch.cuda.synchronize()
    sc.sc_pool_resize(pool, 8)
    sc.sc_pool_resize(pool, 40)
    act = sc.active(k.data_ptr(), v.data_ptr(), 20)
    sc.sc_fetch_layer_kv(pool, nxt, 2, act, stream())
    torch.cuda.synchronize()
    codes, s = od.quantise(x, "e4m3", "bf16")
    want = round16(od.dequantise(codes, s, "e4m3"), "bf16")
    assert np.array_equal(round16(host64(k), "bf16"), want) and np.array_equal(round16(host64(v), "bf16"), want)
    with pytest.raises(sc.SwiftCacheError) as e:
        sc.sc_fetch_layer_kv_dma(pool, nxt, 2, act, False, stream())
    assert e.value.status == sc.SC_ERR_UNSUPPORTED
    sc.sc_table_destroy(t)
    sc.sc_table_destroy(nxt)
    sc.sc_pool_destroy(pool)
