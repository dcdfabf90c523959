"""Decode steps over a pool in place: attention, the shared prefix and the
fused write of the step's tokens, against the 64-bit oracle."""

import numpy as np
import pytest

from oracle import decode as od

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sc():
    from _gpu_util import require_gpu
    return require_gpu()


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


class Step:
    """A batch over a pool: own lists, a shared list, and its device arrays."""

    def __init__(self, sc, rng, pool, lens, n_new, shared=0, max_len=None, extra=0, ids=None):
        import torch
        self.sc, self.pool, self.lens, self.n_new, self.shared = sc, pool, list(lens), n_new, shared
        block = pool.block
        per = [max(0, -(-x // block)) for x in lens]
        n_sh = -(-shared // block)
        total = pool.blocks + pool.host_blocks + pool.rc_blocks
        place = rng.permutation(total)[:sum(per) + n_sh] if ids is None else np.asarray(ids)
        self.shared_ids = place[:n_sh]
        self.width = max(per + [1]) + extra
        self.table = np.full((len(lens), self.width), -1, dtype=np.int32)
        at = n_sh
        self.ids = []
        for b, m in enumerate(per):
            self.table[b, :m] = place[at:at + m]
            self.ids.append(place[at:at + m])
            at += m
        self.d_table = torch.tensor(self.table, device="cuda")
        self.d_len = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.d_shared = torch.tensor(np.asarray(self.shared_ids, dtype=np.int32), device="cuda")
        self.max_len = max([0] + self.lens) if max_len is None else max_len
        self.batch = sc.decode_batch(len(lens), n_new, self.width, self.max_len, self.d_table.data_ptr(),
                                     self.d_len.data_ptr(), self.d_shared.data_ptr() if shared else 0, shared)

    def fill(self, rng, layer, scale=1.0):
        """Random rows in every list; keeps what the pool then holds."""
        p = self.pool

        def rows(n):
            from _decode_util import rand16
            return rand16(rng, (n, p.heads, p.d), p.dtype, scale)
        self.sh = p.write(self.shared_ids, layer, rows(self.shared), rows(self.shared))
        self.given = [(rows(max(0, t)), rows(max(0, t))) for t in self.lens]
        self.own = [p.write(i, layer, *kv) for i, kv in zip(self.ids, self.given)]

    def attend(self, layer, q, hq, scale=0.0, lse=True, guard=True):
        """sc_decode_attn on its own buffers; returns out (float64) and lse."""
        import torch
        from _decode_util import TD, device16, host64
        sc, p = self.sc, self.pool
        rows = len(self.lens) * self.n_new
        qd = device16(q, p.dtype) if isinstance(q, np.ndarray) else q
        out = torch.full((rows + 1, hq, p.d), 77.0, dtype=TD[p.dtype], device="cuda")
        l = torch.full((hq * rows + 3,), 77.0, dtype=torch.float32, device="cuda")
        n = sc.sc_decode_workspace(p.handle, self.batch, hq)
        ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device="cuda")    # NaN: nothing unwritten may be used
        torch.cuda.synchronize()
        sc.sc_decode_attn(p.handle, layer, self.batch, qd.data_ptr(), hq, out.data_ptr(), ws.data_ptr(), n,
                          l.data_ptr() if lse else 0, scale, stream())
        torch.cuda.synchronize()
        assert torch.all(out[rows] == 77.0) and torch.all(l[hq * rows:] == 77.0) and torch.all(ws[n:] == 0xFF)
        if not lse:
            assert torch.all(l == 77.0)
        return host64(out[:rows]), l[:hq * rows].double().cpu().numpy().reshape(hq, rows)

    def check(self, q, hq, out, lse, scale=None, skip=()):
        from _decode_util import attention_bound, lse_bound
        p, n = self.pool, self.n_new
        for b, t in enumerate(self.lens):
            if b in skip:
                continue
            rows = slice(b * n, (b + 1) * n)
            if t < 0:
                assert not out[rows].any() and np.all(lse[:, rows] == -np.inf)
                continue
            k, v = (np.concatenate([self.sh[i], self.own[b][i]]) for i in (0, 1))
            limits = [self.shared + max(0, t - n + i + 1) for i in range(n)]
            ref, rl, absv, mag = od.attend(q[rows], k, v, limits, scale)
            keys = max(1, self.shared + t)
            bd = attention_bound(ref, absv, mag, p.dtype, p.fmt, keys, np.abs(v).max() if len(v) else 0.0)
            err = np.abs(out[rows] - ref)
            assert np.all(err <= bd), (b, float((err / bd).max()))
            none = np.array(limits) == 0
            assert np.all(lse[:, rows][:, none] == -np.inf) and not out[rows][none].any()
            lb = lse_bound(rl[:, ~none], mag.T[:, ~none], keys)
            le = np.abs(lse[:, rows][:, ~none] - rl[:, ~none])
            assert np.all(le <= lb), (b, float((le / lb).max()))


def test_first_call_of_a_kernel_made_in_a_capture(sc):
    """Steps captured before the process has launched their kernels, over the
    largest LDS use among them; the replays equal the eager call."""
    import torch
    from _decode_util import Pool, device16, rand16
    rng = np.random.default_rng(17)
    pool = Pool(sc, "e4m3", "bf16", 1, 2, 64, 16, 40)
    try:
        st = Step(sc, rng, pool, [5, 30, 1] * 4, 1, 200)
        st.fill(rng, 0)
        q = device16(rand16(rng, (12, 8, 64), "bf16"), "bf16")
        n = sc.sc_decode_workspace(pool.handle, st.batch, 8)
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            sc.sc_decode_attn(pool.handle, 0, st.batch, q.data_ptr(), 8, out.data_ptr(), ws.data_ptr(), n,
                              stream=stream())
        want = None
        for _ in range(3):
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            eager, lse = st.attend(0, q, 8)
            st.check(q.double().cpu().numpy(), 8, eager, lse)
            assert np.array_equal(got.double().cpu().numpy(), eager)
            assert want is None or torch.equal(got, want)
            want = got
    finally:
        pool.close()


@pytest.mark.parametrize("fmt", ["16bit", "e4m3"])
def test_steps_without_own_keys(sc, fmt):
    """max_len and max_blocks of 0: only the shared keys, or none at all."""
    import torch
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(4)
    pool = Pool(sc, fmt, "f16", 1, 2, 64, 16, 8)
    try:
        for shared in (0, 1, 70):
            st = Step(sc, rng, pool, [0, -1, 0, 0, 0], 1, shared)
            st.fill(rng, 0)
            st.batch = sc.decode_batch(5, 1, 0, 0, 0, st.d_len.data_ptr(), st.d_shared.data_ptr() if shared else 0,
                                       shared)
            q = rand16(rng, (5, 8, 64), "f16")
            out, lse = st.attend(0, q, 8)
            st.check(q, 8, out, lse)
            assert torch.isfinite(torch.from_numpy(out)).all()
    finally:
        pool.close()


CASES = [
    # fmt, type, head_dim, q heads, KV heads, block, lengths, new, shared
    ("16bit", "bf16", 128, 8, 2, 16, [1], 1, 0),
    ("16bit", "f16", 64, 4, 4, 16, [1, 2, 63, 64, 65], 1, 0),
    ("16bit", "bf16", 64, 12, 4, 7, [300, 0, 1, -1, 129], 1, 0),
    ("int8", "bf16", 128, 32, 8, 16, [700], 1, 0),
    ("int8", "f16", 64, 7, 1, 1, [50, 257, -1], 1, 0),
    ("e4m3", "bf16", 128, 5, 1, 256, [1000, 513], 1, 0),
    ("e4m3", "f16", 128, 16, 1, 12, [129, 3], 1, 0),
    ("16bit", "bf16", 128, 8, 2, 16, [40, 3, 2, 0, -1, 300], 4, 0),
    ("16bit", "f16", 64, 6, 6, 16, [70, 16, 5], 16, 0),
    ("int8", "bf16", 64, 15, 3, 16, [65, 127, 128], 3, 0),
    ("e4m3", "f16", 128, 32, 2, 32, [1, 900], 2, 0),
    ("16bit", "f16", 128, 32, 2, 16, [257, 64], 16, 0),
    ("16bit", "bf16", 128, 8, 2, 16, [768, 33, 0, -1, 97, 128, 32, 1], 1, 0),
    ("16bit", "f16", 64, 12, 2, 32, [1536, 5, 2, 260], 4, 0),
    ("e4m3", "bf16", 128, 8, 8, 16, [1536, 64, 65, 256, 257], 1, 0),
    ("16bit", "bf16", 128, 8, 8, 16, [5], 1, 100),
    ("int8", "f16", 64, 8, 2, 16, [5, 0, -1, 300], 1, 1),
    ("e4m3", "bf16", 128, 4, 2, 16, [33, 1], 3, 700),
    ("16bit", "bf16", 128, 8, 2, 16, [9, 200, 0, -1, 31] * 3, 1, 515),
    ("16bit", "f16", 64, 16, 2, 7, [9, 200, 0, -1, 31], 2, 129),
    ("int8", "bf16", 128, 20, 4, 16, [3, 70] * 10, 2, 1000),
    ("e4m3", "f16", 64, 10, 2, 64, [64, 65, 1] * 9, 1, 128),
    ("int8", "f16", 128, 16, 1, 16, [100, 7, 0, 16], 16, 385),
    ("e4m3", "bf16", 64, 3, 3, 5, [1, 2, 3] * 30, 3, 260),
]


@pytest.mark.parametrize("fmt,dtype,d,hq,hkv,block,lens,n_new,shared", CASES)
def test_attention(sc, fmt, dtype, d, hq, hkv, block, lens, n_new, shared):
    from _decode_util import Pool, rand16
    print("[decode]", fmt, dtype, d, hq, hkv, block, lens[:6], n_new, shared, flush=True)
    rng = np.random.default_rng(d + block + len(lens) + shared)
    blocks = sum(-(-max(0, x) // block) for x in lens) + -(-shared // block) + 5
    pool = Pool(sc, fmt, dtype, 2, hkv, d, block, blocks)      # bytes 0xff (NaN) wherever no list reaches
    try:
        st = Step(sc, rng, pool, lens, n_new, shared)
        st.fill(rng, 1)
        q = rand16(rng, (len(lens) * n_new, hq, d), dtype, 2.0)
        out, lse = st.attend(1, q, hq)
        st.check(q, hq, out, lse)
        again, _ = st.attend(1, q, hq, lse=False)
        assert np.array_equal(out, again)
        # An upper bound for later replays: other chunks, the same result within the bound.
        wide = Step(sc, rng, pool, lens, n_new, shared, max_len=max(lens) + 20000, extra=20000 // block + 2,
                    ids=list(st.shared_ids) + [i for x in st.ids for i in x])
        wide.sh, wide.own = st.sh, st.own
        out, lse = wide.attend(1, q, hq, scale=0.21)
        wide.check(q, hq, out, lse, scale=np.float64(np.float32(0.21)))
    finally:
        pool.close()


@pytest.mark.parametrize("fmt,dtype", [("16bit", "bf16"), ("int8", "f16"), ("e4m3", "bf16")])
def test_tiers_and_far_blocks(sc, fmt, dtype):
    """Blocks of every tier in one list, and blocks whose offsets pass 32 bits."""
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(8)
    for far in (False, True):
        rc = 6 if fmt == "16bit" and not far else 0
        blocks = 70000 if far else 8
        pool = Pool(sc, fmt, dtype, 2, 8, 128, 16, blocks, 0 if far else 6, rc, fill=None if far else 0xFF)
        try:
            ids = None
            if far:
                assert pool.block_bytes * blocks > 2**32
                ids = [69999, 3, 69990, 65537, 69000, 1, 40000, 69998, 2, 68000, 69997, 69996]
            st = Step(sc, rng, pool, [100, 33], 1, 30, ids=ids)
            st.fill(rng, 1)
            q = rand16(rng, (2, 32, 128), dtype)
            out, lse = st.attend(1, q, 32)
            st.check(q, 32, out, lse)
        finally:
            pool.close()


@pytest.mark.parametrize("fmt,dtype", [("16bit", "bf16"), ("16bit", "f16"), ("int8", "bf16"), ("e4m3", "f16")])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("hq", [4, 2])
def test_hidden_keys_do_not_arrive(sc, fmt, dtype, value, hq):
    """NaN or infinite K/V behind every row's end, and in the step's later
    tokens: the rows that do not see them are exactly what they are without;
    the rows that do see a NaN are NaN."""
    import torch
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(6)
    block, n_new, lens, shared = 16, 4, [37, 4, 130], 21
    pool = Pool(sc, fmt, dtype, 1, 2, 64, block, 40)
    try:
        st = Step(sc, rng, pool, lens, n_new, shared)
        st.fill(rng, 0)
        q = rand16(rng, (12, hq, 64), dtype)
        clean, clean_lse = st.attend(0, q, hq)
        for b, t in enumerate(lens):      # the last two tokens of the step, and what follows in the block
            k, v = (x.copy() for x in st.given[b])
            k[t - 2:], v[t - 2:] = value, value
            pool.write(st.ids[b], 0, k, v)
        out, lse = st.attend(0, q, hq)
        for b in range(3):
            rows = [b * n_new, b * n_new + 1]
            assert np.array_equal(out[rows], clean[rows]) and np.array_equal(lse[:, rows], clean_lse[:, rows])
            if np.isnan(value) or fmt != "16bit":
                assert np.isnan(out[[r + 2 for r in rows]]).all()
    finally:
        pool.close()


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,shared", [([200, 65, 1], 0), ([3, 40], 300), ([3, 40] * 4, 300)])
def test_v_scales_of_any_size_in_fp16(sc, fmt, lens, shared):
    """V rows whose scales differ by up to 2^24 between tokens, and for one
    sequence are all near fp16's smallest number or largest: the probabilities
    times the scale stay within fp16 all the same."""
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(33)
    hq, hkv, d, block = 8, 2, 64, 16
    pool = Pool(sc, fmt, "f16", 1, hkv, d, block, 80)
    try:
        st = Step(sc, rng, pool, lens, 1, shared)
        st.fill(rng, 0)

        def rows(n, lo, hi):
            x = rand16(rng, (n, hkv, d), "f16") * 2.0 ** rng.integers(lo, hi + 1, (n, hkv, 1))
            return np.clip(x, -60000, 60000).astype(np.float16).astype(np.float64)
        for lo, hi in ((-14, 10), (-14, -14), (13, 13)):
            if shared:
                st.sh = pool.write(st.shared_ids, 0, st.sh[0].astype(np.float16).astype(np.float64), rows(shared, lo, hi))
            st.own = [pool.write(i, 0, given[0], rows(len(given[0]), lo, hi)) for i, given in zip(st.ids, st.given)]
            q = rand16(rng, (len(lens), hq, d), "f16", 2.0)
            out, lse = st.attend(0, q, hq)
            st.check(q, hq, out, lse)
    finally:
        pool.close()


@pytest.mark.parametrize("batch", [1, 4, 5, 8, 9, 16, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("fmt,dtype,d,shared", [
    ("16bit", "bf16", 128, 1), ("16bit", "f16", 64, 127), ("int8", "bf16", 64, 129), ("e4m3", "bf16", 128, 600),
    ("int8", "f16", 128, 257),
])
def test_rows_that_share_keys(sc, fmt, dtype, d, shared, batch):
    """4 to 260 rows of a KV head over shared keys that end anywhere in a tile,
    and a bad id in each place of the list: every row NaN, empty slots zero."""
    from _decode_util import Pool, rand16
    print("[shared]", fmt, dtype, d, shared, batch, flush=True)
    rng = np.random.default_rng(batch + shared)
    hq, hkv, block = 8, 2, 16
    lens = [[1, 5, -1, 0][b % 4] for b in range(batch)]
    pool = Pool(sc, fmt, dtype, 1, hkv, d, block, batch + shared // block + 4)
    try:
        st = Step(sc, rng, pool, lens, 1, shared)
        st.fill(rng, 0)
        q = rand16(rng, (batch, hq, d), dtype, 2.0)
        out, lse = st.attend(0, q, hq)
        st.check(q, hq, out, lse)
        real = np.array(lens) >= 0
        for at in sorted({0, len(st.shared_ids) // 2, len(st.shared_ids) - 1}):
            st.d_shared[at] = [-1, 2**31 - 1, pool.blocks][at % 3]
            out, lse = st.attend(0, q, hq)
            assert np.isnan(out[real]).all() and np.isnan(lse[:, real]).all()
            assert not out[~real].any() and np.all(lse[:, ~real] == -np.inf)
            st.d_shared[at] = int(st.shared_ids[at])
        out2, lse2 = st.attend(0, q, hq)
        st.check(q, hq, out2, lse2)
    finally:
        pool.close()


def test_a_row_of_one_key_is_its_value(sc):
    """The most sequences a step may have, each with one key: its V row itself."""
    import torch
    from _decode_util import Pool, device16, host64, rand16
    rng = np.random.default_rng(2)
    n = 65536
    pool = Pool(sc, "16bit", "bf16", 1, 1, 64, 1, 7)
    try:
        v = rand16(rng, (7, 1, 64), "bf16")
        pool.write(range(7), 0, rand16(rng, (7, 1, 64), "bf16"), v)
        ids = (np.arange(n) % 7).astype(np.int32)
        table, lens = torch.from_numpy(ids).cuda(), torch.ones(n, dtype=torch.int32, device="cuda")
        lens[5::11] = -1
        q = device16(rand16(rng, (n, 2, 64), "bf16"), "bf16")
        for top in (1, 1000):                # with and without partials
            wide = table if top == 1 else torch.full((n, top), -1, dtype=torch.int32, device="cuda")
            if top > 1:
                wide[:, 0] = table
            batch = sc.decode_batch(n, 1, top, top, wide.data_ptr(), lens.data_ptr(), 0, 0)
            size = sc.sc_decode_workspace(pool.handle, batch, 2)
            ws = torch.full((size + 1,), 0xFF, dtype=torch.uint8, device="cuda")
            out = torch.full_like(q, 5.0)
            torch.cuda.synchronize()
            sc.sc_decode_attn(pool.handle, 0, batch, q.data_ptr(), 2, out.data_ptr(), ws.data_ptr(), size, 0, 0.0,
                              stream())
            torch.cuda.synchronize()
            want = np.repeat(v[ids], 2, 1)
            want[5::11] = 0
            assert np.array_equal(host64(out), want)
    finally:
        pool.close()


def test_peaky_and_masked_scores(sc):
    """Scores of thousands, keys that all score -infinity but one, and a row
    whose every score is -infinity (no maximum: NaN, as the formula has it)."""
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(12)
    pool = Pool(sc, "16bit", "bf16", 1, 1, 64, 16, 40)
    try:
        st = Step(sc, rng, pool, [300, 129], 1)
        st.fill(rng, 0)
        q = rand16(rng, (2, 4, 64), "bf16", 300.0)
        out, lse = st.attend(0, q, 4)
        st.check(q, 4, out, lse)
        k = np.full((300, 1, 64), -np.inf)
        k[200] = 1.0
        pool.write(st.ids[0], 0, k, st.own[0][1])
        q = np.ones((2, 4, 64))
        out, lse = st.attend(0, q, 4)
        assert np.array_equal(out[0], np.repeat(st.own[0][1][200], 4, 0)) and np.allclose(lse[:, 0], 8.0)
        k[200] = -np.inf
        pool.write(st.ids[0], 0, k, st.own[0][1])
        out, lse = st.attend(0, q, 4)
        assert np.isnan(out[0]).all() and np.isfinite(out[1]).all()
    finally:
        pool.close()


@pytest.mark.parametrize("shared", [0, 40, 400])
@pytest.mark.parametrize("fmt", ["16bit", "int8"])
def test_bad_lists_give_nan_rows_and_touch_nothing(sc, fmt, shared):
    """Ids outside the pool, HBM ids that are not lent, lengths beyond the
    bounds: that sequence's rows are NaN and only they; a bad shared id: all
    rows.  The kernels check every id and length before any address is
    formed from them."""
    import torch
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(3)
    pool = Pool(sc, fmt, "bf16", 1, 2, 64, 16, 80)
    try:
        lens = [100, 50, 200, 30, 64, -1]
        st = Step(sc, rng, pool, lens, 1, shared, ids=rng.permutation(60))
        st.fill(rng, 0)
        q = rand16(rng, (6, 8, 64), "bf16")
        good, _ = st.attend(0, q, 8)
        st.d_table[0, 6] = 80
        st.d_table[2, 0] = -5
        st.d_len[3] = 10**6
        st.d_len[4] = st.max_len + 1
        out, lse = st.attend(0, q, 8)
        for b in (0, 2, 3, 4):
            assert np.isnan(out[b]).all() and np.isnan(lse[:, b]).all(), b
        for b in (1, 5):
            assert np.array_equal(out[b], good[b])
        kv = torch.ones((6, 2, 64), dtype=torch.bfloat16, device="cuda")
        before = pool.dev.clone()
        st.d_len[:] = torch.tensor([100, -1, 5, 10**6, st.max_len + 1, -1], dtype=torch.int32, device="cuda")
        st.d_table[2, 0] = 2**30
        sc.sc_decode_store(pool.handle, 0, st.batch, kv.data_ptr(), kv.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(before, pool.dev)
        # HBM blocks beyond what the pool lends
        sc.sc_pool_resize(pool.handle, 60)
        st.d_table[0, 0] = 60
        st.d_len[:] = torch.tensor([10, 50, -1, -1, -1, -1], dtype=torch.int32, device="cuda")
        out, _ = st.attend(0, q, 8)
        assert np.isnan(out[0]).all() and np.array_equal(out[1], good[1])
        if shared:
            st.d_table[0, 0] = int(st.ids[0][0])
            st.d_shared[shared // 16 // 2] = 2**31 - 1
            out, _ = st.attend(0, q, 8)
            assert np.isnan(out[:2]).all() and not out[2:].any()
    finally:
        pool.close()


def test_bad_lists_of_long_steps(sc):
    """As above, with a bound on the lengths that makes partials of own keys."""
    from _decode_util import Pool, rand16
    rng = np.random.default_rng(5)
    pool = Pool(sc, "16bit", "f16", 1, 2, 64, 16, 200)
    try:
        lens = [900, 50, 1200, 30, -1, 64]
        st = Step(sc, rng, pool, lens, 1, 0, max_len=2000, extra=60, ids=rng.permutation(150))
        st.fill(rng, 0)
        q = rand16(rng, (6, 8, 64), "f16")
        good, lse = st.attend(0, q, 8)
        st.check(q, 8, good, lse)
        st.d_table[0, 56] = 200               # the last block of a long list, the middle of another
        st.d_table[2, 40] = -1
        st.d_len[5] = 2001
        out, lse = st.attend(0, q, 8)
        for b in (0, 2, 5):
            assert np.isnan(out[b]).all() and np.isnan(lse[:, b]).all(), b
        st.d_len[5] = 64
        out, lse = st.attend(0, q, 8)
        for b in (1, 3, 4, 5):
            assert np.array_equal(out[b], good[b]), b
        assert np.isnan(out[[0, 2]]).all()
    finally:
        pool.close()


@pytest.mark.parametrize("fmt,dtype,d,rot,layout", [
    ("16bit", "bf16", 128, 128, "half"), ("16bit", "f16", 64, 32, "interleaved"), ("int8", "bf16", 128, 64, "half"),
    ("int8", "f16", 64, 64, "interleaved"), ("e4m3", "bf16", 64, 16, "half"), ("e4m3", "f16", 128, 128, "interleaved"),
])
@pytest.mark.parametrize("in_place", [False, True])
def test_store_is_rotation_then_store(sc, fmt, dtype, d, rot, layout, in_place):
    """The fused write equals sc_rope_apply followed by a plain write, bit for
    bit, in k, in q and in every byte of the pool; empty slots' q rows and
    tokens before 0 are left alone."""
    import torch
    from _decode_util import Pool, device16, rand16
    print("[store]", fmt, dtype, d, rot, layout, in_place, flush=True)
    rng = np.random.default_rng(rot)
    lens, n_new, hq, hkv, shared = [20, 3, -1, 64, 1], 3, 10, 5, 37
    rows = len(lens) * n_new
    rope = sc.sc_rope_create(d, rot, sc.ROPE_LAYOUTS[layout], base=10000.0)
    pool = Pool(sc, fmt, dtype, 2, hkv, d, 7, 40)
    try:
        st = Step(sc, rng, pool, lens, n_new, shared)
        q, k, v = (device16(rand16(rng, (rows, h, d), dtype), dtype) for h in (hq, hkv, hkv))
        pos = torch.tensor([shared + t - n_new + i for t in lens for i in range(n_new)], dtype=torch.int32,
                           device="cuda")
        qr, kr = torch.empty_like(q), torch.empty_like(k)
        sc.sc_rope_apply(rope, sc.DTYPE_CODES[dtype], rows, pos.data_ptr(), q.data_ptr(), hq * d, hq, qr.data_ptr(),
                         hq * d, k.data_ptr(), hkv * d, hkv, kr.data_ptr(), hkv * d, stream())
        fresh = pool.dev.clone()
        sc.sc_decode_store(pool.handle, 1, st.batch, kr.data_ptr(), v.data_ptr(), stream=stream())
        torch.cuda.synchronize()
        want = pool.dev.clone()
        pool.dev.copy_(fresh)
        qo = q.clone() if in_place else torch.full_like(q, 9.0)
        src = qo if in_place else q
        left = qo[6:9].clone()
        sc.sc_decode_store(pool.handle, 1, st.batch, k.data_ptr(), v.data_ptr(), rope, src.data_ptr(), hq,
                           qo.data_ptr(), stream())
        torch.cuda.synchronize()
        assert torch.equal(pool.dev, want) and not torch.equal(pool.dev, fresh)
        qr[6:9] = left
        assert torch.equal(qo.view(torch.int16), qr.view(torch.int16))
        # What was written is the oracle's, and nothing else changed.
        held = st.pool.dev.cpu().numpy()
        from _decode_util import host64
        k64, v64 = host64(kr), host64(v)
        for b, t in enumerate(lens):
            for i in range(n_new):
                at = t - n_new + i
                if t < 0 or at < 0:
                    continue
                blk, r = divmod(at, 7)
                for h, x in ((0, k64), (1, v64)):
                    row = pool.unpack(pool.bytes_of(int(st.ids[b][blk]), 1, h))[r]
                    ref = x[b * n_new + i]
                    if fmt != "16bit":
                        codes, s = od.quantise(ref, fmt, dtype)
                        ref = od.dequantise(codes, s, fmt)
                    assert np.array_equal(row, ref)
        changed = (held != fresh.cpu().numpy()).sum()
        n_rows = sum(min(n_new, max(0, t)) for t in lens)
        assert changed <= n_rows * 2 * hkv * (d * (2 if fmt == "16bit" else 1) + 2)
        # k alone, and no rotation at all
        pool.dev.copy_(fresh)
        sc.sc_decode_store(pool.handle, 1, st.batch, k.data_ptr(), v.data_ptr(), rope, stream=stream())
        torch.cuda.synchronize()
        assert torch.equal(pool.dev, want)
    finally:
        pool.close()
        sc.sc_rope_destroy(rope)


@pytest.mark.parametrize("fmt,dtype,shared", [("16bit", "bf16", 0), ("int8", "bf16", 70), ("e4m3", "f16", 300)])
def test_generation_replayed_from_one_graph(sc, fmt, dtype, shared):
    """A step of two layers (write with rotary positions, attend) captured once
    and replayed while lengths grow and blocks are added on the device; every
    replay against the same calls made eagerly into a second pool, bit for
    bit, and the last against the oracle; then the ordinary layer fetch reads
    what the steps wrote."""
    import torch
    from _decode_util import Pool, device16, host64, rand16, round16
    rng = np.random.default_rng(21)
    layers, hq, hkv, d, block, steps = 2, 8, 2, 64, 4, 7
    start = [5, 1, -1, 30]
    final = [t + steps if t >= 0 else -1 for t in start]
    rope = sc.sc_rope_create(d, d)
    theta = od.frequencies(d, 10000.0)
    pools = [Pool(sc, fmt, dtype, layers, hkv, d, block, 120) for _ in range(2)]
    try:
        seed = rng.integers(1 << 30)
        sts = [Step(sc, np.random.default_rng(seed), p, final, 1, shared) for p in pools]
        for l in range(layers):
            for s in sts:
                s.fill(np.random.default_rng(100 + l), l)
        n = sc.sc_decode_workspace(pools[0].handle, sts[0].batch, hq)
        bufs = []
        for _ in range(2):
            bufs.append(dict(
                q=torch.zeros((layers, 4, hq, d), dtype=device16(np.zeros(1), dtype).dtype, device="cuda"),
                ws=torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device="cuda")))
            b = bufs[-1]
            b["qo"], b["out"] = torch.zeros_like(b["q"]), torch.zeros_like(b["q"])
            b["k"], b["v"] = (torch.zeros((layers, 4, hkv, d), dtype=b["q"].dtype, device="cuda") for _ in range(2))
            b["lse"] = torch.zeros((layers, hq, 4), dtype=torch.float32, device="cuda")

        def step(i, s):
            b, st = bufs[i], sts[i]
            for l in range(layers):
                sc.sc_decode_store(pools[i].handle, l, st.batch, b["k"][l].data_ptr(), b["v"][l].data_ptr(), rope,
                                   b["q"][l].data_ptr(), hq, b["qo"][l].data_ptr(), s)
                sc.sc_decode_attn(pools[i].handle, l, st.batch, b["qo"][l].data_ptr(), hq, b["out"][l].data_ptr(),
                                  b["ws"].data_ptr(), n, b["lse"][l].data_ptr(), 0.0, s)

        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(0, torch.cuda.current_stream().cuda_stream)
        rows = []
        for t in range(steps):
            x = [rand16(rng, (layers, 4, h, d), dtype) for h in (hq, hkv, hkv)]
            rows.append(x)
            lens = torch.tensor([a + t + 1 if a >= 0 else -1 for a in start], dtype=torch.int32, device="cuda")
            for b, st in zip(bufs, sts):
                for name, y in zip("qkv", x):
                    b[name].copy_(device16(y, dtype))
                st.d_len.copy_(lens)
            torch.cuda.synchronize()
            graph.replay()
            step(1, stream())
            torch.cuda.synchronize()
            for name in ("out", "lse", "qo"):
                assert torch.equal(bufs[0][name].view(torch.int16), bufs[1][name].view(torch.int16)), (t, name)
            assert torch.equal(pools[0].dev, pools[1].dev)
        st, p = sts[0], pools[0]
        for l in range(layers):
            st.sh = p.read(st.shared_ids, l, shared)
            st.own = [p.read(i, l, max(0, t)) for i, t in zip(st.ids, final)]
            st.check(host64(bufs[0]["qo"][l]), hq, host64(bufs[0]["out"][l]), bufs[0]["lse"][l].double().cpu().numpy())
            for b, a in enumerate(start):         # the rows the steps wrote
                if a < 0:
                    continue
                for t in range(steps):
                    pos = [shared + a + t]
                    k = rows[t][1][l, b:b + 1]
                    ref = od.rotate(k, pos, theta, "half")
                    tol = (2.0**-8 if dtype == "bf16" else 2.0**-11) * np.abs(ref) + 2e-6 * np.abs(k).max()
                    if fmt != "16bit":       # half a code step: half the scale, or 2^-4 of the value and a floor
                        s = od.bf16_up(np.abs(ref).max(-1, keepdims=True) / od.TOP[fmt]) * (1 + 2.0**-6)
                        tol = tol * 1.1 + (0.5 * s if fmt == "int8" else 2.0**-4 * np.abs(ref) * 1.1 + 2.0**-10 * s)
                    assert np.all(np.abs(st.own[b][0][a + t] - ref[0]) <= tol[0])
            ids = [int(i) for x in st.ids for i in x]
            cu = np.concatenate([[0], np.cumsum([len(x) for x in st.ids])])
            have = [max(0, t) for t in final]
            table = p.table(ids, cu, have, [0] * 4)
            k, v = (torch.zeros((sum(have), hkv, d), dtype=bufs[0]["q"].dtype, device="cuda") for _ in range(2))
            sc.sc_fetch_layer_kv(p.handle, table, l, sc.active(k.data_ptr(), v.data_ptr(), sum(have)), stream())
            torch.cuda.synchronize()
            for i, got in enumerate((k, v)):
                want = round16(np.concatenate([x[i] for x in st.own]), dtype)
                assert np.array_equal(round16(host64(got), dtype), want)
    finally:
        for p in pools:
            p.close()
        sc.sc_rope_destroy(rope)


def test_calls_on_two_streams_with_workspaces_of_their_own(sc):
    import torch
    from _decode_util import Pool, device16, host64, rand16
    rng = np.random.default_rng(5)
    pool = Pool(sc, "16bit", "f16", 1, 2, 128, 16, 600)
    try:
        steps = [Step(sc, rng, pool, [1500, 2000], 1), Step(sc, rng, pool, [900, 700, 100], 1, 800)]
        qs, refs = [], []
        for st in steps:
            st.fill(rng, 0)                     # the second may overwrite blocks of the first: read back below
        for st in steps:
            st.sh = pool.read(st.shared_ids, 0, st.shared)
            st.own = [pool.read(i, 0, max(0, t)) for i, t in zip(st.ids, st.lens)]
            qs.append(device16(rand16(rng, (len(st.lens), 8, 128), "f16"), "f16"))
            refs.append(st.attend(0, qs[-1], 8))
        streams = [torch.cuda.Stream() for _ in steps]
        outs = [torch.zeros_like(q) for q in qs]
        ws = [torch.empty(sc.sc_decode_workspace(pool.handle, st.batch, 8), dtype=torch.uint8, device="cuda")
              for st in steps]
        torch.cuda.synchronize()
        for _ in range(10):
            for st, s, q, o, w in zip(steps, streams, qs, outs, ws):
                sc.sc_decode_attn(pool.handle, 0, st.batch, q.data_ptr(), 8, o.data_ptr(), w.data_ptr(), w.numel(),
                                  stream=s.cuda_stream)
        torch.cuda.synchronize()
        for o, (ref, _) in zip(outs, refs):
            assert np.array_equal(host64(o), ref)
        for st, q, (out, lse) in zip(steps, qs, refs):
            st.check(host64(q), 8, out, lse)
    finally:
        pool.close()
