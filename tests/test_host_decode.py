"""Host side of 8-bit pools, rotary positions and decode steps, on the CPU:
layouts, argument validation, workspaces.  Every refused call here fails
before any device work."""

import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # never dereferenced


@pytest.fixture(scope="module")
def sc():
    from paper_2606_16135_amd import swiftcache
    swiftcache.load()
    return swiftcache


@pytest.fixture()
def pool(sc):
    made = []

    def make(fmt=0, layers=2, heads=8, d=128, bs=16, blocks=8, **kw):
        p = sc.sc_pool_create_quant(fmt, layers, heads, d, bs, blocks, 0, 0, FAKE, 0, **kw)
        made.append(p)
        return p
    yield make
    for p in made:
        sc.sc_pool_destroy(p)


def refused(sc, status, call, *args, text="", **kw):
    with pytest.raises(sc.SwiftCacheError) as e:
        call(*args, **kw)
    assert e.value.status == getattr(sc, "SC_ERR_" + status), e.value
    assert text in str(e.value)


@pytest.mark.parametrize("bs,heads,d", [(16, 8, 128), (1, 1, 64), (7, 3, 64), (256, 2, 128)])
def test_layout_of_byte_sized_blocks(sc, pool, bs, heads, d):
    p = pool(sc.SC_KV_INT8, bs=bs, heads=heads, d=d)
    fmt, half, off = sc.sc_pool_quant_get(p)
    lay = sc.sc_pool_layout_get(p)
    assert fmt == sc.SC_KV_INT8 and off == bs * heads * d and half % 16 == 0
    assert off + 2 * bs * heads <= half < off + 2 * bs * heads + 16
    assert lay.slice_bytes == 2 * half and lay.block_bytes == 2 * lay.slice_bytes and lay.row_bytes == heads * d
    assert lay.dtype == sc.SC_DTYPE_BF16
    p = pool(sc.SC_KV_16BIT, bs=bs, heads=heads, d=d)
    assert sc.sc_pool_quant_get(p) == (0, bs * heads * d * 2, bs * heads * d * 2)


def test_quantised_pool_refusals(sc, pool):
    refused(sc, "INVALID", sc.sc_pool_create_quant, 3, 2, 8, 128, 16, 8, 0, 0, FAKE)
    refused(sc, "INVALID", sc.sc_pool_create_quant, -1, 2, 8, 128, 16, 8, 0, 0, FAKE)
    refused(sc, "UNSUPPORTED", sc.sc_pool_create_quant, 1, 2, 8, 96, 16, 8, 0, 0, FAKE)
    for fmt in (1, 2):
        refused(sc, "UNSUPPORTED", sc.sc_pool_create_quant, fmt, 2, 8, 128, 16, 8, 0, 0, FAKE, 0, 4, FAKE,
                text="regular cache")
    refused(sc, "INVALID", sc.sc_pool_quant_get, None)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), "UNSUPPORTED"), (dict(rotary_dim=8), "UNSUPPORTED"), (dict(rotary_dim=40), "UNSUPPORTED"),
    (dict(rotary_dim=144), "UNSUPPORTED"), (dict(rotary_dim=0), "UNSUPPORTED"), (dict(layout=2), "INVALID"),
    (dict(scaling=4), "INVALID"), (dict(scaling=-1), "INVALID"), (dict(base=1.0), "INVALID"),
    (dict(base=float("nan")), "INVALID"), (dict(base=float("inf")), "INVALID"),
    (dict(scaling=1, factor=0.0), "INVALID"), (dict(scaling=1, factor=float("inf")), "INVALID"),
    (dict(scaling=2, factor=2.0, low=1.0, high=4.0), "INVALID"),
    (dict(scaling=2, factor=2.0, original_len=100.0, low=4.0, high=4.0), "INVALID"),
    (dict(scaling=3, factor=2.0, original_len=100.0, low=0.0, high=4.0), "INVALID"),
    (dict(scaling=3, factor=2.0, original_len=float("nan"), low=1.0, high=4.0), "INVALID"),
    (dict(amplitude=-1.0), "INVALID"), (dict(amplitude=float("nan")), "INVALID"),
])
def test_rope_refusals(sc, kw, status):
    args = dict(head_dim=128, rotary_dim=128)
    args.update(kw)
    refused(sc, status, sc.sc_rope_create, **args)


def test_calls_without_objects(sc):
    refused(sc, "INVALID", sc.sc_rope_frequencies, None)
    refused(sc, "INVALID", sc.sc_rope_apply, 0, 0, 1, FAKE, FAKE, 128, 1, FAKE, 128, 0, 0, 0, 0, 0)
    b = sc.decode_batch(1, 1, 4, 10, FAKE, FAKE)
    refused(sc, "INVALID", sc.sc_decode_store, None, 0, b, FAKE, FAKE)
    refused(sc, "INVALID", sc.sc_decode_workspace, None, b, 8)
    refused(sc, "INVALID", sc.sc_decode_attn, None, 0, b, FAKE, 8, FAKE)
    sc.sc_rope_destroy(None)


BATCHES = [
    (dict(batch=0), "INVALID"), (dict(batch=-1), "INVALID"), (dict(n_new=0), "INVALID"), (dict(n_new=17), "INVALID"),
    (dict(max_blocks=-1), "INVALID"), (dict(max_len=-1), "INVALID"), (dict(shared_len=-1), "INVALID"),
    (dict(batch=65537), "RANGE"), (dict(max_len=2**31 - 257), "RANGE"),
    (dict(max_len=2**31 - 2**18), "RANGE"), (dict(max_len=1, shared_len=2**31 - 2**18 - 1), "RANGE"),
    (dict(max_len=2**30, shared_len=2**30), "RANGE"),
]
POINTERS = [dict(kv_len=0), dict(block_ids=0), dict(shared_len=5, shared_ids=0), dict(kv_len=FAKE + 2),
            dict(block_ids=FAKE + 1), dict(shared_len=5, shared_ids=FAKE + 2)]


def batch_of(sc, **kw):
    a = dict(batch=2, n_new=1, max_blocks=4, max_len=60, block_ids=FAKE, kv_len=FAKE, shared_ids=0, shared_len=0)
    a.update(kw)
    return sc.decode_batch(**a)


@pytest.mark.parametrize("kw,status", BATCHES)
def test_decode_batch_refusals(sc, pool, kw, status):
    p, b = pool(), batch_of(sc, **kw)
    refused(sc, status, sc.sc_decode_workspace, p, b, 32)
    refused(sc, status, sc.sc_decode_store, p, 0, b, FAKE, FAKE)
    refused(sc, status, sc.sc_decode_attn, p, 0, b, FAKE, 32, FAKE, FAKE, 1 << 40)


@pytest.mark.parametrize("kw", POINTERS)
def test_decode_index_array_refusals(sc, pool, kw):
    p, b = pool(), batch_of(sc, **kw)
    refused(sc, "INVALID", sc.sc_decode_store, p, 0, b, FAKE, FAKE)
    refused(sc, "INVALID", sc.sc_decode_attn, p, 0, b, FAKE, 32, FAKE, FAKE, 1 << 40)
    sc.sc_decode_workspace(p, b, 32)          # the pointers are not looked at


def test_decode_argument_refusals(sc, pool):
    p, b = pool(), batch_of(sc, max_len=2000, max_blocks=200)
    need = sc.sc_decode_workspace(p, b, 32)
    assert need > 0
    attn = sc.sc_decode_attn
    for layer in (-1, 2):
        refused(sc, "RANGE", attn, p, layer, b, FAKE, 32, FAKE, FAKE, need)
        refused(sc, "RANGE", sc.sc_decode_store, p, layer, b, FAKE, FAKE)
    refused(sc, "INVALID", attn, p, 0, b, FAKE, 12, FAKE, FAKE, need)          # not a multiple of the KV heads
    refused(sc, "INVALID", attn, p, 0, b, FAKE, 0, FAKE, FAKE, need)
    refused(sc, "UNSUPPORTED", attn, p, 0, b, FAKE, 136, FAKE, FAKE, 1 << 40)  # group 17
    for q, out, lse, ws, n in [(0, FAKE, 0, FAKE, need), (FAKE, 0, 0, FAKE, need), (FAKE + 8, FAKE, 0, FAKE, need),
                               (FAKE, FAKE + 2, 0, FAKE, need), (FAKE, FAKE, FAKE + 2, FAKE, need),
                               (FAKE, FAKE, 0, 0, need), (FAKE, FAKE, 0, FAKE + 16, need),
                               (FAKE, FAKE, 0, FAKE, need - 1)]:
        refused(sc, "INVALID", attn, p, 0, b, q, 32, out, ws, n, lse)
    store = sc.sc_decode_store
    refused(sc, "INVALID", store, p, 0, b, 0, FAKE)
    refused(sc, "INVALID", store, p, 0, b, FAKE, 0)
    refused(sc, "INVALID", store, p, 0, b, FAKE + 8, FAKE)
    refused(sc, "INVALID", store, p, 0, b, FAKE, FAKE, 0, FAKE, 32, FAKE, text="rotary")   # q, nothing to turn it by
    refused(sc, "RANGE", attn, p, 0, batch_of(sc, batch=1 << 16, max_len=1 << 30), FAKE, 32, FAKE, FAKE, 1 << 60)
    wide = pool(heads=1 << 12)
    refused(sc, "RANGE", attn, wide, 0, batch_of(sc, batch=1 << 16, n_new=16), FAKE, 1 << 12, FAKE, FAKE, 1 << 62)


def test_workspace_grows_with_the_batch_and_is_nothing_for_one_chunk(sc, pool):
    p = pool()
    assert sc.sc_decode_workspace(p, batch_of(sc, max_len=32), 32) == 0
    assert sc.sc_decode_workspace(p, batch_of(sc, max_len=0, max_blocks=0), 32) == 0
    row = 32 * (128 * 4 + 8)                      # one sequence's partials
    # short sequences, joined within their workgroup
    assert sc.sc_decode_workspace(p, batch_of(sc, max_len=24 * 32), 32) == 0
    # two sequences of up to 25 steps: 50 groups of waves, a partial per group and sequence boundary
    assert sc.sc_decode_workspace(p, batch_of(sc, max_len=24 * 32 + 1), 32) == (50 + 2) * row
    # long ones: what the device holds, 2048 waves over 8 KV heads
    assert sc.sc_decode_workspace(p, batch_of(sc, batch=1, max_len=50000), 32) == (256 + 1) * row
    # with a shared prefix: its chunk's partials of both sequences too
    assert sc.sc_decode_workspace(p, batch_of(sc, max_len=32, shared_len=1), 32) == (2 + 2 + 2) * row
    assert sc.sc_decode_workspace(pool(sc.SC_KV_E4M3), batch_of(sc, max_len=64), 32) == 0     # steps of 64 keys


def test_register_check_covers_the_copy_kernels_of_byte_sized_blocks():
    """As for 16-bit blocks: attention may wait on the device for a slot only
    if every kernel in front of the publication fits beside it."""
    csrc = os.path.join(ROOT, "paper_2606_16135_amd", "csrc")
    src = open(os.path.join(csrc, "kv8_copy.hip")).read()
    kernels = set(re.findall(r"__global__\s+__launch_bounds__\([^)]*\)\s+void\s+(\w+)\(", src))
    assert src.count("__global__") == len(kernels) == 3
    listed = re.search(r"return \{(kv8_\w+)<FMT, DT>, (kv8_\w+)<FMT, DT>, (kv8_\w+)<FMT, DT>\}", src)
    assert kernels == set(listed.groups())
    check = src[src.index("int kv8_copy_vgprs("):]
    check = check[:check.index("\n}")]
    assert set(re.findall(r"\(k\.(\w+)\)", check)) == {"fetch", "store", "layer"}
