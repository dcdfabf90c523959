"""Helpers for the tests of 8-bit pools, rotary positions and decode steps:
pools as torch tensors filled through the oracle, and error bounds."""

import numpy as np
import torch

from oracle import attention as oa
from oracle import decode as od

TD = {"bf16": torch.bfloat16, "f16": torch.float16}
# Largest relative error of one rounding to the type.
HALF_STEP = {"bf16": 2.0**-8, "f16": 2.0**-11}
TINY = {"bf16": 2.0**-134, "f16": 2.0**-25}    # ... and its absolute floor among the subnormals


def round16(x, dtype):
    """float64 -> 16-bit patterns (uint16), to nearest even."""
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64))
    return t.float().to(TD[dtype]).view(torch.int16).numpy().view(np.uint16)


def to64(bits, dtype):
    return oa.bits_to_f64(bits, dtype)


def rand16(rng, shape, dtype, scale=1.0):
    """N(0, scale^2) values of the type, as float64."""
    return to64(round16(rng.standard_normal(shape) * scale, dtype), dtype)


def device16(x, dtype):
    """float64 values of the type -> device tensor."""
    return torch.from_numpy(np.ascontiguousarray(x)).float().to(TD[dtype]).cuda()


def host64(t):
    return t.detach().double().cpu().numpy()


class Pool:
    """A pool over one caller-owned device tensor (`extra`: more tiers), with
    its bytes as numpy through the documented layout."""

    def __init__(self, sc, fmt, dtype, layers, heads, d, block, blocks, host_blocks=0, rc_blocks=0, fill=0xFF,
                 place_bytes=0):
        self.sc, self.fmt, self.dtype = sc, fmt, dtype
        self.layers, self.heads, self.d, self.block = layers, heads, d, block
        self.blocks, self.host_blocks, self.rc_blocks = blocks, host_blocks, rc_blocks
        row = heads * d * (2 if fmt == "16bit" else 1)
        self.half = block * row if fmt == "16bit" else (block * (row + 2 * heads) + 15) // 16 * 16
        self.block_bytes = layers * 2 * self.half

        def tier(n, pinned=False):
            t = torch.empty(max(1, n) * self.block_bytes, dtype=torch.uint8, device="cpu" if pinned else "cuda",
                            pin_memory=pinned)
            return t.fill_(fill) if fill is not None else t
        self.dev = tier(blocks)
        self.host = tier(host_blocks, True) if host_blocks else None
        self.rc = tier(rc_blocks) if rc_blocks else None
        torch.cuda.synchronize()
        self.handle = sc.sc_pool_create_quant(
            sc.KV_FORMAT_CODES[fmt], layers, heads, d, block, blocks, host_blocks, 0, self.dev.data_ptr(),
            self.host.data_ptr() if host_blocks else 0, rc_blocks, self.rc.data_ptr() if rc_blocks else 0,
            sc.DTYPE_CODES[dtype])
        self.tables = []

    def _slice(self, block_id, layer, is_v):
        t, i = self.dev, block_id
        if i >= self.blocks:
            t, i = self.host, i - self.blocks
            if i >= self.host_blocks:
                t, i = self.rc, i - self.host_blocks
        at = i * self.block_bytes + (2 * layer + is_v) * self.half
        return t[at:at + self.half]

    def bytes_of(self, block_id, layer, is_v):
        return self._slice(block_id, layer, is_v).cpu().numpy()

    def pack(self, x, old):
        """Bytes of a half whose rows 0..len(x) hold x [n][heads][d] (float64 of the type); the rest as in `old`."""
        b = old.copy()
        n = x.shape[0]
        if self.fmt == "16bit":
            b[:n * self.heads * self.d * 2] = round16(x, self.dtype).reshape(-1).view(np.uint8)
            return b
        codes, s = od.quantise(x, self.fmt, self.dtype)
        b[:codes.size] = codes.reshape(-1)
        off = self.block * self.heads * self.d
        b[off:off + 2 * s.size] = scale_bits(s).reshape(-1).view(np.uint8)
        return b

    def unpack(self, b):
        """[block][heads][d] float64 values that a half's bytes stand for."""
        shape = (self.block, self.heads, self.d)
        n = self.block * self.heads
        if self.fmt == "16bit":
            return to64(b[:n * self.d * 2].view(np.uint16), self.dtype).reshape(shape)
        s = to64(np.ascontiguousarray(b[n * self.d:n * self.d + 2 * n]).view(np.uint16), "bf16").reshape(shape[:2])
        return od.dequantise(b[:n * self.d].reshape(shape), s, self.fmt)

    def write(self, ids, layer, k, v):
        """Rows k, v [t][heads][d] into the block list; returns what it then holds of them (float64)."""
        kept = []
        for is_v, x in ((0, k), (1, v)):
            rows = []
            for j, i in enumerate(ids):
                part = x[j * self.block:(j + 1) * self.block]
                if len(part) == 0:
                    continue
                half = self._slice(i, layer, is_v)
                b = self.pack(part, half.cpu().numpy())
                half.copy_(torch.from_numpy(b))
                rows.append(self.unpack(b)[:len(part)])
            kept.append(np.concatenate(rows) if rows else np.zeros((0, self.heads, self.d)))
        torch.cuda.synchronize()
        return kept

    def read(self, ids, layer, tokens):
        out = []
        for is_v in (0, 1):
            rows = [self.unpack(self.bytes_of(i, layer, is_v)) for i in ids]
            out.append(np.concatenate(rows)[:tokens] if rows else np.zeros((0, self.heads, self.d)))
        return out

    def table(self, ids, cu, p, n):
        t = self.sc.sc_table_create(self.handle, ids, cu, p, n, torch.cuda.current_stream().cuda_stream)
        self.tables.append(t)
        return t

    def close(self):
        torch.cuda.synchronize()
        for t in self.tables:
            self.sc.sc_table_destroy(t)
        self.sc.sc_pool_destroy(self.handle)


def scale_bits(s):
    """bf16 patterns of scales that are bf16 values or NaN."""
    bits = round16(np.where(np.isnan(s), 1.0, s), "bf16")
    return np.where(np.isnan(s), np.uint16(0x7fc0), bits).astype(np.uint16)


def attention_bound(ref, absv, mag, dtype, fmt, t, vmax):
    """|out - ref| from: each probability (with 8-bit blocks, times V's scale)
    rounded once to the type (half a step of it, for fp16 also its subnormal
    floor over t keys: 2^-25 of the largest such product, which with V's
    largest code is V's row maximum, up to its scale's rounding),
    the output rounded once, fp32 sums (128 terms deep and t / 16 MFMA
    additions) and exponentials (2 ulp), and each score's own fp32 sum over
    head_dim products of magnitude mag in all, which moves a probability by
    as much in proportion, and their sum."""
    p = HALF_STEP[dtype] * absv + (t * 2.0**-25 * vmax * 1.01 if dtype == "f16" else 0.0)
    fp32 = 2.0**-24 * (512 + t / 4 + 2 * 136 * mag[..., None]) * absv
    return (p + fp32) * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * np.abs(ref) + TINY[dtype]


def lse_bound(lse, mag, t):
    """fp32 scores (each a sum of head_dim products, at most mag in
    magnitude), exponentials, a sum over t keys and a logarithm."""
    return 2.0**-24 * (300 * mag + t / 8 + 64 + 4 * np.abs(np.where(np.isfinite(lse), lse, 0)))
