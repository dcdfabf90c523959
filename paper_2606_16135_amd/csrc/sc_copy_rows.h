// Device pieces of the row copies, shared by kv_copy.hip (16-bit blocks) and
// kv8_copy.hip (8-bit blocks).
#pragma once

#include "sc_internal.h"
#include "sc_quant.h"

namespace sc {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 8;
// Buffer instruction cache-policy bits on gfx950: sc0 = 1, nt = 2, sc1 = 16.
constexpr int kLoadPolicy = 1 | 2 | 16;
constexpr int kStorePolicy = 2;

// A record of 32-bit fields read through the constant address space: the
// host writes the copy items before the launch and nothing writes them
// during it, so a uniform index gives one scalar load, the item stays in
// scalar registers and the buffer resources built from it need no
// per-lane loop.  (Read as ordinary global memory, the fields came back
// one dependent vector load at a time and every buffer access was wrapped
// in a loop over the distinct resources of the wave.)
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ CopyItem load_item(const CopyItem *p) {
  static_assert(sizeof(CopyItem) == sizeof(i32x8), "one 32-byte record");
  const i32x8 v = *(const __attribute__((address_space(4))) i32x8 *)p;
  CopyItem r;
  __builtin_memcpy(&r, &v, sizeof(r));
  return r;
}

// poison: write nan2 over the destination instead of copying (fetch and
// append into a slot whose gate timed out).  kSerialStores: one store in
// flight per wave (see launch_kv_copy).  U: loads in flight.
template <int MODE, bool kSerialStores, int U = kUnroll>
__device__ __forceinline__ void copy_rows(const CopyArgs &a, int g, bool poison = false, uint32_t nan2 = 0) {
  const int item_idx = g >> 1;
  const int is_v = g & 1;
  const CopyItem it = load_item(a.items + item_idx);
  if (MODE != COPY_APPEND && !((a.tier_mask >> it.tier) & 1)) return;
  // One item is at most 256 rows of one KV layer (under 4 MiB), so 32-bit
  // chunk indices and byte offsets cover it.
  const int nchunks = (int)(((int64_t)it.nrows * a.row_bytes) >> 4);
  const int64_t half_off = is_v ? a.v_half_off : 0;
  const char *src;
  char *dst;
  if (MODE == COPY_FETCH) {
    src = a.tier_base[it.tier] + it.pool_off + a.layer_off + half_off;
    dst = (is_v ? a.act_v : a.act_k) + it.act_row * a.row_bytes;
  } else if (MODE == COPY_APPEND) {
    src = (is_v ? a.new_v : a.new_k) + it.src_row * a.row_bytes;
    dst = (is_v ? a.act_v : a.act_k) + it.act_row * a.row_bytes;
  } else {
    src = (is_v ? a.new_v : a.new_k) + it.src_row * a.row_bytes;
    dst = a.tier_base[it.tier] + it.pool_off + a.layer_off + half_off;
  }
  const int bytes = nchunks * 16;
  // Lanes past the item's last chunk are not masked off: the buffer
  // resources end at the item's last byte, so their loads return zeros and
  // their stores are dropped by the hardware's range check.
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(src), (short)0, bytes, 0x00020000);
  const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(dst, (short)0, bytes, 0x00020000);
  for (int base = 0; base < nchunks; base += kThreads * U) {
    u32x4 r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int idx = base + u * kThreads + (int)threadIdx.x;
      if (poison)
        r[u] = u32x4{nan2, nan2, nan2, nan2};
      else
        r[u] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, idx * 16, 0, kLoadPolicy));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int idx = base + u * kThreads + (int)threadIdx.x;
      if constexpr (kSerialStores) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_raw_buffer_store_b128(r[u], rd, idx * 16, 0, kStorePolicy);
    }
  }
}

}  // namespace

// Workgroups of a copy kernel that the device runs at once (all CUs).
int copy_resident_groups(const void *kernel, size_t lds_reserve);

}  // namespace sc
