// Row copies of pools with 8-bit blocks (sc_quant.h): the same items, grids
// and cache policies as kv_copy.hip.  A fetch multiplies codes by their
// row's scale and rounds once, a store quantises, an append is the 16-bit
// copy.  Bound by the bytes they move, a third of them on the pool's side.
// 32768 tokens of 8 heads of 128 out of e4m3 blocks: 37 us, 5.5 TB/s of codes
// and elements (a plain copy of 1 GiB: 4.8).
#include "sc_copy_rows.h"

namespace sc {
namespace {

// A lane converts 8 consecutive elements at a time: 8 bytes of codes against
// 16 bytes of elements, so that both sides of a wave's access are contiguous.
// Loads in flight: eight in the fetch alone; four in what shares a kernel with
// a store or append, because a wave beside two attention waves of a SIMD may
// have 48 registers (head_dim 64's widest attention kernel has 229 of 512)
// and the overlapped stack falls back to waiting on stream events otherwise.
constexpr int kFetchUnroll = 8;
constexpr int kUnroll8 = 4;

template <int FMT, int DT, bool kSerialStores, int U>
__device__ __forceinline__ void fetch8_rows(const CopyArgs &a, int g, bool poison = false, uint32_t nan2 = 0) {
  const int is_v = g & 1;
  const CopyItem it = load_item(a.items + (g >> 1));
  const int n8 = (int)(((int64_t)it.nrows * a.row_bytes) >> 3);
  const char *src = a.tier_base[it.tier] + it.pool_off + a.layer_off + (is_v ? a.v_half_off : 0);
  char *dst = (is_v ? a.act_v : a.act_k) + it.act_row * 2 * a.row_bytes;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(src), (short)0, n8 * 8, 0x00020000);
  const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(src + a.scale_off), (short)0,
                                                                      it.nrows * a.n_heads * 2, 0x00020000);
  const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(dst, (short)0, n8 * 16, 0x00020000);
  const int row_shift = a.dim_shift - 3;
  for (int base = 0; base < n8; base += kThreads * U) {
    u32x2 c[U];
    uint16_t sc[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int idx = base + u * kThreads + (int)threadIdx.x;
      c[u] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rs, idx * 8, 0, kLoadPolicy));
      sc[u] = __builtin_amdgcn_raw_buffer_load_b16(rc, (idx >> row_shift) * 2, 0, kLoadPolicy);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int idx = base + u * kThreads + (int)threadIdx.x;
      const float s = __builtin_bit_cast(float, (uint32_t)sc[u] << 16);
      u32x4 r;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float f[4];
        codes_to_f32<FMT>(c[u][h], f);
        r[2 * h] = poison ? nan2 : pack16<DT>(f[0] * s, f[1] * s);
        r[2 * h + 1] = poison ? nan2 : pack16<DT>(f[2] * s, f[3] * s);
      }
      if constexpr (kSerialStores) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_raw_buffer_store_b128(r, rd, idx * 16, 0, kStorePolicy);
      __builtin_amdgcn_sched_barrier(0);     // one conversion's registers at a time
    }
  }
}

template <int FMT, int DT, bool kSerialStores>
__device__ __forceinline__ void store8_rows(const CopyArgs &a, int g) {
  const int is_v = g & 1;
  const CopyItem it = load_item(a.items + (g >> 1));
  const int n8 = (int)(((int64_t)it.nrows * a.row_bytes) >> 3);
  const char *src = (is_v ? a.new_v : a.new_k) + it.src_row * 2 * a.row_bytes;
  char *dst = a.tier_base[it.tier] + it.pool_off + a.layer_off + (is_v ? a.v_half_off : 0);
  // pool_off points at the item's first row; the scales are counted from the block's.
  char *scales = dst - it.act_row * a.row_bytes + a.scale_off + it.act_row * a.n_heads * 2;
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(src), (short)0, n8 * 16, 0x00020000);
  const __amdgpu_buffer_rsrc_t rd = __builtin_amdgcn_make_buffer_rsrc(dst, (short)0, n8 * 8, 0x00020000);
  const __amdgpu_buffer_rsrc_t rc =
      __builtin_amdgcn_make_buffer_rsrc(scales, (short)0, it.nrows * a.n_heads * 2, 0x00020000);
  const int row_shift = a.dim_shift - 3, lanes = 1 << row_shift;
  for (int base = 0; base < n8; base += kThreads * kUnroll8) {
    u32x4 x[kUnroll8];
#pragma unroll
    for (int u = 0; u < kUnroll8; ++u)
      x[u] = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, (base + u * kThreads + (int)threadIdx.x) * 16, 0, kLoadPolicy));
#pragma unroll
    for (int u = 0; u < kUnroll8; ++u) {
      const int idx = base + u * kThreads + (int)threadIdx.x;
      uint32_t sb;
      const u32x2 code = quantise8<DT, FMT>(x[u], lanes, &sb);
      if constexpr (kSerialStores) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_raw_buffer_store_b64(code, rd, idx * 8, 0, kStorePolicy);
      if ((idx & (lanes - 1)) == 0)
        __builtin_amdgcn_raw_buffer_store_b16((uint16_t)sb, rc, (idx >> row_shift) * 2, 0, kStorePolicy);
    }
  }
}

template <int FMT, int DT>
__global__ __launch_bounds__(kThreads) void kv8_fetch_kernel(CopyArgs a) {
  if (a.serial_stores)
    for (int g = blockIdx.x; g < 2 * a.n_items; g += gridDim.x) fetch8_rows<FMT, DT, true, kFetchUnroll>(a, g);
  else
    for (int g = blockIdx.x; g < 2 * a.n_items; g += gridDim.x) fetch8_rows<FMT, DT, false, kFetchUnroll>(a, g);
}
template <int FMT, int DT>
__global__ __launch_bounds__(kThreads) void kv8_store_kernel(CopyArgs a) {
  for (int g = blockIdx.x; g < 2 * a.n_items; g += gridDim.x) store8_rows<FMT, DT, false>(a, g);
}

// kv_layer_copy_kernel over 8-bit blocks.
template <int FMT, int DT>
__global__ __launch_bounds__(kThreads) void kv8_layer_copy_kernel(LayerCopyArgs a) {
  const bool poison =
      a.fail_word != nullptr && __hip_atomic_load(a.fail_word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.fail_tag;
  const int n0 = 2 * a.part[0].n_items;
  const int n1 = n0 + 2 * a.part[1].n_items;
  const int n2 = n1 + 2 * a.part[2].n_items;
  for (int g = blockIdx.x; g < n2; g += gridDim.x) {
    if (g < n0)
      fetch8_rows<FMT, DT, true, kUnroll8>(a.part[0], g, poison, a.nan2);
    else if (g < n1)
      copy_rows<COPY_APPEND, true, kUnroll8>(a.part[1], g - n0, poison, a.nan2);
    else
      store8_rows<FMT, DT, true>(a.part[2], g - n1);
  }
}

// The kernels of one (format, element type).
struct Kernels8 {
  void (*fetch)(CopyArgs);
  void (*store)(CopyArgs);
  void (*layer)(LayerCopyArgs);
};
template <int FMT, int DT>
constexpr Kernels8 kernels8_of() {
  return {kv8_fetch_kernel<FMT, DT>, kv8_store_kernel<FMT, DT>, kv8_layer_copy_kernel<FMT, DT>};
}
Kernels8 kernels8(int kv_format, int dtype) {
  if (kv_format == SC_KV_INT8)
    return dtype == SC_DTYPE_BF16 ? kernels8_of<SC_KV_INT8, SC_DTYPE_BF16>() : kernels8_of<SC_KV_INT8, SC_DTYPE_F16>();
  return dtype == SC_DTYPE_BF16 ? kernels8_of<SC_KV_E4M3, SC_DTYPE_BF16>() : kernels8_of<SC_KV_E4M3, SC_DTYPE_F16>();
}

}  // namespace

int kv8_copy_vgprs(int kv_format) {
  int m = 0;
  for (int dtype : {SC_DTYPE_BF16, SC_DTYPE_F16}) {
    const Kernels8 k = kernels8(kv_format, dtype);
    for (const void *f : {reinterpret_cast<const void *>(k.fetch), reinterpret_cast<const void *>(k.store),
                          reinterpret_cast<const void *>(k.layer)}) {
      hipFuncAttributes at{};
      if (hipFuncGetAttributes(&at, f) != hipSuccess) return -1;
      m = at.numRegs > m ? at.numRegs : m;
    }
  }
  return m;
}

hipError_t launch_kv8_copy(const CopyArgs &args, hipStream_t stream, size_t lds_reserve, int max_groups) {
  const int groups = max_groups > 0 && max_groups < 2 * args.n_items ? max_groups : 2 * args.n_items;
  const Kernels8 k = kernels8(args.kv_format, args.dtype);
  CopyArgs a = args;
  // One store in flight per wave, or all: as launch_kv_copy.
  a.serial_stores =
      (max_groups > 0 || groups <= copy_resident_groups(reinterpret_cast<const void *>(k.fetch), lds_reserve)) ? 1 : 0;
  hipLaunchKernelGGL(a.mode == COPY_FETCH ? k.fetch : k.store, dim3(groups), dim3(kThreads), lds_reserve, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv8_layer_copy(const LayerCopyArgs &a, hipStream_t stream, size_t lds_reserve, int max_groups) {
  const int halves = 2 * (a.part[0].n_items + a.part[1].n_items + a.part[2].n_items);
  if (halves <= 0) return hipSuccess;
  const int groups = max_groups > 0 && max_groups < halves ? max_groups : halves;
  hipLaunchKernelGGL(kernels8(a.part[0].kv_format, a.part[0].dtype).layer, dim3(groups), dim3(kThreads), lds_reserve,
                     stream, a);
  return hipGetLastError();
}

}  // namespace sc
