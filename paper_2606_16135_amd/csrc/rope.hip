// Rotary positions (sc_rope_apply) and the write of a decode step's tokens
// into the pool (sc_decode_store).
//
// A pair (x0, x1) of a head turns by the angle f = position * theta:
//     y0 = x0 cos f - x1 sin f,   y1 = x0 sin f + x1 cos f.
// The angle is taken in turns, in double precision: position * (theta / 2 pi)
// less its nearest whole number is exact to 2^-52 of the product, so a
// position of 10^6 loses nothing, where an fp32 product would be off by a
// tenth of a radian.  The fraction of a turn then needs fp32 only.
//
// Both are bound by the bytes they move (each element read and written once,
// three fp32 operations).  A workgroup first computes its tokens' cosines
// and sines, one per thread, into LDS and then turns every head of q and k
// with them: the double-precision work and the sine are paid once per token
// and pair, not once per head.  Elements move 16 bytes a lane.  16384 tokens
// of 40 + 8 heads of 128, out of a fused projection's rows: 73 us, 5.5 TB/s
// (a plain copy of 1 GiB: 4.8); 8 tokens: 3.5 us, one workgroup's latency.
#include "sc_internal.h"
#include "sc_pool_view.h"
#include "sc_quant.h"

#include <algorithm>

namespace sc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxHalf = 64;          // head_dim 128 / 2
constexpr int kTokens = 16;           // tokens of a workgroup, at most

// cos and sin of pair i at a position, amplitude included.
__device__ __forceinline__ float2 angle_of(const RopeView &r, int32_t position, int i) {
  const double t = (double)position * r.turns[i];
  const float f = (float)(t - __builtin_rint(t));
  float s, c;
  sincospif(2.f * f, &s, &c);
  return float2{c * r.amplitude, s * r.amplitude};
}

__device__ __forceinline__ float turn0(float x0, float x1, float2 cs) { return __builtin_fmaf(x0, cs.x, -(x1 * cs.y)); }
__device__ __forceinline__ float turn1(float x0, float x1, float2 cs) { return __builtin_fmaf(x0, cs.y, x1 * cs.x); }

// 8 elements and the 8 they are paired with (half layout), cs: their pairs'.
template <int DT>
__device__ __forceinline__ void turn_halves(u32x4 &a, u32x4 &b, const float2 *cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 x0 = unpack16<DT>(a[i]), x1 = unpack16<DT>(b[i]);
    const float2 c0 = cs[2 * i], c1 = cs[2 * i + 1];
    a[i] = pack16<DT>(turn0(x0.x, x1.x, c0), turn0(x0.y, x1.y, c1));
    b[i] = pack16<DT>(turn1(x0.x, x1.x, c0), turn1(x0.y, x1.y, c1));
  }
}
// 8 elements, four adjacent pairs (interleaved layout).
template <int DT>
__device__ __forceinline__ void turn_adjacent(u32x4 &a, const float2 *cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 x = unpack16<DT>(a[i]);
    a[i] = pack16<DT>(turn0(x.x, x.y, cs[i]), turn1(x.x, x.y, cs[i]));
  }
}

// Units of work of one head: a unit turns (or copies) 8 or 8 + 8 elements
// and is the only one that reads or writes them, so x == y works.  In place
// the copied elements need none.
__host__ __device__ inline int rope_units(int half, int interleaved, int dim_shift, bool in_place) {
  const int turned = interleaved ? half >> 2 : half >> 3;
  return turned + (in_place ? 0 : ((1 << dim_shift) - 2 * half) >> 3);
}

template <int DT>
__device__ __forceinline__ void rope_unit(const RopeView &r, const uint16_t *x, uint16_t *y, int unit, const float2 *cs) {
  const int turned = r.interleaved ? r.half >> 2 : r.half >> 3;
  if (unit >= turned) {
    const int at = 2 * r.half + 8 * (unit - turned);
    *reinterpret_cast<u32x4 *>(y + at) = *reinterpret_cast<const u32x4 *>(x + at);
  } else if (r.interleaved) {
    u32x4 a = *reinterpret_cast<const u32x4 *>(x + 8 * unit);
    turn_adjacent<DT>(a, cs + 4 * unit);
    *reinterpret_cast<u32x4 *>(y + 8 * unit) = a;
  } else {
    u32x4 a = *reinterpret_cast<const u32x4 *>(x + 8 * unit);
    u32x4 b = *reinterpret_cast<const u32x4 *>(x + r.half + 8 * unit);
    turn_halves<DT>(a, b, cs + 8 * unit);
    *reinterpret_cast<u32x4 *>(y + 8 * unit) = a;
    *reinterpret_cast<u32x4 *>(y + r.half + 8 * unit) = b;
  }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, int tokens_per_group, int units_q, int units_k) {
  __shared__ float2 cs[kTokens * kMaxHalf];
  const int t0 = blockIdx.x * tokens_per_group;
  const int nt = min(tokens_per_group, a.n_tokens - t0);
  const int half = a.rope.half;
  for (int i = threadIdx.x; i < nt * half; i += kThreads) {
    const int t = i / half;
    cs[t * kMaxHalf + (i - t * half)] = angle_of(a.rope, a.positions[t0 + t], i - t * half);
  }
  __syncthreads();
  const int per_q = a.heads[0] * units_q, per = per_q + a.heads[1] * units_k;
  for (int u = threadIdx.x; u < nt * per; u += kThreads) {
    const int t = u / per;
    int v = u - t * per;
    const int which = v >= per_q ? 1 : 0;
    v -= which ? per_q : 0;
    const int units = which ? units_k : units_q;
    const int h = v / units;
    const int64_t tok = t0 + t, head = (int64_t)h << a.dim_shift;
    rope_unit<DT>(a.rope, a.x[which] + tok * a.x_stride[which] + head, a.y[which] + tok * a.y_stride[which] + head,
                  v - h * units, cs + t * kMaxHalf);
  }
}

// ---------------------------------------------------------------------------
// Decode store.  Workgroup (x, y): token row x of the step, 256 of its units
// from 256 y on.  Units of the token: 8 elements each of k, then of v, then
// q's rotary units.  A lane of k or v holds 8 consecutive elements of its
// row (the partners of a half-layout pair are read a second time, from the
// cache), which is the form quantise8 takes.
// 33 sequences' k, v and q (8, 8 and 40 heads of 128): 4.7 us, latency.
// ---------------------------------------------------------------------------
template <int DT, int FMT>
__global__ __launch_bounds__(kThreads) void decode_store_kernel(DecodeStoreArgs a, int units_q) {
  __shared__ float2 cs[kMaxHalf];
  const PoolView &p = a.pool;
  const int row = blockIdx.x;
  const int b = row / a.batch.n_new;
  const int len = a.batch.kv_len[b];
  if (len < 0) return;                       // an empty slot
  const int pos = len - a.batch.n_new + (row - b * a.batch.n_new);
  if (a.rope.turns != nullptr) {
    if ((int)threadIdx.x < a.rope.half) cs[threadIdx.x] = angle_of(a.rope, a.batch.shared_len + pos, threadIdx.x);
    __syncthreads();
  }
  const int dim_shift = p.head_dim == 128 ? 7 : 6;
  const int lanes = p.head_dim >> 3;
  const int n_kv = p.n_kv_heads * lanes;
  const int u = blockIdx.y * kThreads + threadIdx.x;
  // The token's place; a lane group shares u's range below, so lanes of one
  // row stay together (n_kv is a multiple of lanes, kThreads too).
  char *at = nullptr;
  int in_block = 0;
  if (pos >= 0 && u < 2 * n_kv && len <= a.batch.max_len) {
    const int blk = block_of(p, pos);
    in_block = pos - blk * p.block_size;
    if (blk < a.batch.max_blocks)
      at = block_layer(p, a.batch.block_ids[(int64_t)b * a.batch.max_blocks + blk]);
  }
  if (u < 2 * n_kv) {
    const int is_v = u >= n_kv ? 1 : 0;
    const int e = u - is_v * n_kv;           // 8-element chunk of the token's row
    const uint16_t *src = (is_v ? a.v : a.k) + (int64_t)row * p.n_kv_heads * p.head_dim;
    u32x4 x = *reinterpret_cast<const u32x4 *>(src + 8 * e);
    const int d0 = 8 * (e & (lanes - 1));
    if (!is_v && a.rope.turns != nullptr && d0 < 2 * a.rope.half) {
      if (a.rope.interleaved) {
        turn_adjacent<DT>(x, cs + (d0 >> 1));
      } else {
        const bool second = d0 >= a.rope.half;
        u32x4 other = *reinterpret_cast<const u32x4 *>(src + 8 * e + (second ? -a.rope.half : a.rope.half));
        u32x4 lo = second ? other : x, hi = second ? x : other;
        turn_halves<DT>(lo, hi, cs + (second ? d0 - a.rope.half : d0));
        x = second ? hi : lo;
      }
    }
    char *half = at == nullptr ? nullptr : at + (is_v ? p.half_bytes : 0);
    if constexpr (FMT == SC_KV_16BIT) {
      if (half != nullptr)
        *reinterpret_cast<u32x4 *>(half + ((int64_t)in_block * n_kv + e) * 16) = x;
    } else {
      uint32_t sb;
      const u32x2 code = quantise8<DT, FMT>(x, lanes, &sb);
      if (half != nullptr) {
        *reinterpret_cast<u32x2 *>(half + ((int64_t)in_block * n_kv + e) * 8) = code;
        if (d0 == 0)
          *reinterpret_cast<uint16_t *>(half + p.scale_off + ((int64_t)in_block * p.n_kv_heads + e / lanes) * 2) =
              (uint16_t)sb;
      }
    }
  } else if (u - 2 * n_kv < a.n_q_heads * units_q) {
    const int v = u - 2 * n_kv;
    const int h = v / units_q;
    const int64_t off = ((int64_t)row * a.n_q_heads + h) << dim_shift;
    rope_unit<DT>(a.rope, a.q + off, a.q_out + off, v - h * units_q, cs);
  }
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream) {
  const int uq = rope_units(a.rope.half, a.rope.interleaved, a.dim_shift, a.in_place[0] != 0);
  const int uk = rope_units(a.rope.half, a.rope.interleaved, a.dim_shift, a.in_place[1] != 0);
  if (a.n_tokens <= 0 || a.heads[0] + a.heads[1] <= 0) return hipSuccess;
  // One token per workgroup while that leaves CUs idle; else as many as give
  // every thread a unit.  16384 tokens of 40 heads of 128 (320 units) by one
  // 58 us, by four 67; 65536 of 10 heads (80 units) by one 95, by four 59.
  const int units = a.heads[0] * uq + a.heads[1] * uk;
  const int per = a.n_tokens <= 1024 ? 1 : std::min(kTokens, (kThreads + units - 1) / std::max(1, units));
  // A launch's threads are counted in 32 bits.
  constexpr int64_t kSlice = 1 << 23;
  for (int64_t t0 = 0; t0 < a.n_tokens; t0 += kSlice) {
    RopeArgs b = a;
    b.n_tokens = (int32_t)std::min(kSlice, a.n_tokens - t0);
    b.positions += t0;
    for (int i = 0; i < 2; ++i) {
      if (b.heads[i] == 0) continue;
      b.x[i] += t0 * b.x_stride[i];
      b.y[i] += t0 * b.y_stride[i];
    }
    hipLaunchKernelGGL(a.dtype == SC_DTYPE_BF16 ? rope_kernel<SC_DTYPE_BF16> : rope_kernel<SC_DTYPE_F16>,
                       dim3((unsigned)((b.n_tokens + per - 1) / per)), dim3(kThreads), 0, stream, b, per, uq, uk);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_decode_store(const DecodeStoreArgs &a, hipStream_t stream) {
  const int dim_shift = a.pool.head_dim == 128 ? 7 : 6;
  const int uq = a.n_q_heads > 0 ? rope_units(a.rope.half, a.rope.interleaved, dim_shift, a.q_in_place != 0) : 1;
  const int64_t units = 2ll * a.pool.n_kv_heads * (a.pool.head_dim >> 3) + (int64_t)a.n_q_heads * uq;
  const dim3 grid((unsigned)(a.batch.batch * a.batch.n_new), (unsigned)((units + kThreads - 1) / kThreads));
  void (*kernel)(DecodeStoreArgs, int) = nullptr;
  const bool bf16 = a.pool.dtype == SC_DTYPE_BF16;
  switch (a.pool.kv_format) {
    case SC_KV_16BIT:
      kernel = bf16 ? decode_store_kernel<SC_DTYPE_BF16, SC_KV_16BIT> : decode_store_kernel<SC_DTYPE_F16, SC_KV_16BIT>;
      break;
    case SC_KV_INT8:
      kernel = bf16 ? decode_store_kernel<SC_DTYPE_BF16, SC_KV_INT8> : decode_store_kernel<SC_DTYPE_F16, SC_KV_INT8>;
      break;
    default:
      kernel = bf16 ? decode_store_kernel<SC_DTYPE_BF16, SC_KV_E4M3> : decode_store_kernel<SC_DTYPE_F16, SC_KV_E4M3>;
  }
  hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, a, uq);
  return hipGetLastError();
}

}  // namespace sc
