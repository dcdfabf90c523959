// Device arithmetic of 8-bit K/V rows (kv_copy.hip, rope.hip, decode_attn.hip).
//
// A row x[0..D) of one token and KV head is held as one byte per element and
// one bf16 scale, value = code * s:
//     s = max(roundup_bf16(max |x| / T), 2^-126),  T = 127 (int8), 448 (e4m3)
//     code = nearest code to x / s, ties to even.
// The scale is a bf16 rounded up for three reasons: no quotient exceeds T,
// so no code is clipped; it adds 2 bytes a row instead of 4; and x (8 or 11
// significant bits) over s (8) is either exactly halfway between two codes
// or at least 2^-15 away from it, relatively, so an fp32 quotient decides
// every code as exact arithmetic would.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/swiftcache.h"

namespace sc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// 16-bit element pairs <-> fp32.
template <int DT>
__device__ __forceinline__ f32x2 unpack16(uint32_t w) {
  if constexpr (DT == SC_DTYPE_BF16) {
    return f32x2{__builtin_bit_cast(float, w << 16), __builtin_bit_cast(float, w & 0xffff0000u)};
  } else {
    const f16x2 h = __builtin_bit_cast(f16x2, w);
    return f32x2{(float)h.x, (float)h.y};
  }
}

// Rounded to nearest even.
template <int DT>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
  if constexpr (DT == SC_DTYPE_BF16) {
    const bf16x2 r = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, r);
  } else {
    const f16x2 r = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, r);
  }
}

// The four codes of a word as fp32.
template <int FMT>
__device__ __forceinline__ void codes_to_f32(uint32_t w, float (&f)[4]) {
  if constexpr (FMT == SC_KV_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int32_t)(int8_t)(w >> (8 * i));
  } else {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo.x, f[1] = lo.y, f[2] = hi.x, f[3] = hi.y;
  }
}

// Largest |x| of a row whose D / 8 consecutive lanes hold 8 elements each, as
// the 16-bit pattern of its magnitude: patterns of magnitudes order like the
// magnitudes, with infinity above every number and NaN above infinity.
__device__ __forceinline__ uint32_t row_max_bits(u32x4 x, int lanes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = x[i] & 0x7fffu, b = (x[i] >> 16) & 0x7fffu;
    m = max(m, max(a, b));
  }
  for (int s = 1; s < lanes; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
  return m;
}

// Codes of the 8 elements x of a row and the bits of its bf16 scale; every
// lane of the row calls it (`lanes` = D / 8).
template <int DT, int FMT>
__device__ __forceinline__ u32x2 quantise8(u32x4 x, int lanes, uint32_t *scale_bits) {
  constexpr uint32_t kInf = DT == SC_DTYPE_BF16 ? 0x7f80u : 0x7c00u;
  constexpr float kTop = FMT == SC_KV_INT8 ? 127.f : 448.f;
  // Magnitudes from here on round to infinity in the element type.
  constexpr float kOver = DT == SC_DTYPE_BF16 ? 0x1.ffp127f : 65520.f;
  const uint32_t mb = row_max_bits(x, lanes);
  const bool finite = mb < kInf;
  const float top = unpack16<DT>(mb).x;
  const float want = finite ? top / kTop : 0.f;
  uint32_t sb = (__builtin_bit_cast(uint32_t, want) + 0xffffu) >> 16;   // positive: up to the next bf16
  sb = max(sb, 0x0080u);                                                // 2^-126
  const float s = __builtin_bit_cast(float, sb << 16);
  *scale_bits = finite ? sb : 0x7fc0u;
  const float r = 1.f / s;
  const bool near_top = s * kTop >= kOver;   // the same for a whole row
  float y[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 v = unpack16<DT>(finite ? x[i] : 0u);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      // x / s: one correction step makes a representable quotient (every
      // tie is one) exact.
      const float q = v[j] * r;
      y[2 * i + j] = __builtin_fmaf(__builtin_fmaf(-q, s, v[j]), r, q);
    }
  }
  u32x2 code;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (FMT == SC_KV_INT8) {
      uint32_t w = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float c = __builtin_rintf(y[4 * h + i]);
        if (near_top && __builtin_fabsf(c * s) >= kOver) c -= __builtin_copysignf(1.f, c);
        w |= ((uint32_t)(int32_t)c & 0xffu) << (8 * i);
      }
      code[h] = w;
    } else {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], w, true);
      if (near_top) {
        float f[4];
        codes_to_f32<FMT>((uint32_t)w, f);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (__builtin_fabsf(f[i] * s) >= kOver) w -= 1 << (8 * i);   // a code's magnitude is its low 7 bits
      }
      code[h] = (uint32_t)w;
    }
  }
  return code;
}

}  // namespace sc
