// What the calls of the paged 8-bit cache share: its two forms of codes.
#pragma once

#include <cuda_fp16.h>

#include "hs_internal.cuh"

namespace hs {

// A code c of block b and head h stands for c * scale[b, h].
template <int FMT>
struct KvFormat;

template <>
struct KvFormat<HS_KV_E4M3> {
  static constexpr float kLargest = 448.0f;    // 1.75 * 2^8
  static constexpr int kLargestExp = 8;
  static constexpr uint32_t kLargestFrac = 0x600000u;  // the mantissa bits of 1.75

  // Two floats to two codes (x0 in the low byte), to nearest even, saturating; NaN stays NaN.
  static __device__ __forceinline__ uint32_t encode2(float x0, float x1) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(x1), "f"(x0));
    return r;
  }
  // The two codes in the low (HI = 0) or high half of w as half2: exact.
  template <int HI>
  static __device__ __forceinline__ uint32_t decode2(uint32_t w) {
    uint32_t r;
    const uint16_t h = (uint16_t)(HI ? w >> 16 : w & 0xffffu);
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(h));
    return r;
  }
};

template <>
struct KvFormat<HS_KV_INT8> {
  static constexpr float kLargest = 127.0f;    // 1.984375 * 2^6
  static constexpr int kLargestExp = 6;
  static constexpr uint32_t kLargestFrac = 0x7e0000u;  // the mantissa bits of 1.984375

  static __device__ __forceinline__ uint32_t encode1(float x) {
    // fmaxf and fminf would turn a NaN into an end of the range: it becomes 0
    const int i = x != x ? 0 : __float2int_rn(fminf(fmaxf(x, -127.0f), 127.0f));
    return (uint32_t)i & 0xffu;
  }
  static __device__ __forceinline__ uint32_t encode2(float x0, float x1) {
    return encode1(x0) | (encode1(x1) << 8);
  }
  // 1024 + (c + 128) is a half whose low byte is c ^ 0x80: exact.
  template <int HI>
  static __device__ __forceinline__ uint32_t decode2(uint32_t w) {
    const uint32_t u = __byte_perm(w ^ 0x80808080u, 0x64646464u, HI ? 0x4342 : 0x4140);
    const __half2 bias = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&u), bias);  // - 1152
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};

// The least power of two s >= 2^-126 with m <= kLargest * s (m >= 0, finite).
template <int FMT>
__device__ __forceinline__ float kv_scale(float m) {
  const uint32_t b = __float_as_uint(m);
  int e = (int)(b >> 23) - KvFormat<FMT>::kLargestExp;  // biased; subnormal m end at the least
  if ((b & 0x7fffffu) > KvFormat<FMT>::kLargestFrac) ++e;
  return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
}

}  // namespace hs
