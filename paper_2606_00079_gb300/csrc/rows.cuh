// Dense rows of fp32 or bf16 on any pitch and alignment, eight elements a thread at a time, and rows in 8 bits:
// the scale of a row and its codes (library-internal).
#pragma once
#include <stdint.h>

#include "device.cuh"

namespace {

// Eight elements of a row from column c as they are stored, zeros past the columns.
template <typename T>
struct Eight {
  uint32_t w[sizeof(T) * 2];
};
template <typename T, bool VEC>   // VEC: rows on 16-byte boundaries
__device__ __forceinline__ Eight<T> load8(const void* in, int64_t ld, int cols, int64_t row, int c) {
  Eight<T> v;
  const T* p = static_cast<const T*>(in) + row * ld + c;
  if (VEC && c + 8 <= cols) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p) + i);
      v.w[4 * i] = x.x, v.w[4 * i + 1] = x.y, v.w[4 * i + 2] = x.z, v.w[4 * i + 3] = x.w;
    }
    return v;
  }
  if constexpr (VEC) {   // the last columns
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) * 2; ++i) v.w[i] = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < cols) {
        if constexpr (sizeof(T) == 4) v.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
        else v.w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i & 1));
      }
    return v;
  }
  // the aligned 16 bytes that hold one of the columns, shifted
  constexpr int G = sizeof(T) / 2 + 1, W = 2 * sizeof(T);
  const int n = cols - c;   // its columns (8 at most count)
  uint32_t w[4 * G];
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
  const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<const uint8_t*>(p) - off);
#pragma unroll
  for (int i = 0; i < G; ++i) {
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (16 * i < (int)off + (int)sizeof(T) * min(n, 8) && n > 0) x = __ldg(q + i);
    w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
  }
  if (off & 8)
#pragma unroll
    for (int i = 0; i < 4 * G - 2; ++i) w[i] = w[i + 2];
  if (off & 4)
#pragma unroll
    for (int i = 0; i < 4 * G - 1; ++i) w[i] = w[i + 1];
  if constexpr (sizeof(T) == 2) {
    if (off & 2)
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (sizeof(T) == 4) v.w[i] = i < n ? w[i] : 0u;
    else v.w[i] = 2 * i + 2 <= n ? w[i] : 2 * i + 1 == n ? w[i] & 0xFFFFu : 0u;
  }
  return v;
}
template <typename T>
__device__ __forceinline__ float element(const Eight<T>& v, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(v.w[i]);
  else return i & 1 ? bf16hi(v.w[i / 2]) : bf16lo(v.w[i / 2]);
}

// ---------------------------------------------------------------------------
// Rows in 8 bits: E4M3 codes with a power of two a row, the smallest with largest / scale <= 448 = 1.75 * 2^8.
// ---------------------------------------------------------------------------
constexpr int kRowscaleLow = -100;   // the scale's least exponent (rows of zeros)

// Exponent of the scale of a row whose largest magnitude has these bits (a NaN's or an infinity's are above every finite one's).
__device__ __forceinline__ int rowscale_exponent(uint32_t most) {
  return max((int)(most >> 23) - 135 + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0), kRowscaleLow);
}
__device__ __forceinline__ bool rowscale_bad(uint32_t most) { return most >= 0x7F800000u; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }   // -126 .. 127
__device__ __forceinline__ float rowscale_of(uint32_t most) {
  return rowscale_bad(most) ? __uint_as_float(0x7FC00000u) : power_of_two(rowscale_exponent(most));
}
// What the elements are multiplied by (exactly) before they are rounded to codes; 0 for a row that is not finite.
__device__ __forceinline__ float rowscale_inverse(uint32_t most) {
  return rowscale_bad(most) ? 0.f : power_of_two(-rowscale_exponent(most));
}
// Two floats -> two codes, the first in the lower byte (nearest, ties to even).
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) { return e4m3x2(a, b) | e4m3x2(c, d) << 16; }
// Four codes' values.
__device__ __forceinline__ float4 e4m3_values(uint32_t w) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(w & 0xFFFFu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(w >> 16)));
  return make_float4(f16lo(lo), f16hi(lo), f16lo(hi), f16hi(hi));
}

}  // namespace
