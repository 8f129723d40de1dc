// Microscaled 4-bit matrices (library-internal): the stored layout, its host
// checks, and the device conversions of codes and block scales.
//
// Elements are E2M1 (sign, 2 exponent bits, 1 mantissa bit: 0, 1/2, 1, 3/2, 2,
// 3, 4, 6), one scale byte per block of consecutive columns of a row: 2^(c-127)
// per 32 columns (E8M0), or an fp8 E4M3 per 16 columns.  Codes are row-major,
// two a byte.  Scales are stored in tiles of 128 rows x 4 blocks (512 bytes),
// row r of a tile at byte (r % 32) * 16 + (r / 32) * 4: the order in which 32
// tensor-memory lanes x 4 columns take the scales of 128 rows, so that a tile
// goes from global memory to the tensor core by copies alone.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include <atomic>
#include <cmath>

#include "device.cuh"

namespace bmoe {

constexpr int kMaxMicroRows = 1 << 24;
constexpr int kMaxMicroCols = 1 << 20;

__host__ __device__ inline int micro_block(int format) { return format == BITSMOE_MICRO_E8M0 ? 32 : 16; }
__host__ __device__ inline int64_t micro_pitch(int cols) { return ((int64_t)cols + 31) / 32 * 16; }   // bytes of a row's codes
__host__ __device__ inline int micro_blocks(int format, int cols) {
  const int b = micro_block(format);
  return (cols + b - 1) / b;
}
__host__ __device__ inline int micro_tiles(int format, int cols) { return (micro_blocks(format, cols) + 3) / 4; }   // 512-byte tiles across a row
__host__ __device__ inline int64_t micro_scale_at(int tiles, int64_t r, int b) {
  return ((r >> 7) * tiles + (b >> 2)) * 512 + (r & 31) * 16 + ((r & 127) >> 5) * 4 + (b & 3);
}

inline bool micro_format_ok(int f) { return f == BITSMOE_MICRO_E8M0 || f == BITSMOE_MICRO_E4M3; }
inline bool dense_type_ok(int t) { return t == BITSMOE_F32 || t == BITSMOE_BF16; }
inline int dense_size(int t) { return t == BITSMOE_F32 ? 4 : 2; }

// A described matrix: sizes, scale and pointers (BITSMOE_OK or an error code).
inline int micro_check(const bitsmoe_microscale* m) {
  if (!m || !micro_format_ok(m->format) || m->rows < 0 || m->cols < 1) return BITSMOE_ERR_INVALID_ARG;
  if (!(m->scale > 0.f) || !std::isfinite(m->scale)) return BITSMOE_ERR_INVALID_ARG;
  if (m->rows > kMaxMicroRows || m->cols > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  if (m->rows == 0) return BITSMOE_OK;
  if (!m->codes || !m->scales) return BITSMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(m->codes) % 16 || reinterpret_cast<uintptr_t>(m->scales) % 16)
    return BITSMOE_ERR_ALIGNMENT;
  return BITSMOE_OK;
}

// SMs of the current device, asked once for each (a query of the runtime takes as long as a small kernel's launch).
inline cudaError_t device_sms(int* dev, int* sms) {
  static std::atomic<int> known[64];
  const cudaError_t e = cudaGetDevice(dev);
  if (e != cudaSuccess) return e;
  const int i = *dev & 63;
  *sms = *dev < 64 ? known[i].load(std::memory_order_relaxed) : 0;
  if (*sms > 0) return cudaSuccess;
  const cudaError_t r = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
  if (r == cudaSuccess && *dev < 64) known[i].store(*sms, std::memory_order_relaxed);
  return r;
}

// The dynamic shared memory that a kernel may ask for on device `dev`, set once for each (K: the kernel).
template <auto K>
cudaError_t allow_shared(int dev, int bytes) {
  static std::atomic<uint64_t> done;
  if (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
  const cudaError_t r = cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (r == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return r;
}

}  // namespace bmoe

namespace {

// Value of a scale byte in fp32 (both formats' values are fp32 values; NaN codes give NaN).
__device__ __forceinline__ float micro_e8m0(uint32_t c) {
  return __uint_as_float(c == 255u ? 0x7FC00000u : c ? c << 23 : 0x00400000u);
}
__device__ __forceinline__ float micro_e4m3(uint32_t c) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)c, __NV_E4M3)));
}
__device__ __forceinline__ float micro_scale(int format, uint32_t c) {
  return format == BITSMOE_MICRO_E8M0 ? micro_e8m0(c) : micro_e4m3(c);
}
// Value of a code (0..15): as fp16 bits, the code's exponent and mantissa one after the other are the
// value times 2^-14 (E2M1's bias is 1, fp16's is 15; zero exponents are subnormal in both).
__device__ __forceinline__ float micro_value(uint32_t c) {
  return __half2float(__ushort_as_half((unsigned short)(((c & 7u) << 9) | ((c & 8u) << 12)))) * 16384.f;
}

}  // namespace
