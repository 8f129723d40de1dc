// Microscaled 4-bit quantiser of dense rows and its inverse.
//
//   v = x / s,  a = max |v| over a block of a row
//   E8M0 (block 32):  X = 2^clamp(floor(log2 a) - 2, -127, 125)
//   E4M3 (block 16):  X = RNE_E4M3(min(a / 6, 448))
//   code = RNE_E2M1(v / X), saturated at +-6 (0 where X = 0)
//
// s is a power of two, so v is exact, and every rounding is the nearest one of
// the real quotient: the midpoints between codes times X have at most 7
// significant bits (those between scales times 6 at most 6), and a quotient
// v / X rounded to fp32 can only equal such a midpoint when v / X does: the
// nearest other fp32 v is at least 2^-24 |v| away from midpoint * X, more than
// the half ulp of a quotient next to the midpoint.
#include "microscale.cuh"

#include <cuda_runtime.h>

namespace {
using namespace bmoe;

constexpr int kMThreads = 256;

struct MicroArgs {
  const void* in;      // quantise: dense rows
  void* out;           // dequantise: dense rows
  int64_t ld;          // their pitch in elements
  int rows, cols;
  float s, inv;        // tensor scale and (quantise: a power of two) its reciprocal
  uint8_t* codes;
  uint8_t* scales;
  int64_t pitch;
  int tiles;           // 512-byte scale tiles across a row
  int vec;             // dense rows can be read or written 8 elements at a time
};

// Two floats -> two E2M1 codes, b in the lower half of the byte (nearest, ties to even, saturating).
__device__ __forceinline__ uint32_t e2m1x2(float hi, float lo) {
  uint32_t r;
  asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n cvt.u32.u8 %0, t;\n}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <typename T>
__device__ __forceinline__ void load8(const MicroArgs& a, int row, int c, float (&v)[8]) {
  const T* p = static_cast<const T*>(a.in) + (int64_t)row * a.ld + c;
  if (a.vec && c + 8 <= a.cols) {
    if constexpr (sizeof(T) == 4) {
      const float4 x = __ldcs(reinterpret_cast<const float4*>(p)), y = __ldcs(reinterpret_cast<const float4*>(p) + 1);
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
      v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    } else {
      const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16lo(w[i]);
        v[2 * i + 1] = bf16hi(w[i]);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = 0.f;
      if (c + i < a.cols) {
        if constexpr (sizeof(T) == 4) v[i] = p[i];
        else v[i] = __uint_as_float((uint32_t)__bfloat16_as_ushort(p[i]) << 16);
      }
    }
  }
}

// A lane takes 8 columns; 2 (E4M3) or 4 (E8M0) lanes share a block.  Rows and blocks
// past the matrix's own up to whole scale tiles are written as zeros.
template <typename T, int FMT>
__global__ void __launch_bounds__(kMThreads) k_micro_quantize(MicroArgs a) {
  constexpr int LPB = FMT == BITSMOE_MICRO_E8M0 ? 4 : 2;   // lanes of a block
  const int row = blockIdx.y + blockIdx.z * gridDim.y;
  const int c = (blockIdx.x * kMThreads + threadIdx.x) * 8;   // first column of this lane
  if (row >= (a.rows + 127) / 128 * 128) return;
  float v[8];
  float top = 0.f;
  bool bad = false;
  if (row < a.rows) {
    load8<T>(a, row, c, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] *= a.inv;
      bad |= !(fabsf(v[i]) <= 3.402823466e38f);
      top = fmaxf(top, fabsf(v[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
  }
#pragma unroll
  for (int o = 1; o < LPB; o <<= 1) {
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    bad |= __shfl_xor_sync(0xFFFFFFFFu, (int)bad, o) != 0;
  }
  uint32_t byte, code = 0;
  if (FMT == BITSMOE_MICRO_E8M0) {
    // exponent of a: the fp32 field (subnormal a: field 0, below every usable exponent)
    const int e = max((int)(__float_as_uint(top) >> 23) - 2, 0);
    byte = (uint32_t)e;
    const float r = __uint_as_float((uint32_t)(254 - e) << 23);   // 1 / 2^(e - 127), e in [0, 252]
#pragma unroll
    for (int i = 0; i < 4; ++i) code |= e2m1x2(v[2 * i + 1] * r, v[2 * i] * r) << (8 * i);
  } else {
    byte = __nv_cvt_float_to_fp8(__fdiv_rn(top, 6.f), __NV_SATFINITE, __NV_E4M3);
    const float x = micro_e4m3(byte);
    if (x > 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) code |= e2m1x2(__fdiv_rn(v[2 * i + 1], x), __fdiv_rn(v[2 * i], x)) << (8 * i);
    }
  }
  if (bad) {
    byte = FMT == BITSMOE_MICRO_E8M0 ? 255u : 127u;
    code = 0u;
  }
  if (row >= a.rows) byte = 0u;
  if (row < a.rows && c < a.pitch * 2) *reinterpret_cast<uint32_t*>(a.codes + (int64_t)row * a.pitch + c / 2) = code;
  const int b = c / (8 * LPB);
  if (threadIdx.x % LPB == 0 && b < a.tiles * 4)
    a.scales[micro_scale_at(a.tiles, row, b)] = (uint8_t)(c < a.cols ? byte : 0u);
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kMThreads) k_micro_dequantize(MicroArgs a) {
  constexpr int LPB = FMT == BITSMOE_MICRO_E8M0 ? 4 : 2;
  const int row = blockIdx.y + blockIdx.z * gridDim.y;
  const int c = (blockIdx.x * kMThreads + threadIdx.x) * 8;
  if (row >= a.rows || c >= a.cols) return;
  const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(a.codes + (int64_t)row * a.pitch + c / 2));
  const float x = micro_scale(FMT, a.scales[micro_scale_at(a.tiles, row, c / (8 * LPB))]);
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = micro_value((w >> (4 * i)) & 15u) * x * a.s;
  T* p = static_cast<T*>(a.out) + (int64_t)row * a.ld + c;
  if (a.vec && c + 8 <= a.cols) {
    if constexpr (sizeof(T) == 4) {
      reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      uint32_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        h[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
      *reinterpret_cast<uint4*>(p) = make_uint4(h[0], h[1], h[2], h[3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.cols) {
        if constexpr (sizeof(T) == 4) p[i] = v[i];
        else p[i] = __float2bfloat16_rn(v[i]);
      }
  }
}

// Grid: columns in x, rows in y and z (y alone holds 65535 rows).
dim3 row_grid(int64_t cols, int64_t rows) {
  const int64_t y = rows < 32768 ? rows : 32768;
  return dim3((unsigned)((cols + kMThreads * 8 - 1) / (kMThreads * 8)), (unsigned)y, (unsigned)((rows + y - 1) / y));
}

bool rows_aligned(const void* p, int64_t ld, int type) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (ld * dense_size(type)) % 16 == 0;
}

int dense_check(const void* p, int type, int64_t ld, int rows, int cols) {
  if (!dense_type_ok(type) || ld < cols) return BITSMOE_ERR_INVALID_ARG;
  if (rows == 0) return BITSMOE_OK;
  if (!p) return BITSMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(p) % dense_size(type)) return BITSMOE_ERR_ALIGNMENT;
  return BITSMOE_OK;
}

}  // namespace

extern "C" {

int bitsmoe_microscale_bytes(int format, int rows, int cols, size_t* codes, size_t* scales) {
  if (!micro_format_ok(format) || rows < 0 || cols < 1 || !codes || !scales) return BITSMOE_ERR_INVALID_ARG;
  if (rows > kMaxMicroRows || cols > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  *codes = (size_t)rows * (size_t)micro_pitch(cols);
  *scales = (size_t)((rows + 127) / 128) * (size_t)micro_tiles(format, cols) * 512;
  return BITSMOE_OK;
}

int bitsmoe_microscale_quantize(const void* x, int type, int64_t ld, const bitsmoe_microscale* q, void* stream) {
  int rc = micro_check(q);
  if (rc) return rc;
  int e = 0;
  if (std::frexp(q->scale, &e) != 0.5f || e < -99 || e > 101) return BITSMOE_ERR_INVALID_ARG;   // 2^-100 .. 2^100
  if ((rc = dense_check(x, type, ld, q->rows, q->cols))) return rc;
  if (q->rows == 0) return BITSMOE_OK;
  MicroArgs a{x, nullptr, ld, q->rows, q->cols, q->scale, 1.f / q->scale, q->codes, q->scales, micro_pitch(q->cols),
              micro_tiles(q->format, q->cols), rows_aligned(x, ld, type)};
  const dim3 g = row_grid((int64_t)a.tiles * 4 * micro_block(q->format), (a.rows + 127) / 128 * 128);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e8 = q->format == BITSMOE_MICRO_E8M0;
  if (type == BITSMOE_F32) {
    if (e8) k_micro_quantize<float, BITSMOE_MICRO_E8M0><<<g, kMThreads, 0, st>>>(a);
    else k_micro_quantize<float, BITSMOE_MICRO_E4M3><<<g, kMThreads, 0, st>>>(a);
  } else {
    if (e8) k_micro_quantize<__nv_bfloat16, BITSMOE_MICRO_E8M0><<<g, kMThreads, 0, st>>>(a);
    else k_micro_quantize<__nv_bfloat16, BITSMOE_MICRO_E4M3><<<g, kMThreads, 0, st>>>(a);
  }
  const cudaError_t r = cudaGetLastError();
  return r == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)r);
}

int bitsmoe_microscale_dequantize(const bitsmoe_microscale* q, void* x, int type, int64_t ld, void* stream) {
  int rc = micro_check(q);
  if (rc) return rc;
  if ((rc = dense_check(x, type, ld, q->rows, q->cols))) return rc;
  if (q->rows == 0) return BITSMOE_OK;
  MicroArgs a{nullptr, x, ld, q->rows, q->cols, q->scale, 0.f, q->codes, q->scales, micro_pitch(q->cols),
              micro_tiles(q->format, q->cols), rows_aligned(x, ld, type)};
  const dim3 g = row_grid(a.cols, a.rows);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e8 = q->format == BITSMOE_MICRO_E8M0;
  if (type == BITSMOE_F32) {
    if (e8) k_micro_dequantize<float, BITSMOE_MICRO_E8M0><<<g, kMThreads, 0, st>>>(a);
    else k_micro_dequantize<float, BITSMOE_MICRO_E4M3><<<g, kMThreads, 0, st>>>(a);
  } else {
    if (e8) k_micro_dequantize<__nv_bfloat16, BITSMOE_MICRO_E8M0><<<g, kMThreads, 0, st>>>(a);
    else k_micro_dequantize<__nv_bfloat16, BITSMOE_MICRO_E4M3><<<g, kMThreads, 0, st>>>(a);
  }
  const cudaError_t r = cudaGetLastError();
  return r == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)r);
}

}  // extern "C"
