// Microscaled 4-bit quantiser of dense rows and its inverse.
//
//   v = x / s,  a = max |v| over a block of a row
//   E8M0 (block 32):  X = 2^clamp(floor(log2 a) - 2, -127, 125)
//   E4M3 (block 16):  X = RNE_E4M3(min(a / 6, 448))
//   code = RNE_E2M1(v / X), saturated at +-6 (0 where X = 0)
//
// s is a power of two, so v is exact where it is a normal number.  (Below that
// E4M3's codes are 0, and E8M0's come from x / X / s, never rounded where it
// counts.)  Every rounding is the nearest one of the real quotient: the midpoints
// between codes times X have at most 7 significant bits (those between scales
// times 6 at most 6), and a quotient v / X rounded to fp32 can only equal such a
// midpoint when v / X does: the nearest other fp32 v is at least 2^-24 |v| away
// from midpoint * X, more than the half ulp of a quotient next to the midpoint.
#include <cuda_runtime.h>

#include "microscale.cuh"
#include "rows.cuh"

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
  int chunks;          // of the columns: quantise 256, dequantise 512 bytes of the result
  int vec;             // dense rows can be read or written 8 elements at a time
};

// v / x on the right side of every midpoint between codes, from r = 1 / x rounded.  bf16 rows: v has 8 significant
// bits and midpoint * x at most 7, so a quotient that is not a midpoint is at least 2^-8 of itself away from one, and
// v r (off by 2^-23) rounded to 16 bits is on its side, and exactly on it for a tie.  fp32 rows: v r is on the wrong
// side only within 2 units in the last place of a midpoint (whose mantissa's low 21 bits are zero); there the division
// decides.
template <typename T>
__device__ __forceinline__ float quotient(float v, float x, float r) {
  const float q = v * r;
  const uint32_t b = __float_as_uint(q);
  if constexpr (sizeof(T) == 4) return ((b + 4u) & 0x1FFFFFu) <= 8u ? __fdiv_rn(v, x) : q;
  return __uint_as_float((b + 0x80u) & 0xFFFFFF00u);
}
// RNE_E4M3(min(top / 6, 448)): the same for midpoints between scales (the low 19 bits).
__device__ __forceinline__ uint32_t scale_e4m3(float top) {
  float t = top * 0.16666667163372040f;
  if (((__float_as_uint(t) + 4u) & 0x7FFFFu) <= 8u) t = __fdiv_rn(top, 6.f);
  return __nv_cvt_float_to_fp8(t, __NV_SATFINITE, __NV_E4M3);
}

// Two floats -> two E2M1 codes, b in the lower half of the byte (nearest, ties to even, saturating).
__device__ __forceinline__ uint32_t e2m1x2(float hi, float lo) {
  uint32_t r;
  asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n cvt.u32.u8 %0, t;\n}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// A warp takes 256 columns of kRowsOfWarp rows 32 apart (r, r + 32, .. of a scale tile: the words of all four are 16 bytes in a
// row), their loads in flight together; a lane 8 columns, LPB lanes a block, LPT lanes the four blocks of a scale word.
// Neighbouring chunks of a row in neighbouring warps.  Rows and blocks past the matrix's own up to whole scale tiles are
// written as zeros.
// Rows of a warp: fp32 (32 bytes a lane and row) 2, bf16 4.  14336 x 4096, us with 1, 2, 4 rows: fp32 46.4, 41.6, 41.4
// (E8M0: 6.4 TB/s) and 65.0, 57.4, 66.0 (E4M3), off 16-byte boundaries 55, 54, 60 and 72, 73, 83; bf16 46.9, 36.2, 35.3
// and 55.2, 48.3, 44.2.  What bounds all but the first is what they issue an element.
// Rows off 16-byte boundaries (VEC false): a lane reads the aligned 16 bytes that hold its columns and shifts; there and
// back 14336 x 4095 fp32 takes 98 us (140 element by element; 82 for 4096 columns).
template <typename T>
constexpr int kRowsOfWarp = sizeof(T) == 4 ? 2 : 4;

template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kMThreads) k_micro_quantize(MicroArgs a) {
  constexpr int V = 8, LPB = FMT == BITSMOE_MICRO_E8M0 ? 4 : 2, LPT = 4 * LPB, R = kRowsOfWarp<T>;
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * (kMThreads / 32) + (threadIdx.x >> 5);   // (rows, chunk of 256 columns)
  const int64_t q = task / a.chunks;
  const int chunk = (int)(task - q * a.chunks);
  // q: row tile, R-th part of its four rows of a lane, lane
  const int64_t rt = q / (128 / R);
  const int rl = (int)(q - rt * (128 / R)), j0 = rl >> 5 << (R == 1 ? 0 : R == 2 ? 1 : 2);
  const int64_t r0 = rt * 128 + (rl & 31) + 32 * j0;
  const int c = (chunk * 32 + lane) * V;
  if (r0 >= (a.rows + 127) / 128 * 128) return;
  Eight<T> in[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    if (r0 + 32 * j < a.rows) {
      in[j] = load8<T, VEC>(a.in, a.ld, a.cols, r0 + 32 * j, c);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) * 2; ++i) in[j].w[i] = 0u;
    }
  }
  uint32_t words[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    float v[V];
    uint32_t most = 0u;   // the largest magnitude's bits; a NaN's or an infinity's are above every finite one's
#pragma unroll
    for (int i = 0; i < V; ++i) {
      v[i] = element<T>(in[j], i);
      most = max(most, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    }
#pragma unroll
    for (int o = 1; o < LPB; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
    most = __float_as_uint(__uint_as_float(most) * a.inv);   // of x / s
    const bool bad = most >= 0x7F800000u;
    uint32_t byte, code = 0;
    if (FMT == BITSMOE_MICRO_E8M0) {
      // exponent of a: the fp32 field (subnormal a: field 0, below every usable exponent)
      byte = bad ? 0u : (uint32_t)max((int)(most >> 23) - 2, 0);
      // 1 / X = 2^(127 - byte), byte in [0, 252].  x / X is below 8 s, and normal unless x / X / s is below 2^-26, so
      // the only rounding that counts is the code's (x / s first would lose bits of subnormals that a midpoint decides by).
      const float r = __uint_as_float((254u - byte) << 23);
#pragma unroll
      for (int i = 0; i < V / 2; ++i) code |= e2m1x2(v[2 * i + 1] * r * a.inv, v[2 * i] * r * a.inv) << (8 * i);
    } else {
      byte = scale_e4m3(__uint_as_float(most));
      const float x = micro_e4m3(byte), r = __frcp_rn(x);
      if (x > 0.f) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i)
          code |= e2m1x2(quotient<T>(v[2 * i + 1] * a.inv, x, r), quotient<T>(v[2 * i] * a.inv, x, r)) << (8 * i);
      }
    }
    if (bad) {
      byte = FMT == BITSMOE_MICRO_E8M0 ? 255u : 127u;
      code = 0u;
    }
    if (r0 + 32 * j >= a.rows || c >= a.cols) byte = 0u;
    if (LPB > 1) byte = __shfl_sync(0xFFFFFFFFu, byte, lane / LPB * LPB);   // (its first lane's: the later ones may be past the columns)
    if (r0 + 32 * j < a.rows && c < a.pitch * 2) {
      *reinterpret_cast<uint32_t*>(a.codes + (r0 + 32 * j) * a.pitch + c / 2) = code;
    }
    // the four blocks' bytes of a scale word
    uint32_t word = byte << (8 * (lane / LPB & 3));
#pragma unroll
    for (int o = LPB; o < LPT; o <<= 1) word |= __shfl_xor_sync(0xFFFFFFFFu, word, o);
    words[j] = word;
  }
  const int tile = chunk * (32 / LPT) + lane / LPT;
  if (lane % LPT == 0 && tile < a.tiles)
#pragma unroll
    for (int j = 0; j < R; ++j)
      *reinterpret_cast<uint32_t*>(a.scales + (rt * a.tiles + tile) * 512 + (rl & 31) * 16 + (j0 + j) * 4) = words[j];
}

// Four rows 32 apart a warp, V columns a lane in 16 bytes of the result, so that a store writes whole sectors (rows off
// 16-byte boundaries: turned in shared memory, so that neighbouring lanes still write neighbouring elements); the rows' scale
// words are one 16-byte load.  14336 x 4096 to fp32: 40 us, 6.6 TB/s (to bf16 27 to 28); with 32 bytes a lane in two stores 56 us.
template <typename T, int FMT, bool VEC>
__global__ void __launch_bounds__(kMThreads) k_micro_dequantize(MicroArgs a) {
  constexpr int V = 16 / sizeof(T), LPB = (FMT == BITSMOE_MICRO_E8M0 ? 32 : 16) / V, LPT = 4 * LPB;
  __shared__ uint4 turn[kMThreads / 32][32];
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * (kMThreads / 32) + (threadIdx.x >> 5);
  const int64_t q = task / a.chunks;
  const int chunk = (int)(task - q * a.chunks);
  const int64_t r0 = (q >> 5) * 128 + (q & 31);
  if (r0 >= a.rows) return;
  const uint8_t* scales = a.scales + (q >> 5) * a.tiles * 512 + (q & 31) * 16;
  const int c = (chunk * 32 + lane) * V;
  if (VEC && c >= a.cols) return;
  const bool in = VEC || c < a.cols;   // (off the boundaries lanes past the columns help to store)
  uint4 sc = make_uint4(0u, 0u, 0u, 0u);
  if (in) sc = __ldg(reinterpret_cast<const uint4*>(scales + (size_t)(chunk * (32 / LPT) + lane / LPT) * 512));
  const uint32_t words[4] = {sc.x, sc.y, sc.z, sc.w};
  uint32_t code[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    code[j] = 0u;
    if (in && r0 + 32 * j < a.rows) {
      const uint8_t* src = a.codes + (r0 + 32 * j) * a.pitch + c / 2;
      if constexpr (V == 8) code[j] = __ldg(reinterpret_cast<const uint32_t*>(src));
      else code[j] = __ldg(reinterpret_cast<const uint16_t*>(src));
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (r0 + 32 * j >= a.rows) break;
    const float x = micro_scale(FMT, words[j] >> (8 * (lane / LPB & 3)) & 255u);
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = micro_value(code[j] >> (4 * i) & 15u) * x * a.s;
    T* p = static_cast<T*>(a.out) + (r0 + 32 * j) * a.ld + c;
    if constexpr (!VEC) {   // neighbouring lanes store neighbouring columns, by way of shared memory
      uint4 x;
      if constexpr (sizeof(T) == 4) {
        x = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
      } else {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          h[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        x = make_uint4(h[0], h[1], h[2], h[3]);
      }
      __syncwarp();
      turn[threadIdx.x >> 5][lane] = x;
      __syncwarp();
      const T* t = reinterpret_cast<const T*>(turn[threadIdx.x >> 5]);
      T* first = static_cast<T*>(a.out) + (r0 + 32 * j) * a.ld + chunk * 32 * V;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (chunk * 32 * V + i * 32 + lane < a.cols) first[i * 32 + lane] = t[i * 32 + lane];
    } else if (c + V <= a.cols) {
      if constexpr (sizeof(T) == 4) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
      } else {
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
          h[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(h[0], h[1], h[2], h[3]));
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < a.cols) {
          if constexpr (sizeof(T) == 4) p[i] = v[i];
          else p[i] = __float2bfloat16_rn(v[i]);
        }
    }
  }
}

// Blocks for a warp per `rows` rows of a row tile and chunk of the columns, neighbouring chunks in neighbouring warps.
int64_t micro_grid(const MicroArgs& a, int rows) {
  return (((int64_t)a.rows + 127) / 128 * (128 / rows) * a.chunks + kMThreads / 32 - 1) / (kMThreads / 32);
}

template <typename T, int FMT>
void launch_quantize(const MicroArgs& a, unsigned grid, cudaStream_t st) {
  if (a.vec) k_micro_quantize<T, FMT, true><<<grid, kMThreads, 0, st>>>(a);
  else k_micro_quantize<T, FMT, false><<<grid, kMThreads, 0, st>>>(a);
}
template <typename T, int FMT>
void launch_dequantize(const MicroArgs& a, unsigned grid, cudaStream_t st) {
  if (a.vec) k_micro_dequantize<T, FMT, true><<<grid, kMThreads, 0, st>>>(a);
  else k_micro_dequantize<T, FMT, false><<<grid, kMThreads, 0, st>>>(a);
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

// Rows of bf16 at any address to rows on 16-byte boundaries: a lane reads the two aligned 16 bytes that hold its
// eight columns (neighbours share them in L1) and shifts.  A warp takes kAlignColumns / 8 of them of a row.
constexpr int kAlignColumns = 1024;
__global__ void __launch_bounds__(256) k_align_rows(const uint8_t* x, int64_t pitch, int T, int cols, uint4* out, int64_t out_pitch) {
  const int c0 = blockIdx.y * (kAlignColumns / 8), nc = min((cols + 7) / 8, c0 + kAlignColumns / 8);
  for (int64_t t = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; t < T; t += (int64_t)gridDim.x * 8) {
    const uint8_t* row = x + t * pitch;
    uint4* to = out + t * out_pitch;
    const uint32_t a = (uint32_t)(reinterpret_cast<uintptr_t>(row) & 15);   // of every 16 bytes of the row
#pragma unroll 4
    for (int c = c0 + threadIdx.x % 32; c < nc; c += 32) {
      const uint4* p = reinterpret_cast<const uint4*>(row - a) + c;
      const uint4 lo = __ldg(p);
      const int n = cols - 8 * c;                                                // its columns (8 at most count)
      const uint4 hi = a && 16 - (int)a < 2 * n ? __ldg(p + 1) : make_uint4(0u, 0u, 0u, 0u);   // holds one of them
      uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
      if (a & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
      if (a & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
      if (a & 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] &= n >= 2 * i + 2 ? 0xFFFFFFFFu : n == 2 * i + 1 ? 0xFFFFu : 0u;
      to[c] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
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
              micro_tiles(q->format, q->cols), (q->cols + 255) / 256, rows_aligned(x, ld, type)};
  const int64_t grid = micro_grid(a, type == BITSMOE_F32 ? kRowsOfWarp<float> : kRowsOfWarp<__nv_bfloat16>);
  if (grid >= (1ll << 31)) return BITSMOE_ERR_SHAPE;
  const unsigned g = (unsigned)grid;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e8 = q->format == BITSMOE_MICRO_E8M0;
  if (type == BITSMOE_F32) {
    if (e8) launch_quantize<float, BITSMOE_MICRO_E8M0>(a, g, st);
    else launch_quantize<float, BITSMOE_MICRO_E4M3>(a, g, st);
  } else {
    if (e8) launch_quantize<__nv_bfloat16, BITSMOE_MICRO_E8M0>(a, g, st);
    else launch_quantize<__nv_bfloat16, BITSMOE_MICRO_E4M3>(a, g, st);
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
              micro_tiles(q->format, q->cols), (q->cols + 512 / dense_size(type) - 1) / (512 / dense_size(type)), rows_aligned(x, ld, type)};
  const int64_t grid = micro_grid(a, 4);
  if (grid >= (1ll << 31)) return BITSMOE_ERR_SHAPE;
  const unsigned g = (unsigned)grid;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool e8 = q->format == BITSMOE_MICRO_E8M0;
  if (type == BITSMOE_F32) {
    if (e8) launch_dequantize<float, BITSMOE_MICRO_E8M0>(a, g, st);
    else launch_dequantize<float, BITSMOE_MICRO_E4M3>(a, g, st);
  } else {
    if (e8) launch_dequantize<__nv_bfloat16, BITSMOE_MICRO_E8M0>(a, g, st);
    else launch_dequantize<__nv_bfloat16, BITSMOE_MICRO_E4M3>(a, g, st);
  }
  const cudaError_t r = cudaGetLastError();
  return r == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)r);
}

}  // extern "C"

extern "C" int bitsmoe_microscale_align(const void* x, int64_t x_ld, int T, int cols, void* out, int64_t out_ld, void* stream) {
  if (T < 0 || cols < 1 || x_ld < cols || out_ld < cols || out_ld % 8) return BITSMOE_ERR_INVALID_ARG;
  if (T > kMaxMicroRows || cols > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  if (T == 0) return BITSMOE_OK;
  if (!x || !out) return BITSMOE_ERR_INVALID_ARG;
  if ((uintptr_t)x % 2 || (uintptr_t)out % 16) return BITSMOE_ERR_ALIGNMENT;
  int dev = 0, sms = 0;
  cudaError_t e = device_sms(&dev, &sms);
  if (e != cudaSuccess) return record_cuda_error((int)e);
  const dim3 grid((unsigned)std::min<int64_t>(((int64_t)T + 7) / 8, 8ll * sms), (unsigned)((cols + kAlignColumns - 1) / kAlignColumns));
  k_align_rows<<<grid, 256, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint8_t*>(x), x_ld * 2, T, cols, static_cast<uint4*>(out), out_ld / 8);
  e = cudaGetLastError();
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
