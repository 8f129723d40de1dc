// Rows in 8 bits (E4M3 codes, a power-of-two scale a row) from dense rows, and back:
//
//   a = max_k |x[r][k]|,  s = 2^max(-100, ceil(log2(a / 448))),  code = RNE_E4M3(x / s)
//
// x / s is exact (s is a power of two, a / s at most 448; what underflows lies far below half of the least code), so
// the conversion's rounding is the only one.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "microscale.cuh"
#include "rows.cuh"

namespace {
using namespace bmoe;

struct RowscaleArgs {
  const void* in;      // quantise: dense rows
  void* out;           // dequantise: dense rows
  int64_t ld;          // their pitch in elements
  int rows, cols;
  uint8_t* codes;
  int64_t pitch;       // of the codes, bytes
  float* scales;
  int vec;             // codes can be read and written 8 at a time
  int chunks, shift;   // dequantise: chunks of a row; log2 of the lanes that take one
};

// The codes of columns c .. c + 7 of a row.
template <typename T>
__device__ __forceinline__ void put8(const RowscaleArgs& a, int64_t row, int c, const Eight<T>& v, float inv, bool bad) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = element<T>(v, i) * inv;
  uint2 w = make_uint2(e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
  if (bad) w = make_uint2(0u, 0u);
  uint8_t* p = a.codes + row * a.pitch + c;
  if (a.vec && c + 8 <= a.cols) {
    *reinterpret_cast<uint2*>(p) = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < a.cols) p[i] = (uint8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3)));
}

template <typename T>
__device__ __forceinline__ uint32_t most8(const Eight<T>& v) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(element<T>(v, i)) & 0x7FFFFFFFu);
  return m;
}

// A row a group of G threads, the whole row in registers (NV times 8 elements a thread): read once, one maximum over the
// group, written.  DRAM bounds it: 14336 x 4096 fp32 38 us (294 MB, of which the codes stay in L2), and back 42.
template <typename T, bool VEC, int G, int NV>
__global__ void __launch_bounds__(G < 128 ? 128 : G) k_rowscale_quantize(const __grid_constant__ RowscaleArgs a) {
  constexpr int kThreads = G < 128 ? 128 : G, kRows = kThreads / G;
  __shared__ uint32_t red[kThreads / 32];
  const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  const int gi = threadIdx.x % G;
  if (G >= 32 && row >= a.rows) return;   // (whole warps; smaller groups help their warp's exchange)
  Eight<T> v[NV];
  uint32_t most = 0u;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * G + gi) * 8;
    if (c < a.cols && (G >= 32 || row < a.rows)) {
      v[k] = load8<T, VEC>(a.in, a.ld, a.cols, row, c);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T) * 2; ++i) v[k].w[i] = 0u;
    }
  }
#pragma unroll
  for (int k = 0; k < NV; ++k) most = max(most, most8<T>(v[k]));
  if constexpr (G < 32) {
#pragma unroll
    for (int o = 1; o < G; o <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, o));
  } else {
    most = __reduce_max_sync(0xFFFFFFFFu, most);
  }
  if constexpr (G > 32) {
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / 32; ++i) most = max(most, red[i]);
  }
  if (G < 32 && row >= a.rows) return;
  const float inv = rowscale_inverse(most);
  const bool bad = rowscale_bad(most);
  if (gi == 0) a.scales[row] = rowscale_of(most);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * G + gi) * 8;
    if (c < a.cols) put8<T>(a, row, c, v[k], inv, bad);
  }
}

// Rows that registers do not hold: a block a row, read twice (the second time from L2).
constexpr int kLongThreads = 512;
template <typename T, bool VEC>
__global__ void __launch_bounds__(kLongThreads) k_rowscale_quantize_long(const __grid_constant__ RowscaleArgs a) {
  __shared__ uint32_t red[kLongThreads / 32];
  const int64_t row = blockIdx.x;
  uint32_t most = 0u;
#pragma unroll 4
  for (int c = threadIdx.x * 8; c < a.cols; c += kLongThreads * 8) most = max(most, most8<T>(load8<T, VEC>(a.in, a.ld, a.cols, row, c)));
  most = __reduce_max_sync(0xFFFFFFFFu, most);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = most;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kLongThreads / 32; ++i) most = max(most, red[i]);
  const float inv = rowscale_inverse(most);
  const bool bad = rowscale_bad(most);
  if (threadIdx.x == 0) a.scales[row] = rowscale_of(most);
#pragma unroll 4
  for (int c = threadIdx.x * 8; c < a.cols; c += kLongThreads * 8) put8<T>(a, row, c, load8<T, VEC>(a.in, a.ld, a.cols, row, c), inv, bad);
}

// A warp (for short rows a part of one) a chunk of a row, V columns of the result a lane at a time: 16 bytes where the rows
// allow it, else 2 or 1.
constexpr int kBackThreads = 256, kBackPieces = 4;
template <typename T, int V>
__global__ void __launch_bounds__(kBackThreads) k_rowscale_dequantize(const __grid_constant__ RowscaleArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * (kBackThreads >> a.shift) + (threadIdx.x >> a.shift);
  const int64_t row = task / a.chunks;
  if (row >= a.rows) return;
  const int piece = V << a.shift, c0 = (int)(task - row * a.chunks) * piece * kBackPieces + (lane & ((1 << a.shift) - 1)) * V;
  const uint8_t* src = a.codes + row * a.pitch;
  T* dst = static_cast<T*>(a.out) + row * a.ld;
  const float s = __ldg(a.scales + row);
  uint32_t w[kBackPieces][(V + 3) / 4];
#pragma unroll
  for (int u = 0; u < kBackPieces; ++u) {   // (the last piece of a row may go past its columns where V is above 2)
    const int c = c0 + u * piece;
#pragma unroll
    for (int i = 0; i < (V + 3) / 4; ++i) w[u][i] = 0u;
    if (c + V <= a.cols) {
      if constexpr (V == 8) {
        const uint2 x = __ldg(reinterpret_cast<const uint2*>(src + c));
        w[u][0] = x.x, w[u][1] = x.y;
      } else if constexpr (V == 4) {
        w[u][0] = __ldg(reinterpret_cast<const uint32_t*>(src + c));
      } else if constexpr (V == 2) {
        w[u][0] = __ldg(reinterpret_cast<const uint16_t*>(src + c));
      } else {
        w[u][0] = __ldg(src + c);
      }
    } else if (V > 1) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < a.cols) w[u][i / 4] |= (uint32_t)__ldg(src + c + i) << (8 * (i & 3));
    }
  }
#pragma unroll
  for (int u = 0; u < kBackPieces; ++u) {
    const int c = c0 + u * piece;
    if (c >= a.cols) break;
    float v[(V + 3) / 4 * 4];
#pragma unroll
    for (int i = 0; i < (V + 3) / 4; ++i) {
      const float4 f = e4m3_values(w[u][i]);
      v[4 * i] = f.x * s, v[4 * i + 1] = f.y * s, v[4 * i + 2] = f.z * s, v[4 * i + 3] = f.w * s;
    }
    uint32_t h[4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4 && i < V; ++i) h[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < (V + 1) / 2; ++i) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        h[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
    }
    if (c + V <= a.cols) {
      if constexpr (V * sizeof(T) == 16) __stcs(reinterpret_cast<uint4*>(dst + c), make_uint4(h[0], h[1], h[2], h[3]));
      else if constexpr (V * sizeof(T) == 8) __stcs(reinterpret_cast<uint2*>(dst + c), make_uint2(h[0], h[1]));
      else if constexpr (V * sizeof(T) == 4) __stcs(reinterpret_cast<uint32_t*>(dst + c), h[0]);
      else *reinterpret_cast<uint16_t*>(dst + c) = (uint16_t)h[0];
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (c + i < a.cols) {
          if constexpr (sizeof(T) == 4) dst[c + i] = v[i];
          else dst[c + i] = __float2bfloat16_rn(v[i]);
        }
    }
  }
}

bool aligned_rows(const void* p, int64_t pitch_bytes, int rows, int to) {
  return reinterpret_cast<uintptr_t>(p) % to == 0 && (rows == 1 || pitch_bytes % to == 0);
}

template <typename T, bool VEC>
cudaError_t launch_quantize(const RowscaleArgs& a, cudaStream_t st) {
  const int64_t n = ((int64_t)a.cols + 7) / 8;
  const auto go = [&](auto kern, int threads, int rows) {
    kern<<<(unsigned)((a.rows + rows - 1) / rows), threads, 0, st>>>(a);
    return cudaGetLastError();
  };
  if (n <= 8) return go(k_rowscale_quantize<T, VEC, 8, 1>, 128, 16);
  if (n <= 16) return go(k_rowscale_quantize<T, VEC, 16, 1>, 128, 8);
  if (n <= 32) return go(k_rowscale_quantize<T, VEC, 32, 1>, 128, 4);
  if (n <= 128) return go(k_rowscale_quantize<T, VEC, 32, 4>, 128, 4);
  if (n <= 512) return go(k_rowscale_quantize<T, VEC, 128, 4>, 128, 1);
  if (n <= 1024) return go(k_rowscale_quantize<T, VEC, 256, 4>, 256, 1);
  if (n <= 2048) return go(k_rowscale_quantize<T, VEC, 512, 4>, 512, 1);
  return go(k_rowscale_quantize_long<T, VEC>, kLongThreads, 1);
}

int rowscale_check(const bitsmoe_rowscale* q, int type, int64_t ld) {
  if (!q || q->rows < 0 || q->cols < 1 || !dense_type_ok(type)) return BITSMOE_ERR_INVALID_ARG;
  if (q->rows > kMaxMicroRows || q->cols > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  if (q->ld < q->cols || ld < q->cols) return BITSMOE_ERR_INVALID_ARG;
  return BITSMOE_OK;
}
int rowscale_pointers(const bitsmoe_rowscale* q, const void* x, int type) {
  if (!x || !q->codes || !q->scales) return BITSMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(x) % dense_size(type) || reinterpret_cast<uintptr_t>(q->scales) % 4) return BITSMOE_ERR_ALIGNMENT;
  return BITSMOE_OK;
}

}  // namespace

extern "C" int bitsmoe_rowscale_quantize(const void* x, int type, int64_t ld, const bitsmoe_rowscale* q, void* stream) {
  int rc = rowscale_check(q, type, ld);
  if (rc || q->rows == 0) return rc;
  if ((rc = rowscale_pointers(q, x, type))) return rc;
  RowscaleArgs a{x, nullptr, ld, q->rows, q->cols, q->codes, q->ld, q->scales, aligned_rows(q->codes, q->ld, q->rows, 8), 0, 0};
  const bool vec = aligned_rows(x, ld * dense_size(type), q->rows, 16);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (type == BITSMOE_F32) e = vec ? launch_quantize<float, true>(a, st) : launch_quantize<float, false>(a, st);
  else e = vec ? launch_quantize<__nv_bfloat16, true>(a, st) : launch_quantize<__nv_bfloat16, false>(a, st);
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}

extern "C" int bitsmoe_rowscale_dequantize(const bitsmoe_rowscale* q, void* x, int type, int64_t ld, void* stream) {
  int rc = rowscale_check(q, type, ld);
  if (rc || q->rows == 0) return rc;
  if ((rc = rowscale_pointers(q, x, type))) return rc;
  RowscaleArgs a{nullptr, x, ld, q->rows, q->cols, q->codes, q->ld, q->scales, 0, 0, 0};
  // columns of a piece: 16 bytes of the result, or 2, where the rows of both start on such boundaries
  const int size = dense_size(type);
  const auto fits = [&](int v) { return aligned_rows(x, ld * size, q->rows, v * size) && aligned_rows(q->codes, q->ld, q->rows, v); };
  const int v = fits(16 / size) ? 16 / size : fits(2) ? 2 : 1;
  a.shift = 2;
  while (a.shift < 5 && (v << a.shift) * kBackPieces < q->cols) ++a.shift;
  const int per = (v << a.shift) * kBackPieces, tasks = kBackThreads >> a.shift;   // columns of a chunk, chunks of a block
  a.chunks = (q->cols + per - 1) / per;
  const int64_t blocks = ((int64_t)q->rows * a.chunks + tasks - 1) / tasks;
  if (blocks >= (1ll << 31)) return BITSMOE_ERR_SHAPE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const auto go = [&](auto kern) {
    kern<<<(unsigned)blocks, kBackThreads, 0, st>>>(a);
    return cudaGetLastError();
  };
  cudaError_t e;
  if (type == BITSMOE_F32) e = v == 4 ? go(k_rowscale_dequantize<float, 4>) : v == 2 ? go(k_rowscale_dequantize<float, 2>) : go(k_rowscale_dequantize<float, 1>);
  else
    e = v == 8   ? go(k_rowscale_dequantize<__nv_bfloat16, 8>)
        : v == 2 ? go(k_rowscale_dequantize<__nv_bfloat16, 2>)
                 : go(k_rowscale_dequantize<__nv_bfloat16, 1>);
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
