// Product of dense rows with a microscaled 4-bit matrix:
//
//   y[t][r] = s_w s_x sum_k W[r][k] x[t][k]
//   or, with a second matrix U of the same shape, SiLU(W x) * (U x)
//
// x in bf16, or itself microscaled.
#include "microscale.cuh"

#include <cuda_runtime.h>

namespace {
using namespace bmoe;

constexpr int kTR = 64, kTT = 64, kTK = 32;   // rows, tokens and columns of a tile
constexpr int kPThreads = 256;

struct MicroMat {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t pitch;
  int tiles;
};

struct ProductArgs {
  MicroMat w, u, xq;   // u.codes null: plain; xq.codes null: x is bf16
  const __nv_bfloat16* x;
  int64_t x_ld;
  int T, rows, cols, format;
  float sw, su;        // tensor scales (the coded activations' multiplied in)
  void* y;
  int y_type;
  int64_t y_ld;
};

// 32 columns of a row from column k (a multiple of 32), a quarter of them per call: 8 values.
__device__ __forceinline__ void decode8(const MicroMat& m, int format, int r, int rows, int k, int cols, float* dst) {
  if (r < rows && k < cols) {
    const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(m.codes + (int64_t)r * m.pitch + k / 2));
    const float s = micro_scale(format, m.scales[micro_scale_at(m.tiles, r, k / micro_block(format))]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = micro_value((w >> (4 * i)) & 15u) * s;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[i] = 0.f;
  }
}

__global__ void __launch_bounds__(kPThreads) k_micro_product(ProductArgs a) {
  __shared__ float ws[2][kTR][kTK + 1], xs[kTT][kTK + 1];
  const int r0 = blockIdx.x * kTR;
  const bool glu = a.u.codes != nullptr;
  const int tr = threadIdx.x & 15, tt = threadIdx.x >> 4;
  const int lr = threadIdx.x >> 2, lk = (threadIdx.x & 3) * 8;
  for (int t0 = blockIdx.y * kTT; t0 < a.T; t0 += gridDim.y * kTT) {
    float acc[2][4][4] = {};
    for (int k0 = 0; k0 < a.cols; k0 += kTK) {
      __syncthreads();
      decode8(a.w, a.format, r0 + lr, a.rows, k0 + lk, a.cols, &ws[0][lr][lk]);
      if (glu) decode8(a.u, a.format, r0 + lr, a.rows, k0 + lk, a.cols, &ws[1][lr][lk]);
      if (a.xq.codes) {
        decode8(a.xq, a.format, t0 + lr, a.T, k0 + lk, a.cols, &xs[lr][lk]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t = t0 + lr, k = k0 + lk + i;
          xs[lr][lk + i] = t < a.T && k < a.cols ? __bfloat162float(a.x[(int64_t)t * a.x_ld + k]) : 0.f;
        }
      }
      __syncthreads();
      for (int k = 0; k < kTK; ++k) {
        float xv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[j] = xs[tt * 4 + j][k];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float wv = ws[0][tr + 16 * i][k];
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[0][i][j] = fmaf(wv, xv[j], acc[0][i][j]);
        }
        if (glu) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float uv = ws[1][tr + 16 * i][k];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[1][i][j] = fmaf(uv, xv[j], acc[1][i][j]);
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = r0 + tr + 16 * i, t = t0 + tt * 4 + j;
        if (r >= a.rows || t >= a.T) continue;
        float v = acc[0][i][j] * a.sw;
        if (glu) v = v / (1.f + expf(-v)) * (acc[1][i][j] * a.su);
        if (a.y_type == BITSMOE_F32) static_cast<float*>(a.y)[(int64_t)t * a.y_ld + r] = v;
        else static_cast<__nv_bfloat16*>(a.y)[(int64_t)t * a.y_ld + r] = __float2bfloat16_rn(v);
      }
  }
}

MicroMat mat_of(const bitsmoe_microscale* m) {
  if (!m) return MicroMat{nullptr, nullptr, 0, 0};
  return MicroMat{m->codes, m->scales, micro_pitch(m->cols), micro_tiles(m->format, m->cols)};
}

}  // namespace

extern "C" int bitsmoe_microscale_product(const bitsmoe_microscale* w, const bitsmoe_microscale* up, const void* x,
                                          int64_t x_ld, const bitsmoe_microscale* xq, int T, void* y, int y_type,
                                          int64_t y_ld, int* status, void* stream) {
  int rc = micro_check(w);
  if (rc) return rc;
  if (up) {
    if ((rc = micro_check(up))) return rc;
    if (up->format != w->format) return BITSMOE_ERR_INVALID_ARG;
    if (up->rows != w->rows || up->cols != w->cols) return BITSMOE_ERR_SHAPE;
  }
  if (T < 0 || !dense_type_ok(y_type) || y_ld < w->rows || (x != nullptr && xq != nullptr)) return BITSMOE_ERR_INVALID_ARG;
  if (T > kMaxMicroRows) return BITSMOE_ERR_SHAPE;
  if (xq) {
    if ((rc = micro_check(xq))) return rc;
    if (xq->format != w->format) return BITSMOE_ERR_INVALID_ARG;
    if (xq->rows != T || xq->cols != w->cols) return BITSMOE_ERR_SHAPE;
  } else if (x_ld < w->cols) {
    return BITSMOE_ERR_INVALID_ARG;
  }
  if (T == 0 || w->rows == 0) return BITSMOE_OK;
  if ((!x && !xq) || !y) return BITSMOE_ERR_INVALID_ARG;
  if ((uintptr_t)x % 2 || (uintptr_t)y % dense_size(y_type) || (uintptr_t)status % 4) return BITSMOE_ERR_ALIGNMENT;
  const float sx = xq ? xq->scale : 1.f;
  ProductArgs a{mat_of(w), mat_of(up), mat_of(xq), static_cast<const __nv_bfloat16*>(x), x_ld, T, w->rows, w->cols,
                w->format, w->scale * sx, up ? up->scale * sx : 0.f, y, y_type, y_ld};
  const dim3 g((unsigned)((w->rows + kTR - 1) / kTR), (unsigned)((T + kTT - 1) / kTT < 65535 ? (T + kTT - 1) / kTT : 65535));
  k_micro_product<<<g, kPThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
  const cudaError_t r = cudaGetLastError();
  return r == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)r);
}
