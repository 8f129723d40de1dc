// Products grouped by expert, ragged: for offsets[e] <= p < offsets[e + 1]
//
//   y[p][r] = sum_k W_e[r][k] x[q][k]        (q = p, or index[p] / fan)
//   or, with a second set of matrices U, SiLU(W_e x) * (U_e x)
//
// in bf16, or in 8 bits (E4M3) with a scale a row on both sides, which multiplies the finished sum.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "microscale.cuh"
#include "rows.cuh"

namespace {
using namespace bmoe;

constexpr int kMaxExperts = 1024;

struct ExpertArgs {
  int E, P, rows, cols, x_rows, fan;
  int N, mt;             // rows of y and tiles of the matrices' rows of a tile of work
  const int32_t* offsets;
  const int32_t* index;
  const void* w;
  const void* up;
  const float* ws;
  const float* us;
  int64_t w_ld, w_eld, w_sld, u_ld, u_eld, u_sld;
  const void* x;
  const float* xs;
  int64_t x_ld;
  void* y;
  int y_type;
  int64_t y_ld;
  long long spin;
  int lose;
  int* status;
};

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + expf(-g)) * u; }

__device__ __forceinline__ void store_y(void* y, int type, int64_t i, float v) {
  if (type == BITSMOE_F32) static_cast<float*>(y)[i] = v;
  else static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
}

// ---------------------------------------------------------------------------
// The groups in shared memory: first[e] the first row of expert e (of y), tiles[e] the tiles of N rows before it, and
// both past the last one.  Offsets are held between 0 and P, so that whatever they are no row of y lies outside.
// ---------------------------------------------------------------------------
struct Groups {
  int first[kMaxExperts + 1];
  int count[kMaxExperts];
  int tiles[kMaxExperts + 1];
  int part[33];
};

template <int THREADS>
__device__ __forceinline__ void read_groups(const ExpertArgs& a, Groups& s) {
  constexpr int W = THREADS / 32;
  const int tid = threadIdx.x, lane = tid & 31;
  int before = 0;   // tiles of the experts of the rounds before
  for (int e0 = 0; e0 < a.E; e0 += THREADS) {
    const int e = e0 + tid;
    int lo = 0, n = 0;
    if (e < a.E) {
      lo = min(max(__ldg(a.offsets + e), 0), a.P);
      n = max(min(max(__ldg(a.offsets + e + 1), 0), a.P) - lo, 0);
    }
    const int t = (n + a.N - 1) / a.N;
    int sum = t;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
      if (lane >= o) sum += v;
    }
    if (lane == 31) s.part[tid >> 5] = sum;
    __syncthreads();
    int base = before;
    for (int i = 0; i < W; ++i) {
      const int v = s.part[i];
      if (i < (tid >> 5)) base += v;
      before += v;
    }
    if (e < a.E) {
      s.first[e] = lo;
      s.count[e] = n;
      s.tiles[e] = base + sum - t;
      if (e == a.E - 1) s.tiles[a.E] = base + sum;
    }
    __syncthreads();
  }
}

// A tile of work: rows m0 .. of the matrices of expert e, n rows of y from p0 on.  An expert's rows are shared evenly
// among its tiles.
struct Tile {
  int e, m, p0, n;
};
__device__ __forceinline__ Tile tile_of(const ExpertArgs& a, const Groups& s, int tile, int unit) {
  const int q = tile / a.mt;
  int lo = 0, hi = a.E;   // tiles[lo] <= q < tiles[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.tiles[mid] <= q) lo = mid;
    else hi = mid;
  }
  const int i = q - s.tiles[lo], tt = s.tiles[lo + 1] - s.tiles[lo], n = s.count[lo];
  const int per = ((n + tt - 1) / tt + unit - 1) / unit * unit;
  return Tile{lo, tile - q * a.mt, s.first[lo] + i * per, min(per, n - i * per)};
}

// Row of x of row p of y, or -1.
__device__ __forceinline__ int row_of(const ExpertArgs& a, int p) {
  int q = p;
  if (a.index) {
    q = __ldg(a.index + p);
    q = q < 0 ? -1 : a.fan == 1 ? q : q / a.fan;
  }
  return q < a.x_rows ? q : -1;
}

// ---------------------------------------------------------------------------
// Rows on any boundary: tiles of 64 x 64 by fp32 instructions.
// ---------------------------------------------------------------------------
constexpr int kPlainThreads = 256, kPlainTile = 64, kPlainK = 16;

template <bool F8>
__device__ __forceinline__ float element_at(const void* p, int64_t i) {
  if constexpr (F8) return e4m3_values((uint32_t)__ldg(static_cast<const uint8_t*>(p) + i)).x;
  else return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(p) + i) << 16);
}

template <bool F8, bool GLU>
__global__ void __launch_bounds__(kPlainThreads) k_expert_plain(const __grid_constant__ ExpertArgs a) {
  constexpr int NA = GLU ? 2 : 1;
  __shared__ Groups s;
  __shared__ __align__(16) float xt[kPlainK][kPlainTile + 4], wt[NA][kPlainK][kPlainTile + 4];
  read_groups<kPlainThreads>(a, s);
  const int tid = threadIdx.x, lr = tid >> 2, lk = (tid & 3) * 4;   // what a thread brings: 4 columns of a row
  const int tr = (tid & 15) * 4, tp = (tid >> 4) * 4;               // what it sums: 4 rows of the matrix x 4 of y
  const int ntiles = s.tiles[a.E] * a.mt;
  for (int tile = blockIdx.x; tile < ntiles; tile += gridDim.x) {
    const Tile t = tile_of(a, s, tile, 1);
    const int m = t.m * kPlainTile + lr, q = lr < t.n ? row_of(a, t.p0 + lr) : -1;
    float acc[NA][4][4];
#pragma unroll
    for (int i = 0; i < NA * 16; ++i) (&acc[0][0][0])[i] = 0.f;
    for (int k0 = 0; k0 < a.cols; k0 += kPlainK) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = k0 + lk + i;
        xt[lk + i][lr] = q >= 0 && k < a.cols ? element_at<F8>(a.x, q * a.x_ld + k) : 0.f;
        wt[0][lk + i][lr] = m < a.rows && k < a.cols ? element_at<F8>(a.w, t.e * a.w_eld + m * a.w_ld + k) : 0.f;
        if constexpr (GLU) wt[NA - 1][lk + i][lr] = m < a.rows && k < a.cols ? element_at<F8>(a.up, t.e * a.u_eld + m * a.u_ld + k) : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kPlainK; ++k) {
        const float4 xv = *reinterpret_cast<const float4*>(&xt[k][tp]);
        const float xa[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
        for (int b = 0; b < NA; ++b) {
          const float4 wv = *reinterpret_cast<const float4*>(&wt[b][k][tr]);
          const float wa[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[b][i][j] = fmaf(xa[i], wa[j], acc[b][i][j]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (tp + i >= t.n) continue;
      const int64_t p = t.p0 + tp + i;
      const int row = row_of(a, (int)p);
      const float f = row < 0 ? __uint_as_float(0x7FC00000u) : F8 ? __ldg(a.xs + row) : 1.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = t.m * kPlainTile + tr + j;
        if (r >= a.rows) continue;
        float v = acc[0][i][j] * f;
        if (F8) v *= __ldg(a.ws + t.e * a.w_sld + r);
        if constexpr (GLU) {
          float u = acc[NA - 1][i][j] * f;
          if (F8) u *= __ldg(a.us + t.e * a.u_sld + r);
          v = silu_mul(v, u);
        }
        store_y(a.y, a.y_type, p * a.y_ld + r, v);
      }
    }
  }
}

template <bool F8>
cudaError_t launch_plain(ExpertArgs a, int sms, cudaStream_t st) {
  a.N = kPlainTile;
  a.mt = (a.rows + kPlainTile - 1) / kPlainTile;
  const int64_t most = (int64_t)std::min<int64_t>(a.P, (int64_t)a.P / a.N + a.E) * a.mt;
  const unsigned blocks = (unsigned)std::min<int64_t>(most, (int64_t)sms * 4);
  if (a.up) k_expert_plain<F8, true><<<blocks, kPlainThreads, 0, st>>>(a);
  else k_expert_plain<F8, false><<<blocks, kPlainThreads, 0, st>>>(a);
  return cudaGetLastError();
}

int matrices_check(const bitsmoe_expert_matrices* m) {
  if (!m || (m->type != BITSMOE_BF16 && m->type != BITSMOE_E4M3) || m->experts < 1 || m->rows < 0 || m->cols < 1) return BITSMOE_ERR_INVALID_ARG;
  if (m->experts > kMaxExperts || m->rows > kMaxMicroCols || m->cols > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  if (m->ld < m->cols || (m->experts > 1 && m->expert_ld < 0) || (m->type == BITSMOE_E4M3 && m->experts > 1 && m->scale_ld < 0)) return BITSMOE_ERR_INVALID_ARG;
  return BITSMOE_OK;
}
int matrices_pointers(const bitsmoe_expert_matrices* m) {
  if (!m->data || (m->type == BITSMOE_E4M3 && !m->scales)) return BITSMOE_ERR_INVALID_ARG;
  if ((m->type == BITSMOE_BF16 && reinterpret_cast<uintptr_t>(m->data) % 2) || reinterpret_cast<uintptr_t>(m->scales) % 4) return BITSMOE_ERR_ALIGNMENT;
  return BITSMOE_OK;
}

}  // namespace

extern "C" int bitsmoe_expert_product(const bitsmoe_expert_product_args* args, void* stream) {
  if (!args) return BITSMOE_ERR_INVALID_ARG;
  const bitsmoe_expert_product_args& g = *args;
  int rc = matrices_check(g.w);
  if (rc) return rc;
  if (g.up) {
    if ((rc = matrices_check(g.up))) return rc;
    if (g.up->type != g.w->type) return BITSMOE_ERR_INVALID_ARG;
    if (g.up->experts != g.w->experts || g.up->rows != g.w->rows || g.up->cols != g.w->cols) return BITSMOE_ERR_SHAPE;
  }
  if (g.P < 0 || g.x_rows < 0 || g.fan < 1 || !dense_type_ok(g.y_type) || g.x_ld < g.w->cols || g.y_ld < g.w->rows) return BITSMOE_ERR_INVALID_ARG;
  if (g.P > kMaxMicroRows || g.x_rows > kMaxMicroRows) return BITSMOE_ERR_SHAPE;
  if ((((int64_t)g.P + 15) / 16 + g.w->experts) * ((g.w->rows + 63) / 64) >= (1ll << 31)) return BITSMOE_ERR_SHAPE;
  if (g.P == 0 || g.w->rows == 0) return BITSMOE_OK;
  const bool f8 = g.w->type == BITSMOE_E4M3;
  if ((rc = matrices_pointers(g.w)) || (g.up && (rc = matrices_pointers(g.up)))) return rc;
  if ((!g.x && g.x_rows > 0) || !g.offsets || !g.y || (f8 && !g.x_scales && g.x_rows > 0)) return BITSMOE_ERR_INVALID_ARG;
  const auto odd = [](const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (odd(g.x, f8 ? 1 : 2) || odd(g.x_scales, 4) || odd(g.offsets, 4) || odd(g.index, 4) || odd(g.y, dense_size(g.y_type)) || odd(g.status, 4))
    return BITSMOE_ERR_ALIGNMENT;
  int dev = 0, sms = 0;
  cudaError_t e = device_sms(&dev, &sms);
  if (e != cudaSuccess) return record_cuda_error((int)e);
  ExpertArgs a;
  std::memset(&a, 0, sizeof(a));
  a.E = g.w->experts;
  a.P = g.P;
  a.rows = g.w->rows;
  a.cols = g.w->cols;
  a.x_rows = g.x_rows;
  a.fan = g.fan;
  a.offsets = g.offsets;
  a.index = g.index;
  a.w = g.w->data;
  a.ws = g.w->scales;
  a.w_ld = g.w->ld;
  a.w_eld = g.w->expert_ld;
  a.w_sld = g.w->scale_ld;
  if (g.up) {
    a.up = g.up->data;
    a.us = g.up->scales;
    a.u_ld = g.up->ld;
    a.u_eld = g.up->expert_ld;
    a.u_sld = g.up->scale_ld;
  }
  a.x = g.x;
  a.xs = g.x_scales;
  a.x_ld = g.x_ld;
  a.y = g.y;
  a.y_type = g.y_type;
  a.y_ld = g.y_ld;
  a.spin = debug_wait_clocks() > 0 ? debug_wait_clocks() : kWaitClocks;
  a.lose = debug_skip_arrival();
  a.status = g.status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  e = f8 ? launch_plain<true>(a, sms, st) : launch_plain<false>(a, sms, st);
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
