// What stands between two blocks of a decoder, in one pass over each row:
//
//   n  = y rsqrt(mean(y^2) + eps_post) (o + g_post)     (or n = y: no post-norm)
//   h' = a h + b c[d] gate n                            (gate per token or per element, or its sigmoid)
//   x  = h' rsqrt(mean(h'^2) + eps_pre) (o + g_pre)     (the next block's input)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>

#include "device.cuh"

namespace {
using namespace bmoe;

__device__ __forceinline__ float load1(const void* p, int type, int64_t i) {
  if (type == BITSMOE_F32) return static_cast<const float*>(p)[i];
  return __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[i] << 16);
}
__device__ __forceinline__ void store1(void* p, int type, int64_t i, float v) {
  if (type == BITSMOE_F32) static_cast<float*>(p)[i] = v;
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

constexpr int kBThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* red) {
  v = warp_sum(v);
  __syncthreads();   // the previous sum has been read
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < kBThreads / 32; ++w) s += red[w];
  return s;
}

// One block per row; the row's h' stays in shared memory between the two norms.
__global__ void __launch_bounds__(kBThreads) k_block_norm(bitsmoe_block_norm_args a) {
  extern __shared__ float row[];   // [D]
  __shared__ float red[kBThreads / 32];
  const int64_t t = blockIdx.x;
  float inv = 1.f;
  if (a.y && a.post_norm) {
    float ss = 0.f;
    for (int d = threadIdx.x; d < a.D; d += kBThreads) {
      const float v = load1(a.y, a.y_type, t * a.y_ld + d);
      ss = fmaf(v, v, ss);
    }
    inv = rsqrtf(block_sum(ss, red) / (float)a.D + a.post_eps);
  }
  float tg = 1.f;
  if (a.gate_kind == BITSMOE_GATE_TOKEN) {
    tg = load1(a.gate, a.gate_type, t * a.gate_ld);
    if (a.gate_sigmoid) tg = 1.f / (1.f + expf(-tg));
  }
  float ss = 0.f;
  for (int d = threadIdx.x; d < a.D; d += kBThreads) {
    float v = a.residual_scale * load1(a.h, a.h_type, t * a.h_ld + d);
    if (a.y) {
      float n = load1(a.y, a.y_type, t * a.y_ld + d);
      if (a.post_norm) n *= inv * (a.post_gain ? a.gain_offset + load1(a.post_gain, a.gain_type, d) : 1.f);
      float g = tg;
      if (a.gate_kind == BITSMOE_GATE_ELEMENT) {
        g = load1(a.gate, a.gate_type, t * a.gate_ld + d);
        if (a.gate_sigmoid) g = 1.f / (1.f + expf(-g));
      }
      if (a.gate_kind) n *= g;
      if (a.channel_scale) n *= load1(a.channel_scale, a.gain_type, d);
      v = fmaf(a.branch_scale, n, v);
    }
    if (a.h_out) store1(a.h_out, a.h_type, t * a.h_out_ld + d, v);
    row[d] = v;
    ss = fmaf(v, v, ss);
  }
  if (!a.x) return;
  inv = rsqrtf(block_sum(ss, red) / (float)a.D + a.pre_eps);
  for (int d = threadIdx.x; d < a.D; d += kBThreads)
    store1(a.x, a.x_type, t * a.x_ld + d,
           row[d] * inv * (a.pre_gain ? a.gain_offset + load1(a.pre_gain, a.gain_type, d) : 1.f));
}

bool type_ok(int t) { return t == BITSMOE_F32 || t == BITSMOE_BF16; }
bool misaligned(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == BITSMOE_F32 ? 4 : 2) != 0; }

}  // namespace

extern "C" int bitsmoe_block_norm(const bitsmoe_block_norm_args* args, void* stream) {
  if (!args) return BITSMOE_ERR_INVALID_ARG;
  const bitsmoe_block_norm_args a = *args;
  if (a.T < 0 || a.D < 1) return BITSMOE_ERR_INVALID_ARG;
  if (a.D > BITSMOE_BLOCK_NORM_MAX_D || a.T > (1 << 24)) return BITSMOE_ERR_SHAPE;
  if (!type_ok(a.h_type) || !type_ok(a.y_type) || !type_ok(a.gate_type) || !type_ok(a.gain_type) || !type_ok(a.x_type))
    return BITSMOE_ERR_INVALID_ARG;
  if (a.gate_kind < BITSMOE_GATE_NONE || a.gate_kind > BITSMOE_GATE_ELEMENT) return BITSMOE_ERR_INVALID_ARG;
  if (!(a.post_eps >= 0.f) || !(a.pre_eps >= 0.f) || !std::isfinite(a.residual_scale) || !std::isfinite(a.branch_scale) ||
      !std::isfinite(a.gain_offset))
    return BITSMOE_ERR_INVALID_ARG;
  if ((!a.y && (a.post_norm || a.gate_kind || a.channel_scale)) || (a.post_gain && !a.post_norm)) return BITSMOE_ERR_INVALID_ARG;
  if (!a.x && a.pre_gain) return BITSMOE_ERR_INVALID_ARG;
  if (a.T == 0) return BITSMOE_OK;
  if (!a.h || (!a.h_out && !a.x) || (a.gate_kind && !a.gate)) return BITSMOE_ERR_INVALID_ARG;
  if (a.h_ld < a.D || (a.y && a.y_ld < a.D) || (a.h_out && a.h_out_ld < a.D) || (a.x && a.x_ld < a.D) ||
      (a.gate_kind == BITSMOE_GATE_TOKEN && a.gate_ld < 1) || (a.gate_kind == BITSMOE_GATE_ELEMENT && a.gate_ld < a.D))
    return BITSMOE_ERR_INVALID_ARG;
  if (misaligned(a.h, a.h_type) || misaligned(a.y, a.y_type) || misaligned(a.gate, a.gate_type) ||
      misaligned(a.post_gain, a.gain_type) || misaligned(a.pre_gain, a.gain_type) ||
      misaligned(a.channel_scale, a.gain_type) || misaligned(a.h_out, a.h_type) || misaligned(a.x, a.x_type))
    return BITSMOE_ERR_ALIGNMENT;
  const size_t smem = (size_t)a.D * 4;
  cudaError_t e = cudaSuccess;
  if (smem > 40 * 1024)   // 48 KB with the static part need no opt-in
    e = cudaFuncSetAttribute(k_block_norm, cudaFuncAttributeMaxDynamicSharedMemorySize, BITSMOE_BLOCK_NORM_MAX_D * 4);
  if (e == cudaSuccess) {
    k_block_norm<<<(unsigned)a.T, kBThreads, smem, static_cast<cudaStream_t>(stream)>>>(a);
    e = cudaGetLastError();
  }
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
