// What stands between two blocks of a decoder, in one pass over each row:
//
//   n  = y rsqrt(mean(y^2) + eps_post) (o + g_post)     (or n = y: no post-norm)
//   h' = a h + b c[d] gate n                            (gate per token or per element, or its sigmoid)
//   x  = h' rsqrt(mean(h'^2) + eps_pre) (o + g_pre)     (the next block's input; in 8 bits: its codes and a scale a row)
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "microscale.cuh"
#include "rows.cuh"

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

// ---------------------------------------------------------------------------
// A row per group of threads (a warp for rows of up to 256, else a block), the whole
// row in registers: the block's output, its gate and the residual are requested
// together and read once.  Two sums over the group (of the output's and of h's
// squares) are all that it waits for.  VEC elements a load: 8 where every row starts
// on a 16-byte boundary, 2 or 1 otherwise (rows of up to 256; longer ones go through
// the ring).  DRAM bounds it from some thousand rows on:
// 16384 rows of 4096 (fp32, post- and pre-norm) 165 us, 5.7 TB/s; with the rows
// requested into registers instead of the ring of k_block_norm_rows 198 us, without
// requesting ahead 259 us.  One row of 2048: 2.8 us.
// ---------------------------------------------------------------------------
template <int VEC>
struct Raw {          // VEC elements as they are stored: fp32 in w[0 .. VEC), bf16 in w[0 .. (VEC + 1) / 2)
  uint32_t w[VEC];
};

template <int VEC>
__device__ __forceinline__ Raw<VEC> load_raw(const void* p, int type, int64_t i) {
  Raw<VEC> r;
  if (type == BITSMOE_F32) {
    const float* q = static_cast<const float*>(p) + i;
    if constexpr (VEC == 8) {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(q)), b = __ldg(reinterpret_cast<const uint4*>(q) + 1);
      r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w, r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
    } else if constexpr (VEC == 2) {
      const uint2 a = __ldg(reinterpret_cast<const uint2*>(q));
      r.w[0] = a.x, r.w[1] = a.y;
    } else {
      r.w[0] = __ldg(reinterpret_cast<const uint32_t*>(q));
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + i;
    if constexpr (VEC == 8) {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(q));
      r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
    } else if constexpr (VEC == 2) {
      r.w[0] = __ldg(reinterpret_cast<const uint32_t*>(q));
    } else {
      r.w[0] = __ldg(q);
    }
  }
  return r;
}
// The same of memory that this kernel writes (h, where h_out is h).
template <int VEC>
__device__ __forceinline__ Raw<VEC> load_own(const void* p, int type, int64_t i) {
  Raw<VEC> r;
  if (type == BITSMOE_F32) {
    const float* q = static_cast<const float*>(p) + i;
    if constexpr (VEC == 8) {
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(q)), b = __ldcs(reinterpret_cast<const uint4*>(q) + 1);
      r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w, r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
    } else if constexpr (VEC == 2) {
      const uint2 a = __ldcs(reinterpret_cast<const uint2*>(q));
      r.w[0] = a.x, r.w[1] = a.y;
    } else {
      r.w[0] = __ldcs(reinterpret_cast<const uint32_t*>(q));
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + i;
    if constexpr (VEC == 8) {
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(q));
      r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
    } else if constexpr (VEC == 2) {
      r.w[0] = __ldcs(reinterpret_cast<const uint32_t*>(q));
    } else {
      r.w[0] = __ldcs(q);
    }
  }
  return r;
}
// VEC elements of a row in shared memory (filled by a bulk copy).
template <int VEC>
__device__ __forceinline__ Raw<VEC> load_shared(const uint8_t* p, int type, int i) {
  Raw<VEC> r;
  if constexpr (VEC == 8) {
    const uint4 a = lds128(p + (type == BITSMOE_F32 ? 4 : 2) * i);
    r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
    if (type == BITSMOE_F32) {
      const uint4 b = lds128(p + 4 * i + 16);
      r.w[4] = b.x, r.w[5] = b.y, r.w[6] = b.z, r.w[7] = b.w;
    }
  } else {
    static_assert(VEC == 1, "");
    if (type == BITSMOE_F32) r.w[0] = *reinterpret_cast<const uint32_t*>(p + 4 * i);
    else r.w[0] = *reinterpret_cast<const uint16_t*>(p + 2 * i);
  }
  return r;
}
template <int VEC>
__device__ __forceinline__ void unpack(const Raw<VEC>& r, int type, float (&v)[VEC]) {
  if (type == BITSMOE_F32) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = __uint_as_float(r.w[e]);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = e & 1 ? bf16hi(r.w[e / 2]) : bf16lo(r.w[e / 2]);
  }
}
template <int VEC>
__device__ __forceinline__ void store_vec(void* p, int type, int64_t i, const float (&v)[VEC]) {
  if (type == BITSMOE_F32) {
    float* q = static_cast<float*>(p) + i;
    if constexpr (VEC == 8) {
      __stcs(reinterpret_cast<float4*>(q), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(q) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else if constexpr (VEC == 2) {
      *reinterpret_cast<float2*>(q) = make_float2(v[0], v[1]);
    } else {
      *q = v[0];
    }
  } else {
    uint16_t* q = static_cast<uint16_t*>(p) + i;
    if constexpr (VEC == 1) {
      *q = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
      uint32_t h[VEC / 2];
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        h[e] = *reinterpret_cast<const uint32_t*>(&b);
      }
      if constexpr (VEC == 8) *reinterpret_cast<uint4*>(q) = make_uint4(h[0], h[1], h[2], h[3]);
      else *reinterpret_cast<uint32_t*>(q) = h[0];
    }
  }
}

constexpr int kRowThreads = 512, kRowWarps = kRowThreads / 32;

// Sum over a block of at most WARPS warps, in one order whatever their number; `red` holds zeros past them
// and is this sum's own buffer (the two sums of a row take turns).
template <int WARPS = kRowWarps>
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = warp_sum(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int q = 0; q < WARPS / 4; ++q) {
    const float4 p = reinterpret_cast<const float4*>(red)[q];
    s += (p.x + p.y) + (p.z + p.w);
  }
  return s;
}

// The largest of a block's values (bits of magnitudes), as block_sum.
template <int WARPS = kRowWarps>
__device__ __forceinline__ uint32_t block_most(uint32_t v, uint32_t* red) {
  v = __reduce_max_sync(0xFFFFFFFFu, v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  uint32_t m = 0u;
#pragma unroll
  for (int q = 0; q < WARPS / 4; ++q) {
    const uint4 p = reinterpret_cast<const uint4*>(red)[q];
    m = max(m, max(max(p.x, p.y), max(p.z, p.w)));
  }
  return m;
}
template <int VEC>
__device__ __forceinline__ uint32_t most_of(const float (&v)[VEC]) {
  uint32_t m = 0u;
#pragma unroll
  for (int q = 0; q < VEC; ++q) m = max(m, __float_as_uint(v[q]) & 0x7FFFFFFFu);
  return m;
}
// Codes of elements i .. of a row in 8 bits.
template <int VEC>
__device__ __forceinline__ void store_codes(void* x, int64_t i, const float (&v)[VEC], float inv, bool bad) {
  uint8_t* p = static_cast<uint8_t*>(x) + i;
  if constexpr (VEC == 8) {
    const uint2 w = make_uint2(e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    *reinterpret_cast<uint2*>(p) = bad ? make_uint2(0u, 0u) : w;
  } else if constexpr (VEC == 2) {
    *reinterpret_cast<uint16_t*>(p) = bad ? (uint16_t)0 : (uint16_t)e4m3x2(v[0] * inv, v[1] * inv);
  } else {
    *p = bad ? (uint8_t)0 : (uint8_t)e4m3x2(v[0] * inv, 0.f);
  }
}

__device__ __forceinline__ float sigmoid(float v) { return 1.f / (1.f + expf(-v)); }

// What multiplies a normalised output: branch_scale * channel_scale * (offset + post_gain).
template <int VEC>
__device__ __forceinline__ void branch_factor(const bitsmoe_block_norm_args& a, const Raw<VEC>& post, const Raw<VEC>& chan, float (&c)[VEC]) {
  float v[VEC];
#pragma unroll
  for (int q = 0; q < VEC; ++q) c[q] = a.branch_scale;
  if (a.channel_scale) {
    unpack<VEC>(chan, a.gain_type, v);
#pragma unroll
    for (int q = 0; q < VEC; ++q) c[q] *= v[q];
  }
  if (a.post_gain) {
    unpack<VEC>(post, a.gain_type, v);
#pragma unroll
    for (int q = 0; q < VEC; ++q) c[q] *= a.gain_offset + v[q];
  }
}
template <int VEC>
__device__ __forceinline__ void pre_factor(const bitsmoe_block_norm_args& a, const Raw<VEC>& pre, float (&c)[VEC]) {
#pragma unroll
  for (int q = 0; q < VEC; ++q) c[q] = 1.f;
  if (a.pre_gain) {
    unpack<VEC>(pre, a.gain_type, c);
#pragma unroll
    for (int q = 0; q < VEC; ++q) c[q] += a.gain_offset;
  }
}

// One row a group.  Threads at VEC * (k * group + i) hold vector k of a row; k < NV.  Latency counts: the gains are
// requested with the row where the registers hold them.  Q: x in 8 bits, its scale from one more maximum over the group.
template <int VEC, int NV, bool WARP, bool Q>
__global__ void __launch_bounds__(WARP ? 128 : kRowThreads, WARP ? 4 : NV * VEC > 8 ? 1 : 2)
    k_block_norm(const __grid_constant__ bitsmoe_block_norm_args a, float* x_scale) {
  __shared__ __align__(16) float red[2][kRowWarps];
  __shared__ __align__(16) uint32_t redm[kRowWarps];
  const int gsize = WARP ? 32 : blockDim.x, gi = WARP ? (threadIdx.x & 31) : threadIdx.x;
  const int64_t t = WARP ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (t >= a.T) return;   // (whole groups)
  if (!WARP && threadIdx.x < 2 * kRowWarps) red[threadIdx.x / kRowWarps][threadIdx.x % kRowWarps] = 0.f;
  if (Q && !WARP && threadIdx.x < kRowWarps) redm[threadIdx.x] = 0u;
  const auto sum = [&](float v, int which) { return WARP ? warp_sum(v) : block_sum(v, red[which]); };
  int at[NV];
  bool in[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    at[k] = (k * gsize + gi) * VEC;
    in[k] = at[k] < a.D;   // a vector lies inside the row or outside: D is a multiple of VEC
  }
  const bool elem = a.gate_kind == BITSMOE_GATE_ELEMENT;
  constexpr bool kEarly = NV * VEC <= 16;   // what the registers hold
  Raw<VEC> y[NV], h[NV], e[NV], post[NV], pre[NV], chan[NV];
  const auto gain = [&](Raw<VEC>& r, const void* p, int k) {
    if (p && in[k]) r = load_raw<VEC>(p, a.gain_type, at[k]);
  };
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (in[k]) {
      if (a.y) y[k] = load_raw<VEC>(a.y, a.y_type, t * a.y_ld + at[k]);
      h[k] = load_own<VEC>(a.h, a.h_type, t * a.h_ld + at[k]);
      if (elem && kEarly) e[k] = load_raw<VEC>(a.gate, a.gate_type, t * a.gate_ld + at[k]);
    }
  float g = 1.f;
  if (a.gate_kind == BITSMOE_GATE_TOKEN) g = load1(a.gate, a.gate_type, t * a.gate_ld);
  if (!WARP) __syncthreads();   // red is cleared
  const float inv_d = 1.f / (float)a.D;
  float inv = 1.f;
  float v[NV][VEC], c[VEC];
  if (kEarly)
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      gain(post[k], a.post_gain, k);
      gain(chan[k], a.channel_scale, k);
      gain(pre[k], a.pre_gain, k);
    }
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int q = 0; q < VEC; ++q) v[k][q] = 0.f;
  if (a.y) {
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in[k]) {
        unpack<VEC>(y[k], a.y_type, v[k]);
#pragma unroll
        for (int q = 0; q < VEC; ++q) ss = fmaf(v[k][q], v[k][q], ss);
      }
    if (a.post_norm) inv = rsqrtf(sum(ss, 0) * inv_d + a.post_eps);
  }
  if (a.gate_kind == BITSMOE_GATE_TOKEN && a.gate_sigmoid) g = sigmoid(g);
  float ss = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (in[k]) {
      if (a.y) {
        if (!kEarly) {
          gain(post[k], a.post_gain, k);
          gain(chan[k], a.channel_scale, k);
        }
        branch_factor<VEC>(a, post[k], chan[k], c);
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[k][q] = v[k][q] * inv * c[q];
        if (elem) {
          if (!kEarly) e[k] = load_raw<VEC>(a.gate, a.gate_type, t * a.gate_ld + at[k]);
          unpack<VEC>(e[k], a.gate_type, c);
#pragma unroll
          for (int q = 0; q < VEC; ++q) v[k][q] *= a.gate_sigmoid ? sigmoid(c[q]) : c[q];
        } else if (a.gate_kind) {
#pragma unroll
          for (int q = 0; q < VEC; ++q) v[k][q] *= g;
        }
      }
      unpack<VEC>(h[k], a.h_type, c);
#pragma unroll
      for (int q = 0; q < VEC; ++q) {
        v[k][q] = fmaf(a.residual_scale, c[q], v[k][q]);
        ss = fmaf(v[k][q], v[k][q], ss);
      }
    }
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (in[k] && a.h_out) store_vec<VEC>(a.h_out, a.h_type, t * a.h_out_ld + at[k], v[k]);
  if (!a.x) return;
  inv = rsqrtf(sum(ss, 1) * inv_d + a.pre_eps);
  uint32_t most = 0u;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (in[k]) {
      if (!kEarly) gain(pre[k], a.pre_gain, k);
      pre_factor<VEC>(a, pre[k], c);
#pragma unroll
      for (int q = 0; q < VEC; ++q) v[k][q] = v[k][q] * inv * c[q];
      if constexpr (Q) most = max(most, most_of<VEC>(v[k]));
      else store_vec<VEC>(a.x, a.x_type, t * a.x_ld + at[k], v[k]);
    }
  if constexpr (Q) {
    most = WARP ? __reduce_max_sync(0xFFFFFFFFu, most) : block_most(most, redm);
    if (gi == 0) x_scale[t] = rowscale_of(most);
#pragma unroll
    for (int k = 0; k < NV; ++k)
      if (in[k]) store_codes<VEC>(a.x, t * a.x_ld + at[k], v[k], rowscale_inverse(most), rowscale_bad(most));
  }
}

__device__ __forceinline__ void copy1(uint8_t* dst, const uint8_t* src, uint32_t size) {   // an element
  if (size == 4) *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const volatile uint32_t*>(src);
  else *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const volatile uint16_t*>(src);
}

// Blocks that stay, whose rows come ahead by bulk copies into a ring of slots in shared memory; the factors of a
// thread's columns stay in its registers.  VEC 8: many rows on 16-byte boundaries; the same operations in the same
// order as above, so a row's result does not depend on how many there are that are read so.  (A row alone has no pitch:
// at an aligned address it is read by eights also where its batch is not, and its sums then take another order.)
// VEC 1: rows of more than 256 elements off those boundaries, however many.  The copies take the aligned 16 bytes at
// both ends whole (they hold elements of the row, so they can be read; the others are not used).  16384 rows of 4095:
// fp32 162 us (5.8 TB/s), bf16 169 (bound by what it issues, an element at a time); element by element from global
// memory 737 and 691.
constexpr int kMaxSlots = 8;

template <int VEC, int NV, int TH, int HT, int YT, bool Q>   // TH: threads at most; Q: x in 8 bits
__global__ void __launch_bounds__(TH, VEC * NV * TH <= 8 * kRowThreads ? 2 : 1)
    k_block_norm_rows(const __grid_constant__ bitsmoe_block_norm_args a, int slots, float* x_scale) {
  extern __shared__ __align__(128) uint8_t ring[];
  constexpr int kW = TH / 32;
  __shared__ __align__(16) float red[2][kW];
  __shared__ __align__(16) uint32_t redm[kW];   // (read behind a barrier, and written again behind the next row's sum)
  __shared__ uint64_t full[kMaxSlots];
  constexpr uint32_t hs = HT == BITSMOE_F32 ? 4 : 2, ys = YT == BITSMOE_F32 ? 4 : 2;
  const uint32_t es = a.gate_type == BITSMOE_F32 ? 4 : 2;
  const bool elem = a.gate_kind == BITSMOE_GATE_ELEMENT;
  // a slot: y's row, h's, the gate's
  const auto room = [&](uint32_t bytes) { return VEC == 8 ? bytes : (bytes + 15) / 16 * 16 + 16; };
  const uint32_t yb = a.y ? room(a.D * ys) : 0u, hb = room(a.D * hs), eb = elem ? room(a.D * es) : 0u;
  const auto row_at = [](const void* p, int64_t element, uint32_t size) { return static_cast<const uint8_t*>(p) + element * size; };
  const auto off = [](const uint8_t* p) { return VEC == 8 ? 0u : (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15); };
  if (threadIdx.x < 2 * kW) red[threadIdx.x / kW][threadIdx.x % kW] = 0.f;
  if (Q && threadIdx.x < kW) redm[threadIdx.x] = 0u;
  const auto fill = [&](int slot, int64_t row) {   // by one thread
    uint8_t* dst = ring + (size_t)slot * (yb + hb + eb);
    const uint8_t *py = row_at(a.y, row * a.y_ld, ys), *ph = row_at(a.h, row * a.h_ld, hs), *pe = row_at(a.gate, row * a.gate_ld, es);
    const auto bytes = [&](const uint8_t* p, uint32_t size) { return VEC == 8 ? a.D * size : (off(p) + a.D * size + 15) / 16 * 16; };
    const uint32_t ny = yb ? bytes(py, ys) : 0u, nh = bytes(ph, hs), ne = eb ? bytes(pe, es) : 0u;
    mbar_expect_tx(full + slot, ny + nh + ne);
    if (yb) bulk_g2s(dst, py - off(py), ny, full + slot);
    bulk_g2s(dst + yb, ph - off(ph), nh, full + slot);
    if (eb) bulk_g2s(dst + yb + hb, pe - off(pe), ne, full + slot);
  };
  int64_t t = blockIdx.x;
  if (threadIdx.x == 0) {
    for (int i = 0; i < slots; ++i) mbar_init(full + i);
    for (int i = 0; i < slots && t + (int64_t)i * gridDim.x < a.T; ++i) fill(i, t + (int64_t)i * gridDim.x);
  }
  int at[NV];
  bool in[NV];
  float cb[NV][VEC], cp[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    at[k] = (k * blockDim.x + threadIdx.x) * VEC;
    in[k] = at[k] < a.D;
    Raw<VEC> post, chan, pre;
    if (in[k]) {
      if (a.post_gain) post = load_raw<VEC>(a.post_gain, a.gain_type, at[k]);
      if (a.channel_scale) chan = load_raw<VEC>(a.channel_scale, a.gain_type, at[k]);
      if (a.pre_gain) pre = load_raw<VEC>(a.pre_gain, a.gain_type, at[k]);
      branch_factor<VEC>(a, post, chan, cb[k]);
      pre_factor<VEC>(a, pre, cp[k]);
    } else {
#pragma unroll
      for (int q = 0; q < VEC; ++q) cb[k][q] = cp[k][q] = 0.f;
    }
  }
  __syncthreads();
  const float inv_d = 1.f / (float)a.D;
  int slot = 0, use = 0;
  for (; t < a.T; t += gridDim.x) {
    // (after a wait that ran out a thread fetches its own elements)
    const bool here = mbar_wait(full + slot, (uint32_t)use & 1u);
    uint8_t* src = ring + (size_t)slot * (yb + hb + eb);
    uint8_t* sy = src + off(row_at(a.y, t * a.y_ld, ys));
    uint8_t* sh = src + yb + off(row_at(a.h, t * a.h_ld, hs));
    uint8_t* se = src + yb + hb + off(row_at(a.gate, t * a.gate_ld, es));
    if (!here) {
#pragma unroll 1
      for (int n = 0; n < NV * VEC; ++n) {
        const int d = (n / VEC * blockDim.x + threadIdx.x) * VEC + n % VEC;
        if (d < a.D) {
          if (yb) copy1(sy + d * ys, row_at(a.y, t * a.y_ld + d, ys), ys);
          copy1(sh + d * hs, row_at(a.h, t * a.h_ld + d, hs), hs);
          if (eb) copy1(se + d * es, row_at(a.gate, t * a.gate_ld + d, es), es);
        }
      }
    }
    // What is uniform is asked outside the loops over a thread's elements; those past the row count as zeros.
    float v[NV][VEC], c[VEC];
    float inv = 1.f, g = 1.f;
    if (a.gate_kind == BITSMOE_GATE_TOKEN) {
      g = load1(a.gate, a.gate_type, t * a.gate_ld);
      if (a.gate_sigmoid) g = sigmoid(g);
    }
    const auto take = [&](const uint8_t* p, int type, int k, float (&r)[VEC]) {
      if (in[k]) {
        unpack<VEC>(load_shared<VEC>(p, type, at[k]), type, r);
      } else {
#pragma unroll
        for (int q = 0; q < VEC; ++q) r[q] = 0.f;
      }
    };
    const auto all = [&](auto&& f) {
#pragma unroll
      for (int k = 0; k < NV; ++k) f(k);
    };
    if (a.y) {
      float ss = 0.f;
      all([&](int k) {
        take(sy, YT, k, v[k]);
#pragma unroll
        for (int q = 0; q < VEC; ++q) ss = fmaf(v[k][q], v[k][q], ss);
      });
      if (a.post_norm) inv = rsqrtf(block_sum<kW>(ss, red[0]) * inv_d + a.post_eps);
      all([&](int k) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[k][q] = v[k][q] * inv * cb[k][q];
      });
      if (elem) {
        const auto gate = [&](auto&& f, int type) {
          all([&](int k) {
            take(se, type, k, c);
#pragma unroll
            for (int q = 0; q < VEC; ++q) v[k][q] *= f(c[q]);
          });
        };
        const auto same = [](float e) { return e; };
        if (a.gate_type == BITSMOE_F32) {
          if (a.gate_sigmoid) gate(sigmoid, BITSMOE_F32);
          else gate(same, BITSMOE_F32);
        } else {
          if (a.gate_sigmoid) gate(sigmoid, BITSMOE_BF16);
          else gate(same, BITSMOE_BF16);
        }
      } else if (a.gate_kind) {
        all([&](int k) {
#pragma unroll
          for (int q = 0; q < VEC; ++q) v[k][q] *= g;
        });
      }
    } else {
      all([&](int k) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[k][q] = 0.f;
      });
    }
    float ss = 0.f;
    all([&](int k) {
      take(sh, HT, k, c);
#pragma unroll
      for (int q = 0; q < VEC; ++q) {
        v[k][q] = fmaf(a.residual_scale, c[q], v[k][q]);
        ss = fmaf(v[k][q], v[k][q], ss);
      }
    });
    if (a.h_out) all([&](int k) {
      if (in[k]) store_vec<VEC>(a.h_out, HT, t * a.h_out_ld + at[k], v[k]);
    });
    if (a.x) inv = rsqrtf(block_sum<kW>(ss, red[1]) * inv_d + a.pre_eps);
    if (!(a.y && a.post_norm && a.x)) __syncthreads();   // one sum a row: its buffer is read before the next row's
    if (threadIdx.x == 0 && t + (int64_t)slots * gridDim.x < a.T) fill(slot, t + (int64_t)slots * gridDim.x);   // all have read it
    if (++slot == slots) {
      slot = 0;
      ++use;
    }
    const auto put = [&](int type) {
      all([&](int k) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[k][q] = v[k][q] * inv * cp[k][q];
        if (in[k]) store_vec<VEC>(a.x, type, t * a.x_ld + at[k], v[k]);
      });
    };
    if constexpr (Q) {
      uint32_t most = 0u;
      all([&](int k) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[k][q] = v[k][q] * inv * cp[k][q];
        if (in[k]) most = max(most, most_of<VEC>(v[k]));
      });
      most = block_most<kW>(most, redm);
      const float to = rowscale_inverse(most);
      const bool bad = rowscale_bad(most);
      if (threadIdx.x == 0) x_scale[t] = rowscale_of(most);
      all([&](int k) {
        if (in[k]) store_codes<VEC>(a.x, t * a.x_ld + at[k], v[k], to, bad);
      });
    } else if (a.x) {
      if (a.x_type == BITSMOE_F32) put(BITSMOE_F32);
      else put(BITSMOE_BF16);
    }
  }
}

// Wide rows that registers do not hold: one block per row, h' in shared memory between the two norms.
constexpr int kWideThreads = 1024;
__global__ void __launch_bounds__(kWideThreads) k_block_norm_wide(const __grid_constant__ bitsmoe_block_norm_args a, float* x_scale) {
  extern __shared__ float row[];   // [D]
  __shared__ float red[2][32];
  __shared__ uint32_t redm[32];
  const auto sum = [&](float v, float* r) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) r[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(r[threadIdx.x & 31]);
  };
  const int64_t t = blockIdx.x;
  float inv = 1.f;
  if (a.y && a.post_norm) {
    float ss = 0.f;
    for (int d = threadIdx.x; d < a.D; d += kWideThreads) {
      const float v = load1(a.y, a.y_type, t * a.y_ld + d);
      ss = fmaf(v, v, ss);
    }
    inv = rsqrtf(sum(ss, red[0]) / (float)a.D + a.post_eps);
  }
  float tg = 1.f;
  if (a.gate_kind == BITSMOE_GATE_TOKEN) {
    tg = load1(a.gate, a.gate_type, t * a.gate_ld);
    if (a.gate_sigmoid) tg = sigmoid(tg);
  }
  float ss = 0.f;
  for (int d = threadIdx.x; d < a.D; d += kWideThreads) {
    float v = a.residual_scale * load1(a.h, a.h_type, t * a.h_ld + d);
    if (a.y) {
      float n = load1(a.y, a.y_type, t * a.y_ld + d);
      if (a.post_norm) n *= inv * (a.post_gain ? a.gain_offset + load1(a.post_gain, a.gain_type, d) : 1.f);
      float g = tg;
      if (a.gate_kind == BITSMOE_GATE_ELEMENT) {
        g = load1(a.gate, a.gate_type, t * a.gate_ld + d);
        if (a.gate_sigmoid) g = sigmoid(g);
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
  inv = rsqrtf(sum(ss, red[1]) / (float)a.D + a.pre_eps);
  const auto x_of = [&](int d) { return row[d] * inv * (a.pre_gain ? a.gain_offset + load1(a.pre_gain, a.gain_type, d) : 1.f); };
  if (!x_scale) {
    for (int d = threadIdx.x; d < a.D; d += kWideThreads) store1(a.x, a.x_type, t * a.x_ld + d, x_of(d));
    return;
  }
  uint32_t most = 0u;   // x in 8 bits (a thread reads the elements of row that it wrote)
  for (int d = threadIdx.x; d < a.D; d += kWideThreads) {
    row[d] = x_of(d);
    most = max(most, __float_as_uint(row[d]) & 0x7FFFFFFFu);
  }
  most = __reduce_max_sync(0xFFFFFFFFu, most);
  if ((threadIdx.x & 31) == 0) redm[threadIdx.x >> 5] = most;
  __syncthreads();
  most = __reduce_max_sync(0xFFFFFFFFu, redm[threadIdx.x & 31]);
  if (threadIdx.x == 0) x_scale[t] = rowscale_of(most);
  for (int d = threadIdx.x; d < a.D; d += kWideThreads) {
    const float v[1] = {row[d]};
    store_codes<1>(a.x, t * a.x_ld + d, v, rowscale_inverse(most), rowscale_bad(most));
  }
}

// Rows can be read VEC elements at a time: D a multiple of it and every row on a boundary of their size (16 bytes at most).
bool rows_of(const bitsmoe_block_norm_args& a, int vec) {
  if (a.D % vec) return false;
  const auto ok = [&](const void* p, int type, int64_t ld) {
    if (!p) return true;
    const int64_t size = type == BITSMOE_F32 ? 4 : type == BITSMOE_BF16 ? 2 : 1, align = size * vec < 16 ? size * vec : 16;
    return reinterpret_cast<uintptr_t>(p) % align == 0 && (a.T == 1 || ld * size % align == 0);
  };
  return ok(a.h, a.h_type, a.h_ld) && ok(a.y, a.y_type, a.y_ld) && ok(a.h_out, a.h_type, a.h_out_ld) && ok(a.x, a.x_type, a.x_ld) &&
         ok(a.gate_kind == BITSMOE_GATE_ELEMENT ? a.gate : nullptr, a.gate_type, a.gate_ld) &&
         ok(a.post_gain, a.gain_type, 0) && ok(a.pre_gain, a.gain_type, 0) && ok(a.channel_scale, a.gain_type, 0);
}

template <int VEC, int NV, int TH, bool Q>
cudaError_t launch_rows(const bitsmoe_block_norm_args& a, float* x_scale, int dev, int64_t blocks, int per_sm, int threads, cudaStream_t st) {
  const bool hf = a.h_type == BITSMOE_F32, yf = a.y_type == BITSMOE_F32;
  const auto room = [&](int type) {
    const size_t bytes = (size_t)a.D * (type == BITSMOE_F32 ? 4 : 2);
    return VEC == 8 ? bytes : (bytes + 15) / 16 * 16 + 16;
  };
  const size_t row = (a.y ? room(a.y_type) : 0) + room(a.h_type) + (a.gate_kind == BITSMOE_GATE_ELEMENT ? room(a.gate_type) : 0);
  const int slots = (int)std::min<size_t>(kMaxSlots, (size_t)(220 / per_sm - 2) * 1024 / row);
  if (slots < 1) return cudaErrorInvalidValue;   // (VEC 8: at most 12 x 16384 bytes a row; VEC 1: half of it)
  const auto go = [&](auto kern, cudaError_t e) {
    if (e == cudaSuccess) kern<<<(unsigned)blocks, threads, slots * row, st>>>(a, slots, x_scale);
    return e;
  };
  constexpr int F = BITSMOE_F32, B = BITSMOE_BF16, kRing = 220 * 1024;
  const cudaError_t e =
      hf ? (yf ? go(k_block_norm_rows<VEC, NV, TH, F, F, Q>, allow_shared<k_block_norm_rows<VEC, NV, TH, F, F, Q>>(dev, kRing))
               : go(k_block_norm_rows<VEC, NV, TH, F, B, Q>, allow_shared<k_block_norm_rows<VEC, NV, TH, F, B, Q>>(dev, kRing)))
         : (yf ? go(k_block_norm_rows<VEC, NV, TH, B, F, Q>, allow_shared<k_block_norm_rows<VEC, NV, TH, B, F, Q>>(dev, kRing))
               : go(k_block_norm_rows<VEC, NV, TH, B, B, Q>, allow_shared<k_block_norm_rows<VEC, NV, TH, B, B, Q>>(dev, kRing)));
  return e == cudaSuccess ? cudaGetLastError() : e;
}

// Rows of up to 256: a warp a row, four rows a block.
template <int VEC, int NV, bool Q>
cudaError_t launch_warps(const bitsmoe_block_norm_args& a, float* x_scale, cudaStream_t st) {
  k_block_norm<VEC, NV, true, Q><<<(unsigned)(((int64_t)a.T + 3) / 4), 128, 0, st>>>(a, x_scale);
  return cudaGetLastError();
}

template <bool Q, int VEC, int NV, int TH = kRowThreads>
cudaError_t launch_norm(const bitsmoe_block_norm_args& a, float* x_scale, cudaStream_t st) {
  int dev = 0, sms = 0;
  cudaError_t e = device_sms(&dev, &sms);
  if (e != cudaSuccess) return e;
  const int nvec = a.D / VEC, threads = ((nvec + NV - 1) / NV + 31) / 32 * 32;
  // as many blocks as run at once (64 registers a thread: 1024 threads; 128 with more than 8 elements a thread)
  const int per_sm = std::max(1, (VEC * NV > 8 ? 512 : 1024) / threads);
  const int64_t full = (int64_t)sms * per_sm;
  if constexpr (VEC == 8) {
    if (a.T <= full) {
      k_block_norm<VEC, NV, false, Q><<<(unsigned)a.T, threads, 0, st>>>(a, x_scale);
      return cudaGetLastError();
    }
  }
  return launch_rows<VEC, NV, TH, Q>(a, x_scale, dev, std::min<int64_t>(a.T, full), per_sm, threads, st);
}

bool type_ok(int t) { return t == BITSMOE_F32 || t == BITSMOE_BF16; }
bool misaligned(const void* p, int type) { return reinterpret_cast<uintptr_t>(p) % (type == BITSMOE_F32 ? 4 : 2) != 0; }

template <bool Q>
cudaError_t launch_block_norm(const bitsmoe_block_norm_args& a, float* x_scale, cudaStream_t st) {
  if (a.D <= 256)
    return rows_of(a, 8)   ? launch_warps<8, 1, Q>(a, x_scale, st)
           : rows_of(a, 2) ? launch_warps<2, 4, Q>(a, x_scale, st)
                           : launch_warps<1, 8, Q>(a, x_scale, st);
  if (a.D <= 16384 && rows_of(a, 8))
    return a.D <= 4096   ? launch_norm<Q, 8, 1>(a, x_scale, st)
           : a.D <= 8192 ? launch_norm<Q, 8, 2>(a, x_scale, st)
                         : launch_norm<Q, 8, 4>(a, x_scale, st);
  if (a.D <= 8192) return a.D <= 4096 ? launch_norm<Q, 1, 8>(a, x_scale, st) : launch_norm<Q, 1, 8, 1024>(a, x_scale, st);
  const size_t smem = (size_t)a.D * 4;
  if (smem > 40 * 1024) {   // 48 KB with the static part need no opt-in
    const cudaError_t e = cudaFuncSetAttribute(k_block_norm_wide, cudaFuncAttributeMaxDynamicSharedMemorySize, BITSMOE_BLOCK_NORM_MAX_D * 4);
    if (e != cudaSuccess) return e;
  }
  k_block_norm_wide<<<(unsigned)a.T, kWideThreads, smem, st>>>(a, x_scale);
  return cudaGetLastError();
}

// x_scale NULL and `coded` false: x of a dense type.
int block_norm(const bitsmoe_block_norm_args* args, bool coded, float* x_scale, void* stream) {
  if (!args) return BITSMOE_ERR_INVALID_ARG;
  const bitsmoe_block_norm_args a = *args;
  if (a.T < 0 || a.D < 1) return BITSMOE_ERR_INVALID_ARG;
  if (a.D > BITSMOE_BLOCK_NORM_MAX_D || a.T > (1 << 24)) return BITSMOE_ERR_SHAPE;
  if (!type_ok(a.h_type) || !type_ok(a.y_type) || !type_ok(a.gate_type) || !type_ok(a.gain_type) ||
      (coded ? a.x_type != BITSMOE_E4M3 : !type_ok(a.x_type)))
    return BITSMOE_ERR_INVALID_ARG;
  if (a.gate_kind < BITSMOE_GATE_NONE || a.gate_kind > BITSMOE_GATE_ELEMENT) return BITSMOE_ERR_INVALID_ARG;
  if (!(a.post_eps >= 0.f) || !(a.pre_eps >= 0.f) || !std::isfinite(a.residual_scale) || !std::isfinite(a.branch_scale) ||
      !std::isfinite(a.gain_offset))
    return BITSMOE_ERR_INVALID_ARG;
  if (a.T == 0) return BITSMOE_OK;   // (pointers of empty rows may be null)
  if ((!a.y && (a.post_norm || a.gate_kind || a.channel_scale)) || (a.post_gain && !a.post_norm)) return BITSMOE_ERR_INVALID_ARG;
  if (coded && (!a.x || !x_scale)) return BITSMOE_ERR_INVALID_ARG;
  if (!a.x && a.pre_gain) return BITSMOE_ERR_INVALID_ARG;
  if (!a.h || (!a.h_out && !a.x) || (a.gate_kind && !a.gate)) return BITSMOE_ERR_INVALID_ARG;
  if (a.h_ld < a.D || (a.y && a.y_ld < a.D) || (a.h_out && a.h_out_ld < a.D) || (a.x && a.x_ld < a.D) ||
      (a.gate_kind == BITSMOE_GATE_TOKEN && a.gate_ld < 1) || (a.gate_kind == BITSMOE_GATE_ELEMENT && a.gate_ld < a.D))
    return BITSMOE_ERR_INVALID_ARG;
  if (misaligned(a.h, a.h_type) || misaligned(a.y, a.y_type) || misaligned(a.gate, a.gate_type) ||
      misaligned(a.post_gain, a.gain_type) || misaligned(a.pre_gain, a.gain_type) ||
      misaligned(a.channel_scale, a.gain_type) || misaligned(a.h_out, a.h_type) || (coded ? reinterpret_cast<uintptr_t>(x_scale) % 4 != 0 : misaligned(a.x, a.x_type)))
    return BITSMOE_ERR_ALIGNMENT;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = coded ? launch_block_norm<true>(a, x_scale, st) : launch_block_norm<false>(a, nullptr, st);
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}

}  // namespace

extern "C" int bitsmoe_block_norm(const bitsmoe_block_norm_args* args, void* stream) {
  return block_norm(args, false, nullptr, stream);
}

extern "C" int bitsmoe_block_norm_rowscale(const bitsmoe_block_norm_args* args, float* x_scale, void* stream) {
  return block_norm(args, true, x_scale, stream);
}
