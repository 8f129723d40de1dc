// Product of dense rows with a microscaled 4-bit matrix:
//
//   y[t][r] = s_w s_x sum_k W[r][k] x[t][k]
//   or, with a second matrix U of the same shape, SiLU(W x) * (U x)
//
// x in bf16, or itself microscaled.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "microscale.cuh"
#include "tc.cuh"

namespace {
using namespace bmoe;

struct MicroMat {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t pitch;
  int tiles;
};

__device__ __forceinline__ float silu_mul(float g, float u) { return g / (1.f + expf(-g)) * u; }

__device__ __forceinline__ void store_y(void* y, int type, int64_t i, float v) {
  if (type == BITSMOE_F32) static_cast<float*>(y)[i] = v;
  else static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
}

// What is stored (NaN) for results that a wait that ran out has lost, so that a call without a status word shows it too.  A
// warp whose wait ran out passes nothing on: who waits for it runs out as well, up to the warps that store.
constexpr uint32_t kLost = 0x7FC00000u;

// ---------------------------------------------------------------------------
// Few tokens: the weights' codes pass once through shared memory into warp-level
// products (mma.sync m16n8k16, 16 weight rows x 8 tokens x 16 columns).
//
// A code is exact in fp16, and two of them are converted by one instruction
// (e2m1x2 -> f16x2: 7 operations for 8 codes with the byte picks; forming bf16
// bit patterns takes 15).  The activations of a CTA's columns are kept in fp16 where
// all of them are exact there: times 2^6 (bf16's 8 bits from 2^-23 to 2^10), or else
// times the power of two that brings their largest to [2^14, 2^15) (32 binades below
// it).  Otherwise the CTA takes the bf16 products (the codes as bf16 bit patterns
// times 2^126).  So nothing is rounded but the fp32 sums.
//
// The matrix's bytes are the floor, streamed once: 4096 rows x 14336, one token, 31 MB
// in 11.2 us (2.8 TB/s; 4.6 us at the copy bandwidth), 19456 x 8192, 85 MB in 21 us
// (4.0 TB/s; the copies alone 16.3).  Above the copies lies what the decode issues,
// and on small matrices the fixed 5 us of a launch, a cluster's start, the
// first copies' latency and the sum over the cluster (2048 x 2048: 5.2 us in all); more
// tokens add their conversion and its reads from shared memory (8 tokens of the first
// 15.7 us).
// ---------------------------------------------------------------------------
constexpr int kFewWarps = 16;                      // consumers: 8 row tiles x 2 halves of a stage's columns
constexpr int kFewThreads = 32 * (kFewWarps + 1);  // and the warp that copies
constexpr int kFewTokens = 16;
constexpr int kStageK = 256;                       // columns of a stage (128 bytes of codes a row)
constexpr uint32_t kCodeTile = 128 * 128;          // bytes of 128 rows of a stage's codes

// Bytes of a CTA's buffer of partial sums: 2 groups of warps x tokens x 128 rows (a CTA's share of the rows from
// every CTA of the cluster).
__host__ __device__ constexpr uint32_t few_red_bytes(int nt) { return 2u * nt * 8 * 512; }

struct FewArgs {
  int T, rows, cols, tiles, mt;
  int nst, sps, splits, stages;
  uint32_t stage;
  uint32_t x_pitch;      // bytes of a token's activations in shared memory
  const uint8_t* ws;
  const uint8_t* us;
  const __nv_bfloat16* x;
  int64_t x_ld;
  int x_vec;             // x's rows can be read 16 bytes at a time
  MicroMat xq;
  float sw, su;
  void* y;
  int y_type;
  int64_t y_ld;
  long long spin;
  int lose;
  int* status;
};

template <bool BF>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const float (&c)[4]) {
  if constexpr (BF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// The 8 codes of w as 4 pairs (columns 2i, 2i + 1) of fp16, or of bf16 (the codes' bits as bf16 are the
// values times 2^-126).
template <bool BF>
__device__ __forceinline__ void code_pairs(uint32_t w, uint32_t (&r)[4]) {
  if constexpr (!BF) {
    asm("{\n .reg .b8 t0, t1, t2, t3;\n mov.b32 {t0, t1, t2, t3}, %4;\n cvt.rn.f16x2.e2m1x2 %0, t0;\n cvt.rn.f16x2.e2m1x2 %1, t1;\n"
        " cvt.rn.f16x2.e2m1x2 %2, t2;\n cvt.rn.f16x2.e2m1x2 %3, t3;\n}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
  } else {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const uint32_t n = ((w >> (8 * b)) & 0xFu) | (((w >> (8 * b + 4)) & 0xFu) << 16);
      r[b] = ((n & 0x00080008u) << 12) | ((n & 0x00070007u) << 6);
      asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(r[b]) : "r"(0x7E807E80u));   // 2^126: exact
    }
  }
}

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 lds128a(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t e4m3x2_f16(uint32_t p) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)p));
  return r;
}
template <bool BF>
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (BF) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  else asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// This warp's 16 rows x 128 columns of a stage (half kh) with NT tiles of 8 tokens.  Lane (g, t) takes the codes
// of columns 8t .. 8t + 7 of every 32, of rows g and g + 8: two products of 16 columns.
// E8M0: the 32 columns are a block of each row; its scale (times inv, in fp32) multiplies the products' fp32 sum.
// E4M3: a lane's 8 columns lie in one block, whose scale multiplies the codes (6 significant bits between 2^-10
// and 2688: exact in fp16 and bf16).
template <int FMT, int NT, bool BF>
__device__ __forceinline__ void few_half(uint32_t code, uint32_t sf, const uint32_t (&xo)[NT], int rt, int kh, int lane,
                                         int tiles_left, float inv, float (&acc)[NT][4]) {
  constexpr bool E8 = FMT == BITSMOE_MICRO_E8M0;
  constexpr int TPH = E8 ? 1 : 2;   // scale tiles of a half
  const int g = lane >> 2, t = lane & 3;
  const int r = 16 * rt + g;
  const uint32_t pick = t >= 2 ? 0x3232u : 0x1010u;   // E4M3: this lane's block of the two of 32 columns
#pragma unroll
  for (int q = 0; q < TPH; ++q) {
    const int tile = kh * TPH + q;
    if (tile >= tiles_left) return;   // past the matrix's columns (and its scales)
    uint32_t sw[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int rr = r + 8 * h;
      sw[h] = lds32(sf + (uint32_t)tile * 512 + (rr & 31) * 16 + (rr >> 5) * 4);
    }
#pragma unroll
    for (int b = 0; b < 4 / TPH; ++b) {
      const int j = kh * 4 + q * 2 + b;   // 32 columns: 16-byte chunk of the row
      uint4 xb[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) xb[n] = lds128a(xo[n] + (uint32_t)j * 64);
      const uint32_t base = code + (uint32_t)r * 128 + (uint32_t)((j ^ g) << 4) + t * 4;
      uint32_t p0[4], p1[4];
      code_pairs<BF>(lds32(base), p0);
      code_pairs<BF>(lds32(base + 1024), p1);
      if constexpr (E8) {
        float s[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t v;
          asm("cvt.rn.bf16x2.ue8m0x2 %0, %1;" : "=r"(v) : "h"((uint16_t)(sw[h] >> (16 * (b >> 1)))));
          s[h] = ((b & 1) ? bf16hi(v) : bf16lo(v)) * inv;
        }
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float d[4], e[4];
          mma16<BF>(d, {p0[0], p1[0], p0[1], p1[1]}, xb[n].x, xb[n].y, zero);
          mma16<BF>(e, {p0[2], p1[2], p0[3], p1[3]}, xb[n].z, xb[n].w, d);
          acc[n][0] = fmaf(s[0], e[0], acc[n][0]);
          acc[n][1] = fmaf(s[0], e[1], acc[n][1]);
          acc[n][2] = fmaf(s[1], e[2], acc[n][2]);
          acc[n][3] = fmaf(s[1], e[3], acc[n][3]);
        }
      } else {
        uint32_t m[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          m[h] = e4m3x2_f16(sw[h] >> (16 * b));
          if constexpr (BF) {
            const __nv_bfloat162 v = __floats2bfloat162_rn(f16lo(m[h]), f16hi(m[h]));   // exact
            m[h] = *reinterpret_cast<const uint32_t*>(&v);
          }
          m[h] = __byte_perm(m[h], 0u, pick);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p0[i] = mul2<BF>(p0[i], m[0]);
          p1[i] = mul2<BF>(p1[i], m[1]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float d[4];
          mma16<BF>(d, {p0[0], p1[0], p0[1], p1[1]}, xb[n].x, xb[n].y, acc[n]);
          mma16<BF>(acc[n], {p0[2], p1[2], p0[3], p1[3]}, xb[n].z, xb[n].w, d);
        }
      }
    }
  }
}

__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, %0;" ::"n"(kFewWarps * 32) : "memory"); }

// Eight activations of token t from column k (a multiple of 8) as they are stored, zeros past the columns: 8 bf16, or
// a word of codes and its scale byte.
__device__ __forceinline__ uint4 few_raw(const FewArgs& g, int format, int t, int k) {
  uint4 q = make_uint4(0u, 0u, 0u, 0u);
  if (k >= g.cols) return q;
  if (g.xq.codes) {
    q.x = __ldg(reinterpret_cast<const uint32_t*>(g.xq.codes + (int64_t)t * g.xq.pitch + k / 2));
    q.y = g.xq.scales[micro_scale_at(g.xq.tiles, t, k / micro_block(format))];
  } else {
    const __nv_bfloat16* p = g.x + (int64_t)t * g.x_ld + k;
    if (g.x_vec && k + 8 <= g.cols) {
      q = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (k + i < g.cols) w[i / 2] |= (uint32_t)__bfloat16_as_ushort(p[i]) << (16 * (i & 1));
      q = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  return q;
}
__device__ __forceinline__ void few_values(const FewArgs& g, int format, const uint4& q, float (&v)[8]) {
  if (g.xq.codes) {
    const float s = micro_scale(format, q.y);
    uint32_t h[4];
    code_pairs<false>(q.x, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = f16lo(h[i]) * s;
      v[2 * i + 1] = f16hi(h[i]) * s;
    }
  } else {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16lo(w[i]);
      v[2 * i + 1] = bf16hi(w[i]);
    }
  }
}

// A cluster takes row tiles of 128 one after the other; its CTAs split the columns.  Each warp sends its part of a
// tile to the CTA that stores those rows, by asynchronous stores into that CTA's shared memory; the next tile's
// parts wait until every CTA has read this one's.
template <int FMT, bool GLU, int NT>
__global__ void __launch_bounds__(kFewThreads, 1)
    k_micro_few(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap, FewArgs g) {
  constexpr bool E8 = FMT == BITSMOE_MICRO_E8M0;
  constexpr int NA = GLU ? 2 : 1, CPS = E8 ? 2 : 4;
  extern __shared__ uint8_t raw[];
  __shared__ uint32_t top;     // the largest finite |activation| of the CTA's columns (fp32 bits)
  __shared__ int inexact_any;
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int S = g.stages;
  constexpr uint32_t kRed = few_red_bytes(NT);   // [rank][group of warps][token][rows of this CTA] fp32
  uint8_t* redb = sm + (size_t)S * g.stage;
  uint8_t* xs = redb + kRed;
  uint64_t* full = reinterpret_cast<uint64_t*>(xs + (size_t)g.T * g.x_pitch);
  uint64_t* empty = full + S;
  uint64_t* rfull = empty + S;                        // the parts of a tile are there
  uint64_t* rfree = rfull + 1;                        // every CTA of the cluster has read them
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = blockIdx.y;
  const int st0 = rank * g.sps, nk = max(0, min(g.sps, g.nst - st0));
  if (tid == kFewWarps * 32) {
    prefetch_map(&wmap);
    if (GLU) prefetch_map(&umap);
  }
  if (tid == 0) {
    for (int i = 0; i < S; ++i) {
      mbar_init_n(full + i, 1);
      mbar_init_n(empty + i, !GLU && nk == 1 ? kFewWarps : kFewWarps / 2);
    }
    mbar_init_n(rfull, 1);
    mbar_init_n(rfree, (uint32_t)g.splits);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    mbar_expect_tx(rfull, kRed);
    top = 0u;
    inexact_any = 0;
  }
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  bool ok = true;

  if (wid == kFewWarps) {
    if (lane == 0) {
      int st = 0, u = 0, n = 0;
      for (int mi = blockIdx.x; mi < g.mt && ok; mi += gridDim.x) {
        for (int i = 0; i < nk * NA; ++i, ++n) {
          if (u > 0) ok = mbar_wait(empty + st, (uint32_t)(u - 1) & 1u, g.spin);
          if (!ok) break;
          const bool second = GLU && (i & 1);
          const int kb = st0 + (GLU ? i >> 1 : i), cnt = min(CPS, g.tiles - kb * CPS);
          uint8_t* base = sm + (size_t)st * g.stage;
          mbar_expect_tx(full + st, kCodeTile + (uint32_t)cnt * 512u);
          tma_load_2d(smem_u32(base), second ? &umap : &wmap, kb * 128, mi * 128, smem_u32(full + st));
          bulk_g2s(base + kCodeTile, (second ? g.us : g.ws) + ((size_t)mi * g.tiles + (size_t)kb * CPS) * 512, (uint32_t)cnt * 512u,
                   full + st);
          if (++st == S) {
            st = 0;
            ++u;
          }
        }
      }
      for (int j = max(0, n - S); j < n; ++j) mbar_wait(full + j % S, (uint32_t)(j / S) & 1u);   // copies in flight
    }
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  } else {
    // The activations of this CTA's columns, 8 a thread at a time (a warp within one token).
    const int k0 = st0 * kStageK, n8 = nk * (kStageK / 8), per = (n8 + 31) / 32;
    float inv = 1.f;   // undoes the activations' power of two
    bool bf = false;
    // each(t, c, raw): place c of token t, four places of a thread requested at a time
    const auto each = [&](auto&& use) {
      const int items = g.T * per;
      for (int w0 = wid; w0 < items; w0 += 4 * kFewWarps) {
        uint4 q[4];
        int t[4], c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int w = w0 + i * kFewWarps;
          t[i] = w / per;
          c[i] = (w - t[i] * per) * 32 + lane;
          if (w < items && c[i] < n8) q[i] = few_raw(g, FMT, t[i], k0 + c[i] * 8);
          else c[i] = -1;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c[i] >= 0) *reinterpret_cast<uint4*>(xs + (size_t)t[i] * g.x_pitch + (size_t)c[i] * 16) = use(q[i]);
      }
    };
    if (!E8 && g.xq.codes) {   // code times E4M3 scale: exact in fp16 as it is
      each([&](const uint4& q) {
        uint32_t h[4];
        code_pairs<false>(q.x, h);
        const uint32_t m = __byte_perm(e4m3x2_f16(q.y), 0u, 0x1010u);
        return make_uint4(mul2<false>(h[0], m), mul2<false>(h[1], m), mul2<false>(h[2], m), mul2<false>(h[3], m));
      });
      bar_consumers();
    } else {
      // In fp16 times mul; whether all of them are exact there; the largest finite magnitude.
      const auto stage = [&](float mul) {
        bool inexact = false;
        float m = 0.f;
        each([&](const uint4& raw) {
          float v[8];
          few_values(g, FMT, raw, v);
          uint32_t h[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = v[2 * i] * mul, q = v[2 * i + 1] * mul;
            const __half2 f = __floats2half2_rn(p, q);
            const float2 back = __half22float2(f);
            inexact |= (back.x != p && p == p) || (back.y != q && q == q) || (p == 0.f && v[2 * i] != 0.f) ||
                       (q == 0.f && v[2 * i + 1] != 0.f);
            h[i] = *reinterpret_cast<const uint32_t*>(&f);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (fabsf(v[i]) <= 3.402823466e38f) m = fmaxf(m, fabsf(v[i]));
          return make_uint4(h[0], h[1], h[2], h[3]);
        });
        if (inexact) inexact_any = 1;
        if (__float_as_uint(m) > *(volatile uint32_t*)&top) atomicMax(&top, __float_as_uint(m));
        bar_consumers();
        return inexact_any != 0;
      };
      inv = 0.015625f;
      if (stage(64.f)) {   // not all of them in 2^-23 .. 2^10: the largest to [2^14, 2^15)
        bar_consumers();
        if (tid == 0) inexact_any = 0;
        bar_consumers();
        const int e = (int)(top >> 23) - 127;
        // The inverse only makes scales smaller (none of another block overflows), and those that leave fp32's range
        // are of sums below 2^-127.
        const bool norm = e >= -86 && e <= 14;
        inv = norm ? __uint_as_float((uint32_t)(e - 14 + 127) << 23) : 1.f;
        bf = !norm || stage(__uint_as_float((uint32_t)(14 - e + 127) << 23));
        if (bf) {
          inv = 1.f;
          bar_consumers();
          each([&](const uint4& raw) {
            float v[8];
            few_values(g, FMT, raw, v);
            uint32_t h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const __nv_bfloat162 f = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);   // exact
              h[i] = *reinterpret_cast<const uint32_t*>(&f);
            }
            return make_uint4(h[0], h[1], h[2], h[3]);
          });
          bar_consumers();
        }
      }
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");   // the cluster's barriers are set up
    const int rt = wid & 7, kh = wid >> 3;
    uint32_t xo[NT];   // this lane's activations of column 0 (tokens past T read the last one's; nothing stores their results)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      xo[n] = smem_u32(xs) + (uint32_t)min(n * 8 + (lane >> 2), g.T - 1) * g.x_pitch + (uint32_t)(lane & 3) * 16;
    // The two groups of eight warps take every other slot (with GLU: one matrix each); of a single one, half of its
    // columns each.
    const bool halves = !GLU && nk == 1;
    const int rs = 128 / g.splits;                              // rows that a CTA stores
    const int owner = 16 * rt / rs, orow = 16 * rt - owner * rs + (lane >> 2);
    int st = -1, it = 0;     // slot of the ring and its phase's parity
    uint32_t ph = 0;
    // All lanes poll the barriers and one arrives by its predicate: with waits of one lane the warps ran diverged
    // (4096 x 14336, one token, 12.3 us where this takes 11.2).
    // The ring has an even number of slots, so a slot is always the same group's: a group that waits for a slot's next
    // use has seen its last one, and a phase's parity cannot stand for the one before.
    for (int mi = blockIdx.x; mi < g.mt; mi += gridDim.x, ++it) {
      float acc[NT][4] = {};
      for (int i = 0; i < nk * NA; ++i) {
        if (++st == S) st = 0, ph ^= 1u;
        if (!ok || (!halves && (st & 1) != kh)) continue;
        ok = mbar_try_wait(full + st, ph) || mbar_wait(full + st, ph, g.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) continue;
        const uint32_t code = smem_u32(sm) + (uint32_t)st * g.stage, sf = code + kCodeTile;
        const int ks = GLU ? i >> 1 : i, left = g.tiles - (st0 + ks) * CPS;
        uint32_t xi[NT];
#pragma unroll
        for (int q = 0; q < NT; ++q) xi[q] = xo[q] + (uint32_t)ks * (kStageK * 2);
        // one copy of the code for both halves: unrolled, it did not stay in the instruction cache
        const int h0 = halves ? kh : 0, h1 = halves ? kh + 1 : 2;
        if (bf) {
#pragma unroll 1
          for (int h = h0; h < h1; ++h) few_half<FMT, NT, true>(code, sf, xi, rt, h, lane, left, inv, acc);
        } else {
#pragma unroll 1
          for (int h = h0; h < h1; ++h) few_half<FMT, NT, false>(code, sf, xi, rt, h, lane, left, inv, acc);
        }
        __syncwarp();
        mbar_arrive(lane == 0 && !(g.lose && i == 0 && it == 0 && wid == 0 && (blockIdx.x | blockIdx.y) == 0), empty + st);
      }
      // this warp's part to the CTA that stores these rows, counted in bytes on its barrier
      if (it > 0) {
        if (ok) ok = mbar_wait_cluster(rfree, (uint32_t)(it - 1) & 1u, g.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
      }
      uint32_t dst, bar;
      const uint32_t buf = smem_u32(redb);
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(dst) : "r"(buf), "r"(owner));
      asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar) : "r"(smem_u32(rfull)), "r"(owner));
      const float unit = E8 ? 1.f : inv;
      if (ok)
#pragma unroll
        for (int q = 0; q < NT; ++q)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int c = q * 8 + (lane & 3) * 2 + (j & 1);
            asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];" ::
                             "r"(dst + (uint32_t)(((rank * 2 + kh) * NT * 8 + c) * rs + orow + (j >> 1) * 8) * 4u),
                         "r"(__float_as_uint(acc[q][j] * unit)), "r"(bar) : "memory");
          }
      if (mi + (int)gridDim.x >= g.mt) {   // everything sent: the others may leave once they have their parts
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
      }
      // the parts of this CTA's rows, added in the order of the CTAs and halves
      // (a warp whose wait ran out sends nothing and stores NaN from then on, but keeps every barrier)
      if (ok) ok = mbar_wait_cluster(rfull, (uint32_t)it & 1u, g.spin);
      ok = __all_sync(0xFFFFFFFFu, ok);
      for (int e = tid; e < rs * g.T; e += kFewWarps * 32) {
        const int c = e / rs, r = e - c * rs;
        float p[16];   // [CTA][group]
#pragma unroll
        for (int q = 0; q < 16; ++q)
          p[q] = q < 2 * g.splits ? __uint_as_float(lds32(buf + (uint32_t)((q * NT * 8 + c) * rs + r) * 4u)) : 0.f;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 16; ++q) sum[GLU ? q & 1 : 0] += p[q];
        const int m = mi * 128 + rank * rs + r;
        if (m >= g.rows) continue;
        float o = sum[0] * g.sw;
        if (GLU) o = silu_mul(o, sum[1] * g.su);
        store_y(g.y, g.y_type, (int64_t)c * g.y_ld + m, ok ? o : __uint_as_float(kLost));
      }
      __syncwarp();
      if (mi + (int)gridDim.x < g.mt) {
        bar_consumers();   // the whole CTA has read the parts
        if (tid == 0 && ok) mbar_expect_tx(rfull, kRed);   // for the next tile
        if (tid < g.splits) {
          uint32_t to;
          asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(smem_u32(rfree)), "r"(tid));
          asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(to) : "memory");
        }
      }
    }
  }
  // No CTA leaves while others may still write to its shared memory: it has all parts that are sent to it, or,
  // after a wait that ran out, every CTA of the cluster has sent its own and they have had time to arrive.
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  if (!ok) {
    const long long t0 = clock64();
    while (clock64() - t0 < 100000) {
    }
    if (g.status) atomicCAS(g.status, 0, BITSMOE_ERR_TIMEOUT);
  }
}

// Clusters of `splits` CTAs of a kernel (one CTA an SM) that run at once on the current device, asked once for each.
template <typename K>
int resident_clusters(K kern, int threads, int splits) {
  static std::atomic<int> known[64][4];
  int dev = 0, q = splits == 1 ? 0 : splits == 2 ? 1 : splits == 4 ? 2 : 3;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  if (dev < 64) {
    const int n = known[dev][q].load(std::memory_order_relaxed);
    if (n > 0) return n;
  }
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024) != cudaSuccess) return 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = (unsigned)splits;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1, (unsigned)splits, 1);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = 220 * 1024;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) return 0;
  if (dev < 64) known[dev][q].store(n, std::memory_order_relaxed);
  return n;
}

struct FewPlan {
  int splits, sps, stages, clusters;
  uint32_t stage, x_pitch;
  size_t smem;
};

// How T tokens run on the kernel for few of them, or false when their activations do not fit shared memory.
// Measured, us here and by the decoded tiles: 1, 8, 12, 16 tokens of 14336 rows x 4096 (16 slots a CTA) 12.0, 16.9,
// 22.2, 25.5 and 21.6, 22.1, 22.3, 22.3, with SwiGLU 19.9, 25.1, 32.7, 36.1 and 32.9, 34.0, 34.4, 34.7; of 4096 x 14336
// (14 slots) 11.6, 15.7, 20.2, 22.6 and 21.3, 21.4, 21.6, 21.6; 16 of 2048 x 2048 (2 slots) 6.9 and 11.8.  Longer
// ones: 9, 12 tokens of 14336 x 8192 (32 slots) 32.9, 34.5 and 40.0, 40.1, with SwiGLU 54.9, 56.5 and 62.1, 62.5; of
// 8192 x 28672 (56 slots) 52.4, 61.0 and 66.8, 66.8.  For
// coded tokens the block-scaled MMAs take 9.5 at 1 to 24 tokens, so only small products stay here (2048 x 2048: 5.0
// to 6.6 against 9.1 to 10.1).
bool few_plan(int format, bool glu, bool coded, int T, int rows, int cols, int (*resident)(int), FewPlan* p) {
  if (T > kFewTokens) return false;
  const int CPS = format == BITSMOE_MICRO_E8M0 ? 2 : 4;
  const int nst = (cols + kStageK - 1) / kStageK, mt = (rows + 127) / 128;
  p->stage = kCodeTile + (uint32_t)CPS * 512;
  const size_t room = 225 * 1024 - 1024 - 512;
  int64_t best = -1;
  for (int splits = 1; splits <= 8; splits *= 2) {   // CTAs of a cluster: the fewest of those with the least work a CTA
    const int sps = (nst + splits - 1) / splits;
    // 64 bytes beyond a multiple of 128: the tokens of a fragment's 16-byte loads in different banks
    const uint32_t pitch = (uint32_t)sps * kStageK * 2 + 64;
    const size_t xb = (size_t)T * pitch;
    const int clusters = std::min(mt, resident(splits));
    if (clusters < 1) continue;
    const size_t red = (size_t)few_red_bytes(T > 8 ? 2 : 1);
    if (xb + red + 4 * (size_t)p->stage > room) continue;   // slots enough to cover a copy's latency
    const int64_t work = (int64_t)((mt + clusters - 1) / clusters) * sps;
    if (best >= 0 && work >= best) continue;
    best = work;
    p->splits = splits;
    p->sps = sps;
    p->clusters = clusters;
    p->x_pitch = pitch;
    p->stages = (int)std::min<size_t>((room - xb - red) / p->stage, 16) & ~1;   // even: see the kernel
    p->smem = 1024 + (size_t)p->stages * p->stage + red + xb + (size_t)(2 * p->stages + 2) * 8;
  }
  if (coded) return best >= 0 && best * (glu ? 2 : 1) * (T > 8 ? 2 : 1) <= 8;
  return best >= 0 && (T <= 12 || best <= 12);
}

template <int FMT, bool GLU, int NT>
cudaError_t launch_few(const FewPlan& p, const bitsmoe_microscale* w, const bitsmoe_microscale* up, FewArgs g, int dev, cudaStream_t st) {
  g.nst = (g.cols + kStageK - 1) / kStageK;
  g.mt = (g.rows + 127) / 128;
  g.splits = p.splits;
  g.sps = p.sps;
  g.stages = p.stages;
  g.stage = p.stage;
  g.x_pitch = p.x_pitch;
  CUtensorMap wm, um;
  const int64_t pitch = micro_pitch(g.cols);
  if (!make_row_map(&wm, true, w->codes, g.rows, pitch, pitch, 128)) return cudaErrorInvalidValue;
  um = wm;
  if (GLU && !make_row_map(&um, true, up->codes, g.rows, pitch, pitch, 128)) return cudaErrorInvalidValue;
  auto kern = k_micro_few<FMT, GLU, NT>;
  cudaError_t e = allow_shared<k_micro_few<FMT, GLU, NT>>(dev, 226 * 1024);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = (unsigned)p.splits;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)p.clusters, (unsigned)p.splits, 1);
  cfg.blockDim = dim3(kFewThreads);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, wm, um, g);
}

// (all variants have the same threads and take a whole SM)
int few_resident(int splits) { return resident_clusters(k_micro_few<BITSMOE_MICRO_E8M0, false, 1>, kFewThreads, splits); }

template <int FMT, bool GLU>
cudaError_t launch_few_nt(const FewPlan& p, const bitsmoe_microscale* w, const bitsmoe_microscale* up, const FewArgs& g, int dev, cudaStream_t st) {
  return g.T > 8 ? launch_few<FMT, GLU, 2>(p, w, up, g, dev, st) : launch_few<FMT, GLU, 1>(p, w, up, g, dev, st);
}

// Sixteen tokens' results of weight row m (a lane's; the warp's lanes hold consecutive rows) from token t on.
template <int NA>
__device__ __forceinline__ void store_tokens(const uint32_t (&v)[NA][16], int t, int T, int m, float sw, float su, void* y,
                                             int y_type, int64_t y_ld) {
#pragma unroll
  for (int q = 0; q < 16; ++q) {
    if (t + q >= T) break;
    float o = __uint_as_float(v[0][q]) * sw;
    if (NA == 2) o = silu_mul(o, __uint_as_float(v[NA - 1][q]) * su);
    store_y(y, y_type, (int64_t)(t + q) * y_ld + m, o);
  }
}

// NaN for tokens [c, end) of a tile at weight row m: in the cluster's partial tile (red: this row of [na][N][128]) or in y.
__device__ __noinline__ void lost_tokens(int c, int end, float* red, int N, int na, int t0, int T, int m, int rows, void* y, int y_type,
                                         int64_t y_ld) {
  for (; c < end; ++c) {
    if (red) {
      for (int a = 0; a < na; ++a) red[(size_t)(a * N + c) * 128] = __uint_as_float(kLost);
    } else if (m < rows && t0 + c < T) {
      store_y(y, y_type, (int64_t)(t0 + c) * y_ld + m, __uint_as_float(kLost));
    }
  }
}

// A CTA's share of the rows of a tile split over a cluster: the partial tiles red [NA][N][128] of the
// cluster's CTAs added in rank order (all of an element's requested before the first is used), scaled, stored.
template <int NA, int THREADS>
__device__ __forceinline__ void sum_splits(const float* red, int N, int splits, int rank, int m0, int rows, int t0, int T,
                                           float sw, float su, void* y, int y_type, int64_t y_ld) {
  const int rs = 128 / splits, rbeg = rank * rs;
  const uint32_t lred = smem_u32(red);
  for (int e = threadIdx.x; e < rs * N; e += THREADS) {
    const int c = e / rs, r = rbeg + (e - c * rs);
    float p[NA][8];
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        p[a][q] = 0.f;
        if (q < splits) {
          uint32_t ra;
          asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(ra) : "r"(lred + (uint32_t)((a * N + c) * 128 + r) * 4u), "r"(q));
          asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p[a][q]) : "r"(ra) : "memory");
        }
      }
    float sum[NA];
#pragma unroll
    for (int a = 0; a < NA; ++a)
      sum[a] = ((p[a][0] + p[a][1]) + (p[a][2] + p[a][3])) + ((p[a][4] + p[a][5]) + (p[a][6] + p[a][7]));
    const int t = t0 + c;
    if (m0 + r >= rows || t >= T) continue;
    float o = sum[0] * sw;
    if (NA == 2) o = silu_mul(o, sum[NA - 1] * su);
    store_y(y, y_type, (int64_t)t * y_ld + m0 + r, o);
  }
}

// ---------------------------------------------------------------------------
// Coded activations: both operands go to the tensor core as they are stored.
// ---------------------------------------------------------------------------
// The kernels that allocate tensor memory ask for all of an SM's shared memory, whatever their rings need: two CTAs on
// one SM, each of a cluster (of this kernel or of another stream's) whose CTAs wait for one another, could otherwise
// hold the tensor memory that the other's cluster waits for.
constexpr int kAllShared = 227 * 1024;

constexpr int kCodedThreads = 320;   // warp 0: copies, warp 1: scales and MMA, warps 2-9: epilogue

struct CodedArgs {
  int T, rows, cols;
  int N;             // tokens of a tile: the MMA's N
  int mt, ntiles;    // 128-row tiles, tiles in all
  int nbuf;          // accumulators in tensor memory
  int nst, sps;      // stages of the whole product, of a split
  int splits;        // CTAs of a cluster, one per range of stages
  int stages;        // ring depth
  uint32_t stage;    // bytes of a stage
  int tiles;         // 512-byte scale tiles across a row
  const uint8_t* ws;
  const uint8_t* us;
  const uint8_t* xs;
  float sw, su;
  void* y;
  int y_type;
  int64_t y_ld;
  long long spin;    // bound of the waits, in SM clocks
  int lose;          // testing hook: the first CTA's ring never reports its first slot free
  int* status;
};

// The product's floor is the MMAs': 128 rows x 256 tokens x 64 columns take 128 clocks of the tensor core (9.8 PFLOP/s
// on all SMs).  14336 rows x 4096, 8192 tokens to bf16: 181 us, 5.3 PFLOP/s; 512 tokens 23 us.  What bounds it is the
// tiles' way from L2 to the SMs: loads alone 175 us, MMAs alone 125 (100, and the turn of the accumulator: one of 256
// tokens leaves no room for a second beside the scales).  Every CTA loads its own tiles: the library also runs as
// replicas on several GPUs, which rules out loads spread over a cluster (with them 166 us).
// Few tokens: 4096 x 14336, 1 token 9.9 us, 14336 x 4096, 8 tokens 9.3 (floor 4.9: the codes' bytes; 112 of 152 SMs have
// a row tile).
//
// 128 weight rows x N tokens a CTA at a time (with GLU 128 rows of both matrices).  Codes come by TMA, 256 columns
// a stage, scale tiles by bulk copies; the MMA warp moves a stage's scales into tensor memory (columns of the
// stage's own, so that the ring's barriers order their reuse) and issues the block-scaled products.  It runs
// converged, with one lane's predicate on the instructions, so that their operands stay in uniform registers, and
// copies whole stages (scale tiles that the matrix does not have are what an earlier stage left: no product reads
// them): with a loop of one lane over the tiles that exist, a copy of 512 bytes took 74 clocks.  CTAs stay for
// all their tiles; the ring runs on while eight warps empty the accumulator.  With few tiles the columns are
// split over a cluster, whose CTAs add their partial tiles through distributed shared memory in rank order.
// G: groups of 128 tokens of a tile.
template <int FMT, bool GLU, int G>
__global__ void __launch_bounds__(kCodedThreads, 1)
    k_micro_coded(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap,
                  const __grid_constant__ CUtensorMap xmap, const __grid_constant__ CodedArgs g) {
  constexpr bool E8 = FMT == BITSMOE_MICRO_E8M0;
  constexpr int NA = GLU ? 2 : 1;
  constexpr int CPS = E8 ? 2 : 4;   // scale tiles of a stage's 256 columns
  constexpr uint32_t kSfCols = (NA + G) * CPS * 4;
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int S = g.stages, N = g.N;
  const uint32_t ring = (uint32_t)S * g.stage, redb = g.splits > 1 ? (uint32_t)(NA * N) * 512u : 0u;
  float* red = reinterpret_cast<float*>(sm);   // split: [NA][N][128], reuses the ring once the MMAs are done
  uint64_t* full = reinterpret_cast<uint64_t*>(sm + (ring > redb ? ring : redb));
  uint64_t* empty = full + S;
  uint64_t* afull = empty + S;
  uint64_t* aempty = afull + 2;
  uint64_t* drained = aempty + 2;   // after a wait of the MMA warp that ran out: the MMAs that it had issued
  uint64_t* quiet = drained + 1;    // nothing more is written to the rings
  uint32_t* slot = reinterpret_cast<uint32_t*>(quiet + 1);
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = blockIdx.y;
  const int st0 = rank * g.sps, nk = max(0, min(g.sps, g.nst - st0));
  const uint32_t b_bytes = (uint32_t)N * 128, sf_off = NA * kCodeTile + b_bytes;

  if (tid == 0) {
    prefetch_map(&wmap);
    prefetch_map(&xmap);
    if (GLU) prefetch_map(&umap);
    for (int i = 0; i < S; ++i) {
      mbar_init_n(full + i, 1);
      mbar_init_n(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init_n(afull + i, 1);
      mbar_init_n(aempty + i, 8);
    }
    mbar_init_n(drained, 1);
    mbar_init_n(quiet, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (wid == 1) tmem_alloc(slot, 512);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *slot, 0);
  bool ok = true;

  if (wid == 0) {
    if (lane == 0) {
      int st = 0, u = 0, n = 0;
      for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x) {
        const int mi = tile % g.mt, t0 = tile / g.mt * N;
        const int nbg = min(G, (g.T + 127) / 128 - t0 / 128);   // the tokens' scale groups that exist
        for (int i = 0; i < nk; ++i, ++n) {
          if (u > 0) ok = mbar_wait(empty + st, (uint32_t)(u - 1) & 1u, g.spin);
          if (!ok) break;
          const int kb = st0 + i, cnt = min(CPS, g.tiles - kb * CPS);
          uint8_t* base = sm + (size_t)st * g.stage;
          uint8_t* sf = base + sf_off;
          const uint32_t bar = smem_u32(full + st), sb = (uint32_t)cnt * 512u;
          const size_t at = ((size_t)mi * g.tiles + (size_t)kb * CPS) * 512;
          mbar_expect_tx(full + st, NA * kCodeTile + b_bytes + (uint32_t)(NA + nbg) * sb);
          tma_load_2d(smem_u32(base), &wmap, kb * 128, mi * 128, bar);
          if (GLU) tma_load_2d(smem_u32(base) + kCodeTile, &umap, kb * 128, mi * 128, bar);
          tma_load_2d(smem_u32(base) + NA * kCodeTile, &xmap, kb * 128, t0, bar);
          bulk_g2s(sf, g.ws + at, sb, full + st);
          if (GLU) bulk_g2s(sf + CPS * 512, g.us + at, sb, full + st);
          for (int j = 0; j < nbg; ++j)
            bulk_g2s(sf + (NA + j) * CPS * 512, g.xs + ((size_t)(t0 / 128 + j) * g.tiles + (size_t)kb * CPS) * 512, sb, full + st);
          if (++st == S) {
            st = 0;
            ++u;
          }
        }
      }
      for (int j = max(0, n - S); j < n; ++j) mbar_wait(full + j % S, (uint32_t)(j / S) & 1u);   // copies in flight
      mbar_arrive(quiet);
    }
    __syncwarp();
  } else if (wid == 1) {
    const uint32_t one = elect_one();
    const int nk64 = (g.cols + 63) / 64;
    const uint64_t da = sw128_desc(smem_u32(sm)), db = sw128_desc(smem_u32(sm) + NA * kCodeTile);
    const uint64_t ds = scale_desc(smem_u32(sm) + sf_off);
    const uint32_t sstep = g.stage >> 4, id0 = idesc_e2m1(N, E8, 0), id2 = idesc_e2m1(N, E8, 2);
    const uint32_t sf0 = tmem + (uint32_t)(g.nbuf * NA * N);
    int st = 0, u = 0, it = 0;
    for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x, ++it) {
      const int buf = it % g.nbuf, used = it / g.nbuf;
      if (used > 0) ok = mbar_wait(aempty + buf, (uint32_t)(used - 1) & 1u, g.spin);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const uint32_t acc = tmem + (uint32_t)(buf * NA * N);
      for (int i = 0; i < nk; ++i) {
        ok = mbar_wait(full + st, (uint32_t)u & 1u, g.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t so = (uint64_t)((uint32_t)st * sstep);
        const uint64_t a0 = da + so, b0 = db + so, s0 = ds + so;
        const uint32_t ta = sf0 + (uint32_t)st * kSfCols, tb = ta + NA * CPS * 4;
#pragma unroll
        for (int q = 0; q < CPS; ++q) {
#pragma unroll
          for (int a = 0; a < NA; ++a) tmem_copy_scales(one, ta + (a * CPS + q) * 4, s0 + (a * CPS + q) * 32);
#pragma unroll
          for (int j = 0; j < G; ++j) tmem_copy_scales(one, tb + (q * G + j) * 4, s0 + ((NA + j) * CPS + q) * 32);
        }
        const int k64 = nk64 - (st0 + i) * 4;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k >= k64) break;
          const int q = E8 ? k >> 1 : k;
#pragma unroll
          for (int a = 0; a < NA; ++a)
            mma_e2m1<E8>(one, acc + (uint32_t)(a * N), a0 + a * (kCodeTile >> 4) + 2 * k, b0 + 2 * k, E8 && (k & 1) ? id2 : id0,
                         ta + (a * CPS + q) * 4, tb + (q * G) * 4, (uint32_t)(i | k));
        }
        if (!(g.lose && i == 0 && it == 0 && (blockIdx.x | blockIdx.y) == 0)) mma_commit(one, empty + st);
        if (++st == S) {
          st = 0;
          ++u;
        }
      }
      if (!ok) break;
      mma_commit(one, afull + buf);
    }
    if (!ok) {
      mma_commit(one, drained);
      mbar_wait(drained, 0u);
    }
  } else {
    const int r = 32 * (wid & 3) + lane, half = (wid - 2) >> 2;
    const int nh = (N / 16 + 1) / 2 * 16;   // columns of the first half
    int it = 0;
    for (int tile = blockIdx.x; tile < g.ntiles; tile += gridDim.x, ++it) {
      const int buf = it % g.nbuf, used = it / g.nbuf;
      if (ok) ok = mbar_wait_idle(afull + buf, (uint32_t)used & 1u, g.spin);
      ok = __all_sync(0xFFFFFFFFu, ok);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int m = tile % g.mt * 128 + r, t0 = tile / g.mt * N;
      if (!ok) {
        if (g.splits > 1) mbar_wait_idle(quiet, 0u, 4 * (g.spin + kWaitClocks));   // (the partial tile lies in the rings)
        lost_tokens(half ? nh : 0, half ? N : nh, g.splits > 1 ? red + r : nullptr, N, NA, t0, g.T, m, g.rows, g.y, g.y_type, g.y_ld);
        continue;
      }
      const uint32_t tl = tmem + ((uint32_t)(32 * (wid & 3)) << 16) + (uint32_t)(buf * NA * N);
      // the accumulator goes to registers first: the next tile's products run while this one is stored
      constexpr int kChunks = G * 128 / 32;   // of 16 columns, at most, of a half
      uint32_t v[kChunks][NA][16];
      const int first = half ? nh : 0, last = half ? N : nh;
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          if (nk > 0 && first + c * 16 < last) {
            tmem_ld16(tl + (uint32_t)(a * N + first + c * 16), v[c][a]);
          } else {
#pragma unroll
            for (int q = 0; q < 16; ++q) v[c][a][q] = 0u;
          }
        }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      mbar_arrive(lane == 0, aempty + buf);
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int c0 = first + c * 16;
        if (c0 >= last) break;
        if (g.splits > 1) {
#pragma unroll
          for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int q = 0; q < 16; ++q) red[(size_t)(a * N + c0 + q) * 128 + r] = __uint_as_float(v[c][a][q]);
        } else if (m < g.rows) {
          store_tokens<NA>(v[c], t0 + c0, g.T, m, g.sw, g.su, g.y, g.y_type, g.y_ld);
        }
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (g.splits > 1) {
    // every CTA of the cluster has its partial tile in shared memory; this CTA's share of the rows is summed
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    const int tile = blockIdx.x;
    sum_splits<NA, kCodedThreads>(red, N, g.splits, rank, tile % g.mt * 128, g.rows, tile / g.mt * N, g.T, g.sw, g.su, g.y, g.y_type, g.y_ld);
    // no CTA leaves while others may still read its shared memory
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  } else {
    __syncthreads();
  }
  if (!ok && g.status) atomicCAS(g.status, 0, BITSMOE_ERR_TIMEOUT);
  if (wid == 1) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    tmem_dealloc(tmem, 512);
  }
}

template <int FMT, bool GLU, int G>
cudaError_t launch_coded_g(const bitsmoe_microscale* w, const bitsmoe_microscale* up, const bitsmoe_microscale* xq, CodedArgs g,
                           int dev, int sms, cudaStream_t st) {
  constexpr int NA = GLU ? 2 : 1, CPS = FMT == BITSMOE_MICRO_E8M0 ? 2 : 4;
  g.mt = (g.rows + 127) / 128;
  g.ntiles = g.mt * ((g.T + g.N - 1) / g.N);
  g.nst = (g.cols + kStageK - 1) / kStageK;
  int splits = 1;
  while (splits < 8 && (int64_t)g.ntiles * splits * 2 <= sms && g.nst >= 2 * splits) splits *= 2;
  g.splits = splits;
  g.sps = (g.nst + splits - 1) / splits;
  g.stage = (NA * kCodeTile + (uint32_t)g.N * 128 + (uint32_t)((NA + G) * CPS) * 512 + 1023) / 1024 * 1024;
  const int sf_cols = (NA + G) * CPS * 4;
  const int fit = std::min((int)(216 * 1024 / g.stage), 16);
  // two accumulators where tensor memory holds them beside the scales of every stage
  g.nbuf = splits == 1 && 2 * NA * g.N + fit * sf_cols <= 512 ? 2 : 1;
  g.stages = std::min(fit, (512 - g.nbuf * NA * g.N) / sf_cols);
  const size_t ring = (size_t)g.stages * g.stage, redb = splits > 1 ? (size_t)NA * g.N * 512 : 0;
  if (1024 + std::max(ring, redb) + (size_t)(2 * g.stages + 6) * 8 + 4 > kAllShared) return cudaErrorInvalidValue;
  CUtensorMap wm, um, xm;
  const int64_t pitch = micro_pitch(g.cols);
  if (!make_row_map(&wm, true, w->codes, g.rows, pitch, pitch, 128) || !make_row_map(&xm, true, xq->codes, g.T, pitch, pitch, g.N))
    return cudaErrorInvalidValue;
  um = wm;
  if (GLU && !make_row_map(&um, true, up->codes, g.rows, pitch, pitch, 128)) return cudaErrorInvalidValue;
  auto kern = k_micro_coded<FMT, GLU, G>;
  cudaError_t e = allow_shared<k_micro_coded<FMT, GLU, G>>(dev, kAllShared);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = (unsigned)splits;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(splits > 1 ? g.ntiles : std::min(g.ntiles, sms)), (unsigned)splits, 1);
  cfg.blockDim = dim3(kCodedThreads);
  cfg.dynamicSmemBytes = kAllShared;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, wm, um, xm, g);
}

template <int FMT, bool GLU>
cudaError_t launch_coded(const bitsmoe_microscale* w, const bitsmoe_microscale* up, const bitsmoe_microscale* xq, CodedArgs g,
                         int dev, int sms, cudaStream_t st) {
  g.N = std::min((g.T + 15) / 16 * 16, GLU ? 128 : 256);   // past one tile a multiple of the scale tiles' 128
  if constexpr (!GLU) {
    if (g.N > 128) return launch_coded_g<FMT, GLU, 2>(w, up, xq, g, dev, sms, st);
  }
  return launch_coded_g<FMT, GLU, 1>(w, up, xq, g, dev, sms, st);
}

// ---------------------------------------------------------------------------
// Many 16-bit activations: the codes become bf16 tiles in shared memory.
//
// A CTA takes 128 weight rows (with GLU of both matrices) x N tokens at a time.
// Warp 0 brings codes and scale tiles (256 columns a stage) into one ring.  Two
// groups of eight warps, which take the slots of a second ring in turn, turn them
// into bf16 tiles of 64 columns, code times block scale (exact: at most 6
// significant bits); warp 2 brings the activations of the same columns into the
// same slots by TMA.  Warp 1 issues tcgen05.mma (kind::f16), and four warps
// empty the accumulators, two of them in turn where tensor memory holds two, so
// that the next tile's products run meanwhile.  CTAs stay for all their tiles.
// With few tiles the columns are split over a cluster instead.
//
// 14336 rows x 4096, 4096 tokens: 307 us, 1.56 PFLOP/s (floor 244 at the library's
// measured bf16 rate); 2048 tokens with SwiGLU 385 us; 64 tokens 25 us.  A slot
// of 64 columns x 256 tokens takes 650 to 770 clocks, its MMAs 512: shared memory
// serves the tiles' writes beside the MMAs' reads (253 us without the writes,
// 193 without decoding; the conversions alone need 200 clocks of a slot).
// ---------------------------------------------------------------------------
constexpr int kDecodeWarps = 8, kDecodeGroups = 2;   // groups of eight warps that take the slots in turn
constexpr int kWideThreads = 32 * (4 + kDecodeGroups * kDecodeWarps + 4);   // warps: 0 codes, 1 MMA, 2 activations, 4.. decode, epilogue

struct WideArgs {
  int T, rows, cols, tiles;
  int N, mt, ntiles, nbuf;
  int nst, sps, splits;
  int P, Q;              // depths of the rings of codes and of tiles
  uint32_t pst;          // bytes of a stage of codes
  int btma;              // x's rows are on 16-byte boundaries
  const uint8_t* ws;
  const uint8_t* us;
  const __nv_bfloat16* x;
  int64_t x_ld;
  float sw, su;
  void* y;
  int y_type;
  int64_t y_ld;
  long long spin;
  int lose;
  int* status;
};

// 32 codes (four words) of one row times their block scales -> 64 bytes of bf16 in a 128-byte swizzled tile.  Codes
// become fp16 pairs by one conversion each and bf16 pairs by way of fp32; their products with the scales are exact
// in bf16 (at most 6 significant bits; E8M0's largest scales overflow as fp32 does): 8 operations of the integer
// pipe for 8 codes, where moving the bits into place takes 17.
template <int FMT>
__device__ __forceinline__ void decode32(const uint4& v, uint32_t sc, uint8_t* row, int half, int r7) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  uint32_t f[2];
  if constexpr (FMT == BITSMOE_MICRO_E8M0) {
    asm("cvt.rn.bf16x2.ue8m0x2 %0, %1;" : "=r"(f[0]) : "h"((uint16_t)((sc & 255u) * 0x101u)));
    f[1] = f[0];
  } else {
    const uint32_t p = e4m3x2_f16(sc);
    f[0] = __float_as_uint(f16lo(p)) >> 16;   // 4 significant bits: exact
    f[1] = __float_as_uint(f16hi(p)) >> 16;
    f[0] |= f[0] << 16;
    f[1] |= f[1] << 16;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    uint32_t h[4], o[4];
    code_pairs<false>(w[q], h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 c = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
      const __nv_bfloat162 b = __floats2bfloat162_rn(c.x, c.y);
      o[i] = mul2<true>(*reinterpret_cast<const uint32_t*>(&b), f[q >> 1]);
    }
    *reinterpret_cast<uint4*>(row + (((half * 4 + q) ^ r7) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// KS: steps of 64 columns in a slot (two where tokens are few: a slot's barriers cost the MMA warp about 350 clocks,
// as long as the products of 64 columns with 128 tokens).
template <int FMT, bool GLU, int KS>
__global__ void __launch_bounds__(kWideThreads, 1)
    k_micro_wide(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap,
                 const __grid_constant__ CUtensorMap xmap, const __grid_constant__ WideArgs g) {
  constexpr bool E8 = FMT == BITSMOE_MICRO_E8M0;
  constexpr int NA = GLU ? 2 : 1, CPS = E8 ? 2 : 4;
  constexpr int kSlots = 4 / KS;   // slots of a stage of codes
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const int P = g.P, Q = g.Q, N = g.N;
  constexpr uint32_t kATile = NA * kCodeTile;   // 128 rows x 64 bf16, as many bytes as 256 columns of codes
  const uint32_t b_bytes = (uint32_t)N * 128, step = kATile + b_bytes, qst = KS * step;   // a step: weights, activations
  uint8_t* pring = sm + (size_t)Q * qst;
  float* red = reinterpret_cast<float*>(sm);   // split: [NA][N][128], reuses the rings
  uint64_t* pfull = reinterpret_cast<uint64_t*>(pring + (size_t)P * g.pst);
  uint64_t* pempty = pfull + P;
  uint64_t* qfull = pempty + P;
  uint64_t* qempty = qfull + Q;
  uint64_t* afull = qempty + Q;
  uint64_t* aempty = afull + 2;
  uint64_t* drained = aempty + 2;   // after a wait of the MMA warp that ran out: the MMAs that it had issued
  uint64_t* quiet = drained + 1;    // nothing more is written to the rings
  uint32_t* slot = reinterpret_cast<uint32_t*>(quiet + 1);
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = blockIdx.y;
  const int st0 = rank * g.sps, nk = max(0, min(g.sps, g.nst - st0));
  const int s0 = st0 * 4, n64 = max(0, min(nk * 4, (g.cols + 63) / 64 - s0));   // this CTA's steps of 64 columns
  const int ns = (n64 + KS - 1) / KS;                                            // and slots

  if (tid == 0) {
    prefetch_map(&wmap);
    prefetch_map(&xmap);
    if (GLU) prefetch_map(&umap);
    for (int i = 0; i < P; ++i) {
      mbar_init_n(pfull + i, 1);
      mbar_init_n(pempty + i, kDecodeGroups * kDecodeWarps);
    }
    for (int i = 0; i < Q; ++i) {
      mbar_init_n(qfull + i, kDecodeWarps + (g.btma ? 1 : 0));
      mbar_init_n(qempty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init_n(afull + i, 1);
      mbar_init_n(aempty + i, 4);
    }
    mbar_init_n(drained, 1);
    mbar_init_n(quiet, 2 + kDecodeGroups * kDecodeWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (wid == 1) tmem_alloc(slot, 512);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, *slot, 0);
  bool ok = true;

  if (wid == 0) {
    if (lane == 0) {
      int st = 0, u = 0, n = 0;
      for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x) {
        const int mi = tile % g.mt;
        for (int i = 0; i < nk; ++i, ++n) {
          if (u > 0) ok = mbar_wait(pempty + st, (uint32_t)(u - 1) & 1u, g.spin);
          if (!ok) break;
          const int kb = st0 + i, cnt = min(CPS, g.tiles - kb * CPS);
          uint8_t* base = pring + (size_t)st * g.pst;
          const uint32_t bar = smem_u32(pfull + st);
          mbar_expect_tx(pfull + st, NA * (kCodeTile + (uint32_t)cnt * 512u));
          tma_load_2d(smem_u32(base), &wmap, kb * 128, mi * 128, bar);
          if (GLU) tma_load_2d(smem_u32(base) + kCodeTile, &umap, kb * 128, mi * 128, bar);
          const size_t at = ((size_t)mi * g.tiles + (size_t)kb * CPS) * 512;
          bulk_g2s(base + NA * kCodeTile, g.ws + at, (uint32_t)cnt * 512u, pfull + st);
          if (GLU) bulk_g2s(base + NA * kCodeTile + CPS * 512, g.us + at, (uint32_t)cnt * 512u, pfull + st);
          if (++st == P) {
            st = 0;
            ++u;
          }
        }
      }
      for (int j = max(0, n - P); j < n; ++j) mbar_wait(pfull + j % P, (uint32_t)(j / P) & 1u);   // copies in flight
      mbar_arrive(quiet);
    }
    __syncwarp();
  } else if (wid == 1) {
    // converged, with one lane's predicate on the instructions: their operands stay in uniform registers (issued by
    // one lane of a diverged warp, the four products and the commit of a slot took 490 clocks)
    const uint32_t one = elect_one(), idesc = idesc_bf16(N);
    const uint64_t da = sw128_desc(smem_u32(sm)), db = sw128_desc(smem_u32(sm) + kATile);
    int st = 0, u = 0, it = 0;
    for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x, ++it) {
      const int buf = it % g.nbuf, use = it / g.nbuf;
      if (use > 0) ok = mbar_wait(aempty + buf, (uint32_t)(use - 1) & 1u, g.spin);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const uint32_t acc = tmem + (uint32_t)(buf * NA * N);
      for (int i = 0; i < ns; ++i) {
        ok = mbar_try_wait(qfull + st, (uint32_t)u & 1u) || mbar_wait(qfull + st, (uint32_t)u & 1u, g.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint64_t so = (uint64_t)((uint32_t)st * (qst >> 4)), a0 = da + so, b0 = db + so;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          if (s > 0 && i * KS + s >= n64) break;
          const uint64_t o = (uint64_t)((uint32_t)s * (step >> 4));
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int a = 0; a < NA; ++a)
              mma_f16(one, acc + (uint32_t)(a * N), a0 + o + a * (kCodeTile >> 4) + 2 * k, b0 + o + 2 * k, idesc, (uint32_t)(i | s | k));
        }
        if (!(g.lose && i == 0 && it == 0 && (blockIdx.x | blockIdx.y) == 0)) mma_commit(one, qempty + st);
        if (++st == Q) {
          st = 0;
          ++u;
        }
      }
      if (!ok) break;
      mma_commit(one, afull + buf);
    }
    if (!ok) {
      mma_commit(one, drained);
      mbar_wait(drained, 0u);
    }
  } else if (wid == 2) {
    if (lane == 0 && g.btma) {
      int st = 0, u = 0, n = 0;
      for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x) {
        const int t0 = tile / g.mt * N;
        for (int i = 0; i < ns; ++i, ++n) {
          if (u > 0) ok = mbar_wait(qempty + st, (uint32_t)(u - 1) & 1u, g.spin);
          if (!ok) break;
          const int cnt = min(KS, n64 - i * KS);
          mbar_expect_tx(qfull + st, (uint32_t)cnt * b_bytes);
          for (int s = 0; s < cnt; ++s)
            tma_load_2d(smem_u32(sm) + (uint32_t)st * qst + (uint32_t)s * step + kATile, &xmap, (s0 + i * KS + s) * 64, t0, smem_u32(qfull + st));
          if (++st == Q) {
            st = 0;
            ++u;
          }
        }
      }
      // copies in flight: their bytes end a phase only with the decoders' arrivals, which may be missing after a timeout
      for (int j = max(0, n - Q); j < n; ++j) mbar_wait(qfull + j % Q, (uint32_t)(j / Q) & 1u, ok ? kWaitClocks : g.spin);
    }
    mbar_arrive(lane == 0, quiet);
    __syncwarp();
  } else if (wid >= 4 && wid < 4 + kDecodeGroups * kDecodeWarps) {
    const int dw = (wid - 4) % kDecodeWarps, group = (wid - 4) / kDecodeWarps;
    const int r = 16 * dw + (lane & 15), half = lane >> 4, r7 = r & 7;
    const int bt = dw * 32 + lane;
    const uint8_t* code = pring + r * 128;
    const uint8_t* scale = pring + NA * kCodeTile + (r & 31) * 16 + (r >> 5) * 4;
    uint32_t ps = 0, pp = 0;                     // slot of the codes' ring and its phase's parity
    uint32_t qs = group, qp = 0;                 // and of the tiles' ring (at least as many slots as groups)
    int i = group;                               // this group's next slot, counted in the tile: every other of all tiles' slots
    for (int tile = blockIdx.x; tile < g.ntiles && ok; tile += gridDim.x, i -= ns) {
      const int t0 = tile / g.mt * N;
      for (int i0 = 0; i0 < ns && ok; i0 += kSlots) {   // a stage of codes
        ok = mbar_try_wait(pfull + ps, pp) || mbar_wait(pfull + ps, pp, g.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
        for (; i < min(i0 + kSlots, ns) && ok; i += kDecodeGroups) {
          const int sub = i - i0;
          ok = mbar_try_wait(qempty + qs, qp ^ 1u) || mbar_wait(qempty + qs, qp ^ 1u, g.spin);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            if (s > 0 && i * KS + s >= n64) break;
            const int q = sub * KS + s;   // step of the stage
            uint8_t* out = sm + (size_t)qs * qst + (size_t)s * step + r * 128;
#pragma unroll
            for (int a = 0; a < NA; ++a) {
              const uint4 v = *reinterpret_cast<const uint4*>(code + (size_t)ps * g.pst + (size_t)a * kCodeTile + (((2 * q + half) ^ r7) << 4));
              const uint8_t* sc = scale + (size_t)ps * g.pst + (a * CPS + (E8 ? q >> 1 : q)) * 512;
              const uint32_t f = E8 ? (uint32_t)sc[(q & 1) * 2 + half] : (uint32_t)*reinterpret_cast<const uint16_t*>(sc + half * 2);
              decode32<FMT>(v, f, out + (size_t)a * kCodeTile, half, r7);
            }
            if (!g.btma) {   // rows off 16-byte boundaries: 8 columns a thread at a time
              const int k0 = (s0 + i * KS + s) * 64;
              for (int c = bt; c < N * 8; c += kDecodeWarps * 32) {
                const int t = t0 + (c >> 3), k = k0 + (c & 7) * 8;
                const uint16_t* xr = reinterpret_cast<const uint16_t*>(g.x) + (int64_t)t * g.x_ld + k;
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const uint32_t lo = t < g.T && k + 2 * e < g.cols ? xr[2 * e] : 0u;
                  const uint32_t hi = t < g.T && k + 2 * e + 1 < g.cols ? xr[2 * e + 1] : 0u;
                  w[e] = lo | (hi << 16);
                }
                const int rr = c >> 3;
                *reinterpret_cast<uint4*>(sm + (size_t)qs * qst + (size_t)s * step + kATile + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) =
                    make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
          fence_proxy_async();   // generic writes -> tensor-core reads
          __syncwarp();
          mbar_arrive(lane == 0, qfull + qs);
          qs += kDecodeGroups;
          while (qs >= (uint32_t)Q) qs -= Q, qp ^= 1u;
        }
        __syncwarp();
        mbar_arrive(lane == 0 && ok, pempty + ps);
        if (++ps == (uint32_t)P) ps = 0, pp ^= 1u;
      }
    }
    __syncwarp();
    mbar_arrive(lane == 0, quiet);
  } else if (wid >= 4 + kDecodeGroups * kDecodeWarps) {
    const int r = 32 * (wid & 3) + lane;
    int it = 0;
    for (int tile = blockIdx.x; tile < g.ntiles; tile += gridDim.x, ++it) {
      const int buf = it % g.nbuf, use = it / g.nbuf;
      if (ok) ok = mbar_wait_idle(afull + buf, (uint32_t)use & 1u, g.spin);
      ok = __all_sync(0xFFFFFFFFu, ok);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int m = tile % g.mt * 128 + r, t0 = tile / g.mt * N;
      if (!ok) {
        if (g.splits > 1) mbar_wait_idle(quiet, 0u, 4 * (g.spin + kWaitClocks));
        lost_tokens(0, N, g.splits > 1 ? red + r : nullptr, N, NA, t0, g.T, m, g.rows, g.y, g.y_type, g.y_ld);
        continue;
      }
      const uint32_t tl = tmem + ((uint32_t)(32 * (wid & 3)) << 16) + (uint32_t)(buf * NA * N);
      for (int c0 = 0; c0 < N; c0 += 16) {
        uint32_t v[NA][16];
#pragma unroll
        for (int a = 0; a < NA; ++a) {
          if (n64 > 0) {
            tmem_ld16(tl + (uint32_t)(a * N + c0), v[a]);
          } else {
#pragma unroll
            for (int q = 0; q < 16; ++q) v[a][q] = 0u;
          }
        }
        if (g.splits > 1) {
#pragma unroll
          for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int q = 0; q < 16; ++q) red[(size_t)(a * N + c0 + q) * 128 + r] = __uint_as_float(v[a][q]);
        } else if (m < g.rows) {
          store_tokens<NA>(v, t0 + c0, g.T, m, g.sw, g.su, g.y, g.y_type, g.y_ld);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      mbar_arrive(lane == 0, aempty + buf);
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  if (g.splits > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
    const int tile = blockIdx.x;
    sum_splits<NA, kWideThreads>(red, N, g.splits, rank, tile % g.mt * 128, g.rows, tile / g.mt * N, g.T, g.sw, g.su, g.y, g.y_type, g.y_ld);
    // no CTA leaves while others may still read its shared memory
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
  } else {
    __syncthreads();
  }
  if (!ok && g.status) atomicCAS(g.status, 0, BITSMOE_ERR_TIMEOUT);
  if (wid == 1) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    tmem_dealloc(tmem, 512);
  }
}

template <int FMT, bool GLU, int KS>
cudaError_t launch_wide_k(const bitsmoe_microscale* w, const bitsmoe_microscale* up, WideArgs g, int dev, int sms, cudaStream_t st) {
  constexpr int NA = GLU ? 2 : 1, CPS = FMT == BITSMOE_MICRO_E8M0 ? 2 : 4;
  constexpr uint32_t kRoom = 216 * 1024;
  const int tt = (g.T + g.N - 1) / g.N;
  g.mt = (g.rows + 127) / 128;
  g.ntiles = g.mt * tt;
  g.nbuf = 2 * NA * g.N <= 512 ? 2 : 1;
  g.nst = (g.cols + kStageK - 1) / kStageK;
  g.pst = (uint32_t)NA * (kCodeTile + CPS * 512);
  const uint32_t qst = (uint32_t)KS * (NA * kCodeTile + (uint32_t)g.N * 128);
  g.Q = std::min<int>(4, (kRoom - 2 * g.pst) / qst);
  // A group of decoders steps by as many slots as there are groups; with fewer slots it would wait for a phase two
  // ahead of the one in progress, which a wait by parity takes for complete.
  if (g.Q < kDecodeGroups) return cudaErrorInvalidValue;
  g.P = std::min<int>(8, (kRoom - g.Q * qst) / g.pst);
  const uint32_t rings = g.Q * qst + g.P * g.pst;
  int splits = 1;
  while (splits < 8 && (int64_t)g.ntiles * splits * 2 <= sms && g.nst >= 2 * splits && (uint32_t)(NA * g.N) * 512u <= rings) splits *= 2;
  g.splits = splits;
  g.sps = (g.nst + splits - 1) / splits;
  if (1024 + (size_t)rings + (size_t)(2 * g.P + 2 * g.Q + 6) * 8 + 4 > kAllShared) return cudaErrorInvalidValue;
  const int64_t pitch = micro_pitch(g.cols);
  CUtensorMap wm, um, xm;
  if (!make_row_map(&wm, true, w->codes, g.rows, pitch, pitch, 128)) return cudaErrorInvalidValue;
  um = xm = wm;
  if (GLU && !make_row_map(&um, true, up->codes, g.rows, pitch, pitch, 128)) return cudaErrorInvalidValue;
  g.btma = (uintptr_t)g.x % 16 == 0 && (g.x_ld % 8 == 0 || g.T == 1);
  if (g.btma) g.btma = make_row_map(&xm, false, g.x, g.T, g.cols, g.T == 1 ? (g.cols * 2 + 15) / 16 * 16 : g.x_ld * 2, g.N);
  auto kern = k_micro_wide<FMT, GLU, KS>;
  cudaError_t e = allow_shared<k_micro_wide<FMT, GLU, KS>>(dev, kAllShared);
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 1;
  attr[0].val.clusterDim.y = (unsigned)splits;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(splits > 1 ? g.ntiles : std::min(g.ntiles, sms)), (unsigned)splits, 1);
  cfg.blockDim = dim3(kWideThreads);
  cfg.dynamicSmemBytes = kAllShared;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = splits > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, wm, um, xm, g);
}

template <int FMT, bool GLU>
cudaError_t launch_wide(const bitsmoe_microscale* w, const bitsmoe_microscale* up, WideArgs g, int dev, int sms, cudaStream_t st) {
  // at most 256 tokens a tile, with GLU 128 (two accumulators in turn; three slots fit)
  const int most = GLU ? 128 : 256, tt = (g.T + most - 1) / most;
  g.N = ((g.T + tt - 1) / tt + 15) / 16 * 16;
  // two steps a slot where three such slots fit beside two stages of codes
  if constexpr (!GLU) {
    if (g.N <= 96) return launch_wide_k<FMT, GLU, 2>(w, up, g, dev, sms, st);
  }
  return launch_wide_k<FMT, GLU, 1>(w, up, g, dev, sms, st);
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
    // the sums are multiplied by the two tensor scales' product
    if (!std::isnormal(w->scale * xq->scale) || (up && !std::isnormal(up->scale * xq->scale))) return BITSMOE_ERR_INVALID_ARG;
  } else if (x_ld < w->cols) {
    return BITSMOE_ERR_INVALID_ARG;
  }
  if (T == 0 || w->rows == 0) return BITSMOE_OK;
  if ((!x && !xq) || !y) return BITSMOE_ERR_INVALID_ARG;
  if ((uintptr_t)x % 2 || (uintptr_t)y % dense_size(y_type) || (uintptr_t)status % 4) return BITSMOE_ERR_ALIGNMENT;
  if ((int64_t)((w->rows + 127) / 128) * ((T + 127) / 128) >= (1ll << 31)) return BITSMOE_ERR_SHAPE;
  const float sx = xq ? xq->scale : 1.f;
  const long long spin = debug_wait_clocks() > 0 ? debug_wait_clocks() : kWaitClocks;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int dev = 0, sms = 0;
  cudaError_t e = device_sms(&dev, &sms);
  if (e != cudaSuccess) return record_cuda_error((int)e);
  const bool e8 = w->format == BITSMOE_MICRO_E8M0;
  FewPlan fp;
  if (few_plan(w->format, up != nullptr, xq != nullptr, T, w->rows, w->cols, few_resident, &fp)) {
    FewArgs f;
    std::memset(&f, 0, sizeof(f));
    f.T = T;
    f.rows = w->rows;
    f.cols = w->cols;
    f.tiles = micro_tiles(w->format, w->cols);
    f.ws = w->scales;
    f.us = up ? up->scales : nullptr;
    f.x = static_cast<const __nv_bfloat16*>(x);
    f.x_ld = x_ld;
    f.x_vec = (uintptr_t)x % 16 == 0 && x_ld % 8 == 0;
    f.xq = mat_of(xq);
    f.sw = w->scale * sx;
    f.su = up ? up->scale * sx : 0.f;
    f.y = y;
    f.y_type = y_type;
    f.y_ld = y_ld;
    f.spin = spin;
    f.lose = debug_skip_arrival();
    f.status = status;
    if (e8) e = up ? launch_few_nt<BITSMOE_MICRO_E8M0, true>(fp, w, up, f, dev, st) : launch_few_nt<BITSMOE_MICRO_E8M0, false>(fp, w, up, f, dev, st);
    else e = up ? launch_few_nt<BITSMOE_MICRO_E4M3, true>(fp, w, up, f, dev, st) : launch_few_nt<BITSMOE_MICRO_E4M3, false>(fp, w, up, f, dev, st);
    return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
  }
  if (xq) {
    CodedArgs c;
    std::memset(&c, 0, sizeof(c));
    c.T = T;
    c.rows = w->rows;
    c.cols = w->cols;
    c.tiles = micro_tiles(w->format, w->cols);
    c.ws = w->scales;
    c.us = up ? up->scales : nullptr;
    c.xs = xq->scales;
    c.sw = w->scale * sx;
    c.su = up ? up->scale * sx : 0.f;
    c.y = y;
    c.y_type = y_type;
    c.y_ld = y_ld;
    c.spin = spin;
    c.lose = debug_skip_arrival();
    c.status = status;
    if (e8)
      e = up ? launch_coded<BITSMOE_MICRO_E8M0, true>(w, up, xq, c, dev, sms, st) : launch_coded<BITSMOE_MICRO_E8M0, false>(w, up, xq, c, dev, sms, st);
    else
      e = up ? launch_coded<BITSMOE_MICRO_E4M3, true>(w, up, xq, c, dev, sms, st) : launch_coded<BITSMOE_MICRO_E4M3, false>(w, up, xq, c, dev, sms, st);
    return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
  }
  WideArgs a;
  std::memset(&a, 0, sizeof(a));
  a.T = T;
  a.rows = w->rows;
  a.cols = w->cols;
  a.tiles = micro_tiles(w->format, w->cols);
  a.ws = w->scales;
  a.us = up ? up->scales : nullptr;
  a.x = static_cast<const __nv_bfloat16*>(x);
  a.x_ld = x_ld;
  a.sw = w->scale;
  a.su = up ? up->scale : 0.f;
  a.y = y;
  a.y_type = y_type;
  a.y_ld = y_ld;
  a.spin = spin;
  a.lose = debug_skip_arrival();
  a.status = status;
  if (e8) e = up ? launch_wide<BITSMOE_MICRO_E8M0, true>(w, up, a, dev, sms, st) : launch_wide<BITSMOE_MICRO_E8M0, false>(w, up, a, dev, sms, st);
  else e = up ? launch_wide<BITSMOE_MICRO_E4M3, true>(w, up, a, dev, sms, st) : launch_wide<BITSMOE_MICRO_E4M3, false>(w, up, a, dev, sms, st);
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
