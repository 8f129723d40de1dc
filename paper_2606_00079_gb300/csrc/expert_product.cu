// Products grouped by expert, ragged: for offsets[e] <= p < offsets[e + 1]
//
//   y[p][r] = sum_k W_e[r][k] x[q][k]        (q = p, or index[p] / fan)
//   or, with a second set of matrices U, SiLU(W_e x) * (U_e x)
//
// in bf16, or in 8 bits (E4M3) with a scale a row on both sides, which multiplies the finished sum.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <type_traits>

#include "microscale.cuh"
#include "tc.cuh"

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
  int w_vec, x_vec;      // rows of the matrices, rows of x start on 16-byte boundaries
  void* y;
  int y_vec;             // bf16 rows on 16-byte boundaries
  int64_t y_ld;
  int nk, stages, nbuf;  // tensor cores: steps of 128 bytes of the columns, depth of the ring, accumulators in turn
  int splits, sps;       // CTAs that share the columns of a tile, steps of each
  int chain;             // steps that an accumulator takes (fp32 results: a few)
  int w_next, u_next;    // 1: an expert has matrices of its own (0: one stands for all)
  long long spin;
  int lose, lose_plan;   // testing hook: block 0 leaves out an arrival (a stage's, the plan's)
  int* status;
};

__device__ __forceinline__ void keep(float* y, float v) { *y = v; }
__device__ __forceinline__ void keep(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }

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
// A CTA has two tiles of 128 rows of an expert's matrix (with U 128 of each, so that
// both products of a result are in one lane) and up to 256 rows of y: the matrix is the operand of many rows, so that an
// expert's few rows cost an MMA of few columns.  With many rows two CTAs are a pair (cta_group::2): each brings half of the
// rows of x for both.
//
// A ring of stages of 128 bytes of the columns: warp 0 brings the matrices' tiles by TMA, four warps the rows of x, wherever
// they are, 16 bytes a thread at a time (cp.async; TMA's gather of four rows took 63 clocks for 512 bytes); their copies arrive
// on a barrier by themselves (of a pair warp 2 hands that on to the first CTA).  Warp 1 (of a pair's first CTA) issues the MMAs;
// eight warps empty the accumulators, two of them in turn where tensor memory holds two.  CTAs stay for all their tiles.  With
// few tiles the columns are split over a cluster, whose CTAs add their partial tiles through distributed shared memory in rank
// order.
//
// Gate and up of 128 experts of 768 x 2048 in bf16 (the kernel alone, replayed from a graph): 8192 tokens 300 us (1.4 PFLOP/s;
// the card's power bounds it, at a stretch 337), 32 tokens 85, one 13.9 with its matrices from DRAM (11.7 from L2); 8 tokens 54
// under a profiler (the matrices of the experts that have one, 302 MB: DRAM).  A matrix of 8 experts of 14336 x 4096 in 8 bits,
// 8192 rows: 333 us, 2.9 PFLOP/s (at a stretch 381).
// ---------------------------------------------------------------------------
// Warps: 0 matrices, 1 MMA, 2 rows of x that are there (of a pair), 3 the tiles to come (of a pair), four of rows of x, eight of
// results.  (Eight of x's fill a stage faster, 685 clocks in place of 780 of the MMAs' 1024, but many large products are bound
// by the card's power, and warps that wait draw it: 4096 rows of y of 14336 x 4096 in 8 bits at a stretch 386 us with eight, 380
// with four.)
constexpr int kXWarps = 4, kOutWarps = 8, kOutThreads = 32 * kOutWarps;
constexpr int kTcThreads = 32 * (4 + kXWarps + kOutWarps);
constexpr int kFewRows = 64;                 // rows of y of a tile from which on pairs take it
constexpr int kSumRows = 128;                // rows of y of a tile of many fp32 results
constexpr int kSumRegs = 184, kOtherRegs = 72;   // registers of the warps that hold their sums, and of the others (128 at launch)
static_assert(32 * kOutWarps * kSumRegs + 32 * (4 + kXWarps) * kOtherRegs <= 128 * kTcThreads && kOutWarps % 4 == 0 && kXWarps % 4 == 0, "");
constexpr int kStagesMost = 8, kAccumulators = 4;
constexpr long long kCopyClocks = 1 << 21;   // what a copy in flight is given where a wait has run out (1 ms)
constexpr uint32_t kATile = 2 * 128 * 128;   // bytes of a stage's tiles of the matrices
constexpr int kTcShared = 227 * 1024;        // (all of an SM's, as of every kernel that allocates tensor memory)
constexpr int kXRows = 4 * kXWarps;          // rows that one pass of x's warps brings

// Pairs take the tiles in waves, a tile each.  Tiles differ (an expert's rows, shared among its tiles): in turn, the pair with
// the most work had 10 to 15 % more than the average.  So warp 3 gives the largest tiles of a wave to the pairs that have had the
// least so far.  Every CTA works that out for itself, for all pairs, ahead of its tiles.
constexpr int kPairsMost = 96, kAhead = 4;   // waves whose tiles are known ahead
struct Plan {
  alignas(16) int2 of[kPairsMost];   // keys of the tiles of a wave, and the pairs' loads
  int by_rank[kPairsMost];           // work by the tiles' rank
};
struct Waves {
  Plan plan;
  int tile[kAhead];
  uint64_t known[kAhead], done[kAhead];
};

struct TcShared {
  Groups groups;
  Waves waves;
  alignas(16) float factor[2][256];      // of the rows of y: x's scale, NaN for a row that is not there
  uint64_t full[kStagesMost], empty[kStagesMost], xfull[kStagesMost], afull[kAccumulators], aempty[kAccumulators], drained;
  uint32_t slot;
  alignas(16) uint8_t turn[kOutWarps][2][1024];   // 16 rows of y of a warp's 32 results each (of both tiles), on their way out
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {   // the rest of the 16 are zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// An arrival of this thread once its copies so far are there.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bytes [0, n) from any address as 16, the rest zeros: the aligned 16 bytes that hold them (each holds one of them, so it
// can be read), shifted.
__device__ __forceinline__ uint4 load16_anywhere(const uint8_t* p, int n) {
  const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15);
  const uint4* q = reinterpret_cast<const uint4*>(p - off);
  uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
  if (n > 0) a = __ldg(q);
  if ((int)off + n > 16) b = __ldg(q + 1);
  uint32_t w[9] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, 0u};
  if (off & 8)
#pragma unroll
    for (int i = 0; i < 7; ++i) w[i] = i + 2 < 9 ? w[i + 2] : 0u;
  if (off & 4)
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 1];
  const uint32_t sh = (off & 3) * 8;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    w[i] = __funnelshift_r(w[i], w[i + 1], sh);
    const int left = n - 4 * i;   // bytes of this word that count
    if (left < 4) w[i] &= left <= 0 ? 0u : (1u << (8 * left)) - 1u;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Whether all of THREADS threads (whole warps, barrier 1) say so; a barrier of theirs.
template <int THREADS>
__device__ __forceinline__ bool all_of(bool v) {
  uint32_t r;
  asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n bar.red.and.pred q, 1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
               : "=r"(r) : "r"((uint32_t)v), "n"(THREADS) : "memory");
  return r != 0;
}
__device__ __forceinline__ void cluster_sync() {   // converged warps
  asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// What a tile costs: its rows, and what it costs whatever they are.
__device__ __forceinline__ int work_of(const ExpertArgs& a, const Groups& g, int tile, int unit) {
  const int n = tile_of(a, g, tile, unit).n;
  return max((n + unit - 1) / unit * unit, 96) + 16;
}
// By one warp: the pairs' work so far, of pairs lane + 32 i, and this pair's tile of a wave (ntiles: none).  The first wave's
// is the pair's own number; the later ones are asked for one after the other.
constexpr int kEach = kPairsMost / 32;
struct Loads {
  int v[kEach];
};
__device__ __forceinline__ Loads first_wave(const ExpertArgs& a, const Groups& g, int ntiles, int pairs, int unit) {
  Loads load;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = (threadIdx.x & 31) + 32 * i;
    load.v[i] = p < pairs && p < ntiles ? work_of(a, g, p, unit) : 0;
  }
  return load;
}
__device__ __forceinline__ int plan_wave(const ExpertArgs& a, const Groups& g, Plan& s, Loads& load, int wave, int ntiles, int pairs, int pair, int unit) {
  const int lane = threadIdx.x & 31, t0 = wave * pairs, n = min(pairs, ntiles - t0);
  int w[kEach], key[kEach], low = 0x7FFFFFFF;
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (lane + 32 * i < pairs) low = min(low, load.v[i]);
  low = __reduce_min_sync(0xFFFFFFFFu, low);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = lane + 32 * i;
    load.v[i] -= low;
    w[i] = p < n ? work_of(a, g, t0 + p, unit) : 0;   // (a pair without a tile: last)
    key[i] = w[i] * 128 + 127 - p;                    // no two alike
    s.of[p] = p < pairs ? make_int2(key[i], load.v[i] * 128 + p) : make_int2(-1, 0x7FFFFFFF);   // (past the pairs: before nobody)
  }
  __syncwarp();
  int tile_rank[kEach] = {}, load_rank[kEach] = {};
#pragma unroll 4
  for (int q = 0; q < pairs; q += 2) {
    const uint4 two = lds128(s.of + q);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int mine = load.v[i] * 128 + lane + 32 * i;
      tile_rank[i] += ((int)two.x > key[i]) + ((int)two.z > key[i]);
      load_rank[i] += ((int)two.y < mine) + ((int)two.w < mine);
    }
  }
#pragma unroll
  for (int i = 0; i < kEach; ++i)
    if (lane + 32 * i < pairs) s.by_rank[tile_rank[i]] = w[i];
  __syncwarp();
  int mine = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = lane + 32 * i;
    if (p == pair) mine = load_rank[i];
    if (p < pairs) load.v[i] += s.by_rank[load_rank[i]];
  }
  mine = __shfl_sync(0xFFFFFFFFu, mine, pair & 31);
  int tile = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = lane + 32 * i;
    if (p < pairs && tile_rank[i] == mine) tile = p < n ? t0 + p : ntiles;
  }
  return __reduce_max_sync(0xFFFFFFFFu, tile);
}
// By one warp: this pair's tile of every wave, ahead of its other warps.  False: a wait for them ran out.
__device__ __forceinline__ bool plan_waves(const ExpertArgs& a, const Groups& g, Waves& s, int ntiles, int pairs, int pair, int unit) {
  const bool first = (threadIdx.x & 31) == 0;
  mbar_arrive(first, s.known);   // (the first wave's phase)
  Loads load = first_wave(a, g, ntiles, pairs, unit);
  for (int wave = 1; (int64_t)wave * pairs < ntiles; ++wave) {
    if (wave >= kAhead &&
        !__all_sync(0xFFFFFFFFu, mbar_wait_idle(s.done + wave % kAhead, (uint32_t)(wave / kAhead - 1) & 1u, 2 * a.spin)))
      return false;
    const int tile = plan_wave(a, g, s.plan, load, wave, ntiles, pairs, pair, unit);
    if (first) s.tile[wave % kAhead] = tile;
    mbar_arrive(first && !(a.lose_plan && wave == 1 && blockIdx.x == 0), s.known + wave % kAhead);
  }
  return true;
}

// What is stored for results that a wait that ran out has lost.  A warp whose wait ran out passes nothing on: who waits for
// it runs out as well, up to the warps that store.
constexpr uint32_t kLost = 0x7FC00000u;

// A lane's results of a lost tile, those that it would have stored: of the matrix's rows m (and m + 128) and every other 16 rows
// of y.
template <typename Y, bool GLU>
__device__ __forceinline__ void lose_tile(const ExpertArgs& a, const Tile& t, int m, int side) {
  for (int c0 = 16 * side; c0 < t.n; c0 += 32)
    for (int c = c0; c < min(c0 + 16, t.n); ++c) {
      const int64_t at = (int64_t)(t.p0 + c) * a.y_ld + m;
      if (m < a.rows) keep(static_cast<Y*>(a.y) + at, __uint_as_float(kLost));
      if (!GLU && m + 128 < a.rows) keep(static_cast<Y*>(a.y) + at + 128, __uint_as_float(kLost));
    }
}
// Where a storing warp's wait for the plan ran out: it works out by itself which tiles from wave `from` on are lost.
template <bool GLU>
__device__ __noinline__ void lose_waves(const ExpertArgs& a, const Groups& g, Plan& plan, int from, int ntiles, int pairs, int pair, int unit,
                                        int half, int side) {
  const int lane = threadIdx.x & 31, quarter = threadIdx.x >> 5 & 3;
  Loads load = first_wave(a, g, ntiles, pairs, unit);
  for (int wave = 1; (int64_t)wave * pairs < ntiles; ++wave) {
    const int tile = plan_wave(a, g, plan, load, wave, ntiles, pairs, pair, unit);
    if (wave < from) continue;
    if (tile < ntiles) {
      const Tile t = tile_of(a, g, tile, unit);
      lose_tile<__nv_bfloat16, GLU>(a, t, (2 * t.m + half) * (GLU ? 128 : 256) + 32 * quarter + lane, side);
    }
  }
}

// A finished sum times its two scales.  The scales' product comes first where it is a normal number (as where a warp's scales
// are known to give only such); else the sum takes one of them first, so that nothing on the way lies outside what sum and
// result span: the larger, or a zero.
__device__ __forceinline__ float scaled(float sum, float f, float s) {
  const float p = f * s;
  if (fabsf(p) >= 0x1p-126f && fabsf(p) <= 0x1.fffffep127f) return sum * p;
  const bool first = fabsf(f) > fabsf(s);
  const float large = first ? f : s, small = first ? s : f;
  return small == 0.f ? sum * small * large : sum * large * small;
}
// Least and largest magnitude (bits) of finite or infinite scales other than zeros.
struct Span {
  uint32_t least = 0x7F800000u, most = 0u;
  __device__ __forceinline__ void add(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7FFFFFFFu;
    if (b - 1u < 0x7F800000u) {
      least = min(least, b);
      most = max(most, b);
    }
  }
  __device__ __forceinline__ void of_warp() {
    least = __reduce_min_sync(0xFFFFFFFFu, least);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
  }
};

// SiLU(g) u.  The quotient's denominator is 1 .. 2, so that the fast one (2 units in the last place) holds for every g.  Gate
// and up of 128 experts of 768 x 2048, 8192 tokens 294 to 300 us; with an exact division 340, with the fast exponential (which loses
// 1.2 |g| units) 288.
__device__ __forceinline__ float silu(float g, float u) {
  const float e = expf(-fabsf(g));
  return g * __fdividef(g < 0.f ? e : 1.f, 1.f + e) * u;
}

// SUMS: fp32 results.  The tensor core cuts off what an addition has below fp32: 500 of them (8000 columns of bf16) lose 7e-6
// of a sum, of SiLU of it twice that; nothing beside the half step of a result in bf16, but 8 times what sums in fp32 lose.  So
// an accumulator takes a few steps, and registers add those up to nearest: 2e-7, and 3e-7.  They hold the sums of SUMS rows of
// y, 64 or 128; large products read the matrices more often for it and L2 bounds them (gate and up of 128 experts of 768 x 2048,
// us, fp32 and bf16: 1 token 14.6 and 13.9, 256 121 and 117, 8192 581 and 300).
template <bool F8, bool GLU, bool PAIR, int SUMS>
__global__ void __launch_bounds__(kTcThreads, 1)
    k_expert_tc(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap umap, const __grid_constant__ ExpertArgs a) {
  constexpr int kCols = F8 ? 128 : 64;         // columns of a stage
  constexpr int kRows = GLU ? 128 : 256;       // rows of y's width that a CTA covers
  constexpr int kUnit = PAIR ? 32 : 16;        // rows of y of a tile are a multiple of it, as the MMA takes them
  constexpr int kBoth = PAIR ? 2 : 1;          // CTAs that share a tile
  constexpr bool kSplit = !PAIR && SUMS <= kFewRows;
  using Y = std::conditional_t<(SUMS > 0), float, __nv_bfloat16>;
  static_assert(!(SUMS && PAIR) && sizeof(Plan) <= sizeof(TcShared::turn[0]), "");
  extern __shared__ uint8_t raw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t stage = kATile + (uint32_t)(a.N / kBoth) * 128;
  float* red = reinterpret_cast<float*>(sm + (size_t)a.stages * stage);   // split: [2][N][128]
  TcShared& s = *reinterpret_cast<TcShared*>(reinterpret_cast<uint8_t*>(red) + (a.splits > 1 ? (size_t)a.N * 1024 : 0));
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  // CTAs of a tile: a pair, or the splits of the columns
  const int group = PAIR ? 2 : a.splits, rank = (int)(blockIdx.x % (unsigned)group), first = (int)(blockIdx.x / (unsigned)group);
  const int step = (int)(gridDim.x / (unsigned)group), half = PAIR ? rank : 0;
  const int k0 = PAIR ? 0 : rank * a.sps, nk = max(0, min(a.sps, a.nk - k0));
  if (tid == 0) {
    if (a.w_vec) {
      prefetch_map(&wmap);
      if (GLU) prefetch_map(&umap);
    }
    // arrivals of the threads that fill a stage: with the matrices stored beside x's copies two each (see there)
    const uint32_t fills = 32 * kXWarps * (!a.w_vec && a.x_vec ? 2 : 1);
    for (int i = 0; i < a.stages; ++i) {
      // the matrices' bytes (if by TMA), x's rows (a pair's first CTA's: of both)
      mbar_init_n(s.full + i, (a.w_vec ? 1 : 0) + (PAIR ? 2 : fills));
      mbar_init_n(s.xfull + i, fills);
      mbar_init_n(s.empty + i, 1);
    }
    for (int i = 0; i < kAccumulators; ++i) {
      mbar_init_n(s.afull + i, 1);
      mbar_init_n(s.aempty + i, kBoth * kOutWarps);
    }
    for (int i = 0; i < kAhead; ++i) {
      mbar_init_n(s.waves.known + i, 1);
      mbar_init_n(s.waves.done + i, kOutWarps);
    }
    mbar_init_n(&s.drained, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (wid == 1) {
    if constexpr (PAIR) tmem_alloc_pair(&s.slot, 512);
    else tmem_alloc(&s.slot, 512);
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  pdl_trigger();   // (the next such kernel may get ready on SMs that are free)
  pdl_wait();      // nothing above reads or writes global memory: the kernel before may still run
  read_groups<kTcThreads>(a, s.groups);   // (with barriers of the block)
  if constexpr (PAIR) {
    __syncwarp();
    cluster_sync();
  }
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, s.slot, 0);
  const int ntiles = s.groups.tiles[a.E] * a.mt;
  const auto at0 = [&](const void* p) {   // the same place in a pair's first CTA, else here
    return PAIR ? cluster_address(smem_u32(p), 0) : smem_u32(p);
  };
  bool ok = true, planned = true;   // waits: of the stages and accumulators, for the plan
  // The tile after `tile`, this group's of wave `wave` (ntiles: none, or, where `planned` is false, not known).  By a whole
  // warp, whose lanes go on together, or by one lane.
  const auto next_tile = [&](int tile, int wave, auto whole) {
    if (!PAIR) return tile + step;
    if ((int64_t)wave * step >= ntiles) return ntiles;
    bool there = mbar_wait(s.waves.known + wave % kAhead, (uint32_t)(wave / kAhead) & 1u, a.spin);
    if constexpr (decltype(whole)::value) there = __all_sync(0xFFFFFFFFu, there);
    if (!there) {
      planned = false;
      return ntiles;
    }
    return *reinterpret_cast<volatile int*>(s.waves.tile + wave % kAhead);
  };
  constexpr std::true_type whole_warp;
  constexpr std::false_type one_lane;

  if (wid >= 4 + kXWarps) {
    if constexpr (SUMS > kFewRows) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSumRegs));   // (128 sums a thread)
    const int quarter = wid & 3, side = (wid - 4 - kXWarps) >> 2;
    const uint32_t aempty0 = at0(s.aempty);
    int buf = 0, use = 0;
    for (int tile = first, it = 0;;) {
      if (!PAIR && tile >= ntiles) break;
      const Tile t = tile < ntiles ? tile_of(a, s.groups, tile, kUnit) : Tile{0, 0, 0, 0};
      float* factor = s.factor[it & 1];
      {
        const int r = tid - 32 * (4 + kXWarps);
        float f = 0.f;
        if (r < t.n) {
          const int row = row_of(a, t.p0 + r);
          f = row < 0 ? __uint_as_float(kLost) : F8 ? __ldg(a.xs + row) : 1.f;
        }
        factor[r] = f;
      }
      const int r = 32 * quarter + lane, m = (kBoth * t.m + half) * kRows + r;   // and, without U, row m + 128
      const bool in0 = m < a.rows, in1 = GLU ? in0 : m + 128 < a.rows;
      float s0 = 1.f, s1 = 1.f;
      if (F8) {
        if (in0) s0 = __ldg(a.ws + t.e * a.w_sld + m);
        if (in1) s1 = GLU ? __ldg(a.us + t.e * a.u_sld + m) : __ldg(a.ws + t.e * a.w_sld + m + 128);
      }
      // (a warp that passes has read the factors of two tiles ago)
      if constexpr (PAIR) {
        planned = all_of<kOutThreads>(planned);   // the warps that store go on together, or lose the rest together
        if (!planned)   // (the warp's own memory for results on their way out: there are none)
          lose_waves<GLU>(a, s.groups, *reinterpret_cast<Plan*>(s.turn[wid - 4 - kXWarps]), it, ntiles, step, first, kUnit, half, side);
        if (!planned || tile >= ntiles) break;
      } else {
        asm volatile("bar.sync 1, %0;" ::"n"(kOutThreads) : "memory");
      }
      bool wide = false;   // products of the warp's scales may leave the normal range
      if (F8) {
        Span fs, ws;
        for (int i = lane; i < t.n; i += 32) fs.add(factor[i]);
        ws.add(s0);
        ws.add(s1);
        fs.of_warp();
        ws.of_warp();
        wide = !(__uint_as_float(fs.least) * __uint_as_float(ws.least) >= 0x1p-126f) ||
               !(__uint_as_float(fs.most) * __uint_as_float(ws.most) <= 0x1.fffffep127f);
      }
      float sum[SUMS ? SUMS / 32 : 1][2][16];   // columns 16 side + 32 i + q of both tiles
      if constexpr (SUMS > 0) {
#pragma unroll
        for (int i = 0; i < SUMS / 32; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 16; ++q) sum[i][h][q] = 0.f;
        for (int i0 = 0;; ) {
          if (ok) ok = mbar_wait_idle(s.afull + buf, (uint32_t)use & 1u, a.spin);
          ok = __all_sync(0xFFFFFFFFu, ok);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t tl = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(buf * 2 * a.N + 16 * side);
#pragma unroll
          for (int i = 0; i < SUMS / 32; ++i)
            if (ok && nk > 0 && 16 * side + 32 * i < t.n) {
              uint32_t v[2][16];
              tmem_ld16_two(tl + (uint32_t)(32 * i), tl + (uint32_t)(a.N + 32 * i), v[0], v[1]);
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 16; ++q) sum[i][h][q] += __uint_as_float(v[h][q]);
            }
          i0 += a.chain;
          if (!ok || i0 >= nk) break;
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster(aempty0 + 8u * (uint32_t)buf);
          if (++buf == a.nbuf) {
            buf = 0;
            ++use;
          }
        }
      } else {
        if (ok) ok = mbar_wait_idle(s.afull + buf, (uint32_t)use & 1u, a.spin);
        ok = __all_sync(0xFFFFFFFFu, ok);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      }
      const uint32_t tl = tmem + ((uint32_t)(32 * quarter) << 16) + (uint32_t)(buf * 2 * a.N);
      if (kSplit && a.splits > 1) {   // the part of the columns: all that is left of it is summed below
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // (N is at most 64)
          const int c0 = 16 * side + 32 * i;
          if (c0 >= t.n) break;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[16];
            if constexpr (SUMS > 0) {
#pragma unroll
              for (int q = 0; q < 16; ++q) v[q] = sum[kSplit ? i : 0][h][q];
            } else {
              uint32_t d[16];
              if (ok && nk > 0) tmem_ld16(tl + (uint32_t)(h * a.N + c0), d);
#pragma unroll
              for (int q = 0; q < 16; ++q) v[q] = nk > 0 ? __uint_as_float(d[q]) : 0.f;
            }
#pragma unroll
            for (int q = 0; q < 16; ++q) red[(h * a.N + c0 + q) * 128 + r] = ok ? v[q] : __uint_as_float(kLost);
          }
        }
      } else if (!ok) {
        lose_tile<Y, GLU>(a, t, m, side);
      } else if (!SUMS && a.y_vec && !wide) {
        // bf16 rows on 16-byte boundaries: rows lie along the lanes of tensor memory; turned by way of shared memory a row of y
        // goes out 16 bytes a lane
        // (a row is 64 bytes; its 16-byte pieces are turned by its number, so that no two of eight rows meet in a bank)
        const int mw = m - lane;   // the warp's first row
        uint8_t(*turn)[1024] = s.turn[wid - 4 - kXWarps];
        const int pr = (lane >> 4) * 8 + (lane & 7);   // the row that this lane says the place of
        const auto piece = [](int row, int i) { return row * 64 + ((i ^ (row >> 1 & 3)) << 4); };
        float sr[2][2][2];   // scales of the lane's rows 16 h + 8 i + l / 4 of both tiles
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            sr[0][h][i] = F8 ? __shfl_sync(0xFFFFFFFFu, s0, 16 * h + 8 * i + (lane >> 2)) : 1.f;
            sr[1][h][i] = F8 ? __shfl_sync(0xFFFFFFFFu, s1, 16 * h + 8 * i + (lane >> 2)) : 1.f;
          }
        uint32_t d[2][2][8];
        const auto load = [&](int c0) {
          tmem_ld_fragments(tl + (uint32_t)c0, d[0]);
          tmem_ld_fragments(tl + (uint32_t)(a.N + c0), d[1]);
        };
        if (16 * side < t.n) load(16 * side);
        for (int c0 = 16 * side; c0 < t.n; c0 += 32) {
          float2 f[2];
          f[0] = *reinterpret_cast<const float2*>(factor + c0 + 2 * (lane & 3));
          f[1] = *reinterpret_cast<const float2*>(factor + c0 + 8 + 2 * (lane & 3));
          tmem_wait(d[0]);
          tmem_wait(d[1]);
          const auto value = [&](int b, int h, int q) {   // element q of 8: columns 8 (q / 4) + q % 2, rows 8 (q / 2 % 2)
            const float g = q & 1 ? f[q >> 2].y : f[q >> 2].x;
            return __uint_as_float(d[b][h][q]) * (F8 ? g * sr[b][h][q >> 1 & 1] : g);
          };
#pragma unroll
          for (int b = 0; b < (GLU ? 1 : 2); ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t o[4];
#pragma unroll
              for (int q = 0; q < 8; q += 2) {
                float x = value(b, h, q), y = value(b, h, q + 1);
                if constexpr (GLU) {
                  x = silu(x, value(1, h, q));
                  y = silu(y, value(1, h, q + 1));
                }
                const __nv_bfloat162 p = __floats2bfloat162_rn(x, y);
                o[q >> 1] = *reinterpret_cast<const uint32_t*>(&p);
              }
              store_transposed(smem_u32(turn[b]) + (uint32_t)piece(pr, 2 * h + (lane >> 3 & 1)), o[0], o[1], o[2], o[3]);
            }
          if (c0 + 32 < t.n) load(c0 + 32);   // (in flight while this one goes out)
          __syncwarp();
#pragma unroll
          for (int b = 0; b < (GLU ? 1 : 2); ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int c = 8 * i + (lane >> 2), col = mw + 128 * b + 8 * (lane & 3);
              const uint4 p = lds128(turn[b] + piece(c, lane & 3));
              if (c0 + c < t.n && col < a.rows) {
                __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + (int64_t)(t.p0 + c0 + c) * a.y_ld + col;
                if (col + 8 <= a.rows) {
                  *reinterpret_cast<uint4*>(y) = p;
                } else {
                  const uint32_t e[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                  for (int n = 0; n < 7; ++n)
                    if (col + n < a.rows) reinterpret_cast<uint16_t*>(y)[n] = (uint16_t)(e[n >> 1] >> (16 * (n & 1)));
                }
              }
            }
          __syncwarp();
        }
      } else {
        // a row of the matrix a lane
        if (F8 && SUMS && wide) {   // (apart: a choice for each sum took 535 us in place of 510, 8192 rows of 14336 x 4096)
#pragma unroll
          for (int i = 0; i < (SUMS ? SUMS / 32 : 0); ++i)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
              const float f = factor[16 * side + 32 * i + q];
              sum[i][0][q] = scaled(sum[i][0][q], f, s0);
              sum[i][1][q] = scaled(sum[i][1][q], f, s1);
            }
          s0 = s1 = 1.f;
        }
        const auto put = [&](int c, float g, float u) {   // column c of both tiles
          if (c >= t.n) return;
          const float f = SUMS && wide ? 1.f : factor[c];   // (fp32 results: scaled above)
          const float v0 = !F8 ? g * f : !SUMS && wide ? scaled(g, f, s0) : g * (s0 * f);
          const float v1 = !F8 ? u * f : !SUMS && wide ? scaled(u, f, s1) : u * (s1 * f);
          Y* at = static_cast<Y*>(a.y) + (int64_t)(t.p0 + c) * a.y_ld + m;
          if constexpr (GLU) {
            if (in0) keep(at, silu(v0, v1));
          } else {
            if (in0) keep(at, v0);
            if (in1) keep(at + 128, v1);
          }
        };
        if constexpr (SUMS > 0) {
#pragma unroll
          for (int i = 0; i < SUMS / 32; ++i)
#pragma unroll
            for (int q = 0; q < 16; ++q) put(16 * side + 32 * i + q, sum[i][0][q], sum[i][1][q]);
        } else {
          for (int c0 = 16 * side; c0 < t.n; c0 += 32) {
            uint32_t v[2][16];
            tmem_ld16_two(tl + (uint32_t)c0, tl + (uint32_t)(a.N + c0), v[0], v[1]);
#pragma unroll
            for (int q = 0; q < 16; ++q) put(c0 + q, __uint_as_float(v[0][q]), __uint_as_float(v[1][q]));
          }
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      // (A warp whose wait ran out arrives nowhere: it may be ahead of the others, who may still read this tile's place in the
      // plan, or its accumulators.  What waits for it runs out as well.)
      if (lane == 0 && ok) mbar_arrive_cluster(aempty0 + 8u * (uint32_t)buf);
      if (PAIR) mbar_arrive(lane == 0 && ok, s.waves.done + it % kAhead);   // (everyone else is past this tile)
      if (++buf == a.nbuf) {
        buf = 0;
        ++use;
      }
      tile = next_tile(tile, ++it, whole_warp);
    }
  } else {
    if constexpr (SUMS > kFewRows) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    if (wid == 0) {
      if (lane == 0 && a.w_vec) {
        const uint32_t full0 = at0(s.full);
        int st = 0, u = 0, n = 0;
        for (int tile = first, it = 0; tile < ntiles && ok; tile = next_tile(tile, ++it, one_lane)) {
          const Tile t = tile_of(a, s.groups, tile, kUnit);
          const int m0 = (kBoth * t.m + half) * kRows;
          for (int i = 0; i < nk; ++i, ++n) {
            if (u > 0) ok = mbar_wait(s.empty + st, (uint32_t)(u - 1) & 1u, a.spin);
            if (!ok) break;
            const uint32_t bar = full0 + 8u * (uint32_t)st, dst = smem_u32(sm) + (uint32_t)st * stage;
            if (half == 0) mbar_expect_tx(s.full + st, kBoth * kATile);   // of both CTAs
            tma_load_3d<PAIR>(dst, &wmap, (k0 + i) * kCols, m0, t.e * a.w_next, bar);   // 256 rows, with U 128
            if (GLU) tma_load_3d<PAIR>(dst + kATile / 2, &umap, (k0 + i) * kCols, m0, t.e * a.u_next, bar);
            if (++st == a.stages) {
              st = 0;
              ++u;
            }
          }
        }
        // copies in flight: they are there, or (a pair's second CTA, whose copies the first one's barriers count) products have
        // read them; after a timeout an arrival may be missing, and the wait is longer than a copy takes
        uint64_t* bars = half == 0 ? s.full : s.empty;
        const long long most = half == 0 && ok && planned ? kWaitClocks : max(a.spin, kCopyClocks);   // (the first CTA may have given up)
        for (int j = max(0, n - a.stages); j < n; ++j) mbar_wait(bars + j % a.stages, (uint32_t)(j / a.stages) & 1u, most);
      }
      __syncwarp();
    } else if (wid == 1 && half == 0) {
      const uint32_t one = elect_one();
      const uint64_t da = sw128_desc(smem_u32(sm)), db = sw128_desc(smem_u32(sm) + kATile);
      uint32_t empty[kBoth], afull[kBoth];
#pragma unroll
      for (int r = 0; r < kBoth; ++r) {
        empty[r] = PAIR ? cluster_address(smem_u32(s.empty), (uint32_t)r) : smem_u32(s.empty);
        afull[r] = PAIR ? cluster_address(smem_u32(s.afull), (uint32_t)r) : smem_u32(s.afull);
      }
      int st = 0, u = 0, buf = 0, use = 0;
      for (int tile = first, it = 0; tile < ntiles && ok; tile = next_tile(tile, ++it, whole_warp)) {
        const int n = (tile_of(a, s.groups, tile, kUnit).n + kUnit - 1) / kUnit * kUnit;
        const uint32_t idesc = idesc_of<F8, PAIR>(n);
        int i0 = 0;
        do {   // (once, but of fp32 results)
          if (use > 0) ok = mbar_wait(s.aempty + buf, (uint32_t)(use - 1) & 1u, a.spin);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t acc = tmem + (uint32_t)(buf * 2 * a.N);
          const int last = SUMS ? min(i0 + a.chain, nk) : nk;
          for (int i = i0; i < last; ++i) {
            if constexpr (PAIR) ok = mbar_wait_shared_cluster(s.full + st, (uint32_t)u & 1u, a.spin);   // (also the other CTA's)
            else ok = mbar_try_wait(s.full + st, (uint32_t)u & 1u) || mbar_wait(s.full + st, (uint32_t)u & 1u, a.spin);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            if (!PAIR) fence_proxy_async();   // x's rows: generic writes -> tensor-core reads
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint64_t o = (uint64_t)((uint32_t)st * (stage >> 4));
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int k = 0; k < 4; ++k)
                mma_of<F8, PAIR>(one, acc + (uint32_t)(h * a.N), da + o + h * (kATile >> 5) + 2 * k, db + o + 2 * k, idesc, (uint32_t)((i - i0) | k));
            if (!(a.lose && (i | it | (int)blockIdx.x) == 0))
#pragma unroll
              for (int r = 0; r < kBoth; ++r) mma_commit_at<PAIR>(one, empty[r] + 8u * (uint32_t)st);
            if (++st == a.stages) {
              st = 0;
              ++u;
            }
          }
          if (!ok) break;
#pragma unroll
          for (int r = 0; r < kBoth; ++r) mma_commit_at<PAIR>(one, afull[r] + 8u * (uint32_t)buf);
          if (++buf == a.nbuf) {
            buf = 0;
            ++use;
          }
          i0 = last;
        } while (SUMS && i0 < nk);
        if (!ok) break;
      }
      // products in flight: who waits for their results may have given up
#pragma unroll
      for (int r = 0; r < kBoth; ++r) mma_commit_at<PAIR>(one, PAIR ? cluster_address(smem_u32(&s.drained), (uint32_t)r) : smem_u32(&s.drained));
      mbar_wait(&s.drained, 0u);
      __syncwarp();
    } else if (PAIR && wid == 2) {
      if (lane == 0) {
        const uint32_t full0 = at0(s.full);
        int st = 0, u = 0;
        for (int tile = first, it = 0; tile < ntiles && ok; tile = next_tile(tile, ++it, one_lane))
          for (int i = 0; i < nk; ++i) {
            ok = mbar_wait(s.xfull + st, (uint32_t)u & 1u, a.spin);
            if (!ok) break;
            fence_proxy_async();   // generic writes -> tensor-core reads
            mbar_release_shared_cluster(full0 + 8u * (uint32_t)st);
            if (++st == a.stages) {
              st = 0;
              ++u;
            }
          }
      }
      __syncwarp();
    } else if (PAIR && wid == 3) {
      planned = plan_waves(a, s.groups, s.waves, ntiles, step, first, kUnit);
    } else if (wid >= 4) {
      const int g = tid - 128, chunk = g & 7, r0 = g >> 3;   // 16 bytes of rows r0 + kXRows j
      const uint32_t at = (uint32_t)r0 * 128u + (uint32_t)((chunk ^ (r0 & 7)) << 4);
      const int width = a.cols * (F8 ? 1 : 2);
      constexpr int kPasses = (PAIR || SUMS > kFewRows ? 128 : kFewRows) / kXRows;
      int st = 0, u = 0;
      for (int tile = first, it = 0; tile < ntiles && ok; tile = next_tile(tile, ++it, whole_warp)) {
        const Tile t = tile_of(a, s.groups, tile, kUnit);
        const int mine = (t.n + kUnit - 1) / kUnit * kUnit / kBoth;   // rows of this CTA
        const uint8_t* src[kPasses];
#pragma unroll
        for (int j = 0; j < kPasses; ++j) {
          const int r = r0 + kXRows * j, q = half * mine + r;
          const int row = r < mine && q < t.n ? row_of(a, t.p0 + q) : -1;
          src[j] = row < 0 ? nullptr : static_cast<const uint8_t*>(a.x) + (int64_t)row * a.x_ld * (F8 ? 1 : 2) + chunk * 16;
        }
        for (int i = 0; i < nk; ++i) {
          if (u > 0) ok = mbar_try_wait(s.empty + st, (uint32_t)(u - 1) & 1u) || mbar_wait(s.empty + st, (uint32_t)(u - 1) & 1u, a.spin);
          ok = __all_sync(0xFFFFFFFFu, ok);
          if (!ok) break;
          const uint32_t dst = smem_u32(sm) + (uint32_t)st * stage + kATile + at;
          const int b = (k0 + i) * 128, left = min(max(width - b - chunk * 16, 0), 16);
          uint64_t* there = (PAIR ? s.xfull : s.full) + st;
          const auto put = [&](uint32_t to, const uint4& v) {
            asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
          };
          if (!a.w_vec) {   // the matrices too: rows r0 + kXRows j of the two tiles
            const int m0 = (kBoth * t.m + half) * kRows;
#pragma unroll 4
            for (int j = 0; j < 256 / kXRows; ++j) {
              const int r = r0 + kXRows * j;
              const bool up = GLU && r >= 128;
              const int m = m0 + (up ? r - 128 : r);
              const uint8_t* row = static_cast<const uint8_t*>(up ? a.up : a.w) +
                                   ((int64_t)t.e * (up ? a.u_eld : a.w_eld) + (int64_t)m * (up ? a.u_ld : a.w_ld)) * (F8 ? 1 : 2);
              put(dst - kATile + (uint32_t)j * (kXRows * 128u), load16_anywhere(row + b + chunk * 16, m < a.rows ? left : 0));
            }
          }
          if (a.x_vec) {
#pragma unroll
            for (int j = 0; j < kPasses; ++j)
              if (r0 + kXRows * j < mine) {
                const int bytes = src[j] ? left : 0;
                cp_async16(dst + (uint32_t)j * (kXRows * 128u), bytes ? src[j] + b : static_cast<const uint8_t*>(a.x), bytes);
              }
            cp_async_arrive(there);
            if (!a.w_vec) mbar_arrive(there);   // (that one stands for the copies alone, this one for the plain stores)
          } else {   // rows off 16-byte boundaries
#pragma unroll
            for (int j = 0; j < kPasses; ++j)
              if (r0 + kXRows * j < mine) {
                put(dst + (uint32_t)j * (kXRows * 128u), load16_anywhere(src[j] ? src[j] + b : static_cast<const uint8_t*>(a.x), src[j] ? left : 0));
              }
            mbar_arrive(there);
          }
          if (++st == a.stages) {
            st = 0;
            ++u;
          }
        }
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  // no CTA leaves while another may still reach its shared or tensor memory
  if (PAIR || (kSplit && a.splits > 1)) cluster_sync();
  else __syncthreads();
  if (PAIR && half == 1 && wid == 1) mbar_wait(&s.drained, 0u);   // (the last arrival that comes from the first CTA)
  if (kSplit && a.splits > 1) {
    if (first < ntiles) {
      // every CTA has its part of the tile in shared memory; each sums and stores its share of the results
      const Tile t = tile_of(a, s.groups, first, kUnit);
      for (int i = rank * kTcThreads + tid; i < t.n * 128; i += a.splits * kTcThreads) {
        const int c = i >> 7, r = i & 127, m = t.m * kRows + r;
        float v[2] = {0.f, 0.f};
        for (int q = 0; q < a.splits; ++q)
#pragma unroll
          for (int h = 0; h < 2; ++h) v[h] += ld_cluster(cluster_address(smem_u32(red + (h * a.N + c) * 128 + r), (uint32_t)q));
        const float f = s.factor[0][c];
        const int64_t at = (int64_t)(t.p0 + c) * a.y_ld + m;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int mh = GLU ? m : m + 128 * h;
          if (mh < a.rows) v[h] = F8 ? scaled(v[h], f, __ldg((GLU && h ? a.us + t.e * a.u_sld : a.ws + t.e * a.w_sld) + mh)) : v[h] * f;
        }
        if constexpr (GLU) {
          if (m < a.rows) keep(static_cast<Y*>(a.y) + at, silu(v[0], v[1]));
        } else {
          if (m < a.rows) keep(static_cast<Y*>(a.y) + at, v[0]);
          if (m + 128 < a.rows) keep(static_cast<Y*>(a.y) + at + 128, v[1]);
        }
      }
    }
    __syncwarp();
    cluster_sync();
  }
  if (!(ok && planned) && a.status) atomicCAS(a.status, 0, BITSMOE_ERR_TIMEOUT);
  if (wid == 1) {
    __syncwarp();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if constexpr (PAIR) tmem_dealloc_pair(tmem, 512);
    else tmem_dealloc(tmem, 512);
  }
}

// Rows of y of a tile: twice an expert's on average and 32 more, so that few experts have more than one tile, each of which
// reads the expert's matrix again; a stage of more rows leaves room for fewer stages.  Without the 32, gate and up of 128
// experts of 768 x 2048 (us): 25 rows an expert 126 in place of 117, 10 rows 117 and 114, 3 rows 87 and 89.
int tile_rows(int P, int E) {
  const int most = (int)std::min<int64_t>(256, ((int64_t)P + 31) / 32 * 32);
  return std::min(most, (int)std::min<int64_t>(256, (2ll * P / E + 31) / 32 * 32 + 32));
}

bool on_boundaries(const void* p, int64_t ld, int64_t size, int64_t rows) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows <= 1 || ld * size % 16 == 0);
}
int64_t pitch_of(int64_t ld, int64_t cols, int64_t size, int64_t rows) {   // (of one row: any)
  return rows <= 1 ? (cols * size + 15) / 16 * 16 : ld * size;
}

// The maps of matrices whose rows start on 16-byte boundaries (false: they are read another way).
bool tc_maps(const ExpertArgs& a, bool f8, CUtensorMap* wm, CUtensorMap* um) {
  const int64_t es = f8 ? 1 : 2;
  const int box = a.up ? 128 : 256;
  const auto matrices = [&](CUtensorMap* m, const void* p, int64_t ld, int64_t eld) {
    return on_boundaries(p, ld, es, a.rows) && make_matrices_map(m, f8, p, a.E, a.rows, a.cols, pitch_of(ld, a.cols, es, a.rows), eld * es, box);
  };
  return matrices(wm, a.w, a.w_ld, a.w_eld) && (!a.up || matrices(um, a.up, a.u_ld, a.u_eld));
}

// Clusters of n CTAs of a kernel (one CTA an SM) that run at once on device `dev`, asked once for each.
template <auto K>
int clusters_at_once(int dev, int n) {
  static std::atomic<int> known[64][4];
  const int q = n == 1 ? 0 : n == 2 ? 1 : n == 4 ? 2 : 3;
  if (dev < 64) {
    const int c = known[dev][q].load(std::memory_order_relaxed);
    if (c > 0) return c;
  }
  if (allow_shared<K>(dev, kTcShared) != cudaSuccess) return 0;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)n;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n);
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = kTcShared;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int c = 0;
  if (cudaOccupancyMaxActiveClusters(&c, K, &cfg) != cudaSuccess) return 0;
  if (dev < 64) known[dev][q].store(c, std::memory_order_relaxed);
  return c;
}

template <bool F8, bool GLU, bool PAIR, int SUMS>
cudaError_t launch_tc_as(const ExpertArgs& a, const CUtensorMap& wm, const CUtensorMap& um, int64_t groups, int dev, cudaStream_t st) {
  auto kern = k_expert_tc<F8, GLU, PAIR, SUMS>;
  const cudaError_t e = allow_shared<k_expert_tc<F8, GLU, PAIR, SUMS>>(dev, kTcShared);
  if (e != cudaSuccess) return e;
  const unsigned size = PAIR ? 2u : (unsigned)a.splits;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = size;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(size * (unsigned)groups);
  cfg.blockDim = dim3(kTcThreads);
  cfg.dynamicSmemBytes = kTcShared;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = size > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, wm, um, a);
}

template <bool F8, bool GLU, bool SUMS>
cudaError_t launch_tc(ExpertArgs a, const CUtensorMap& wm, const CUtensorMap& um, int dev, int sms, cudaStream_t st) {
  a.N = tile_rows(a.P, a.E);
  bool pair = !SUMS && a.N > kFewRows, many = SUMS && a.N > kFewRows;
  if (many) {
    // A tile of 128 rows takes 1.5 times as long as one of 64 (L2 bounds both, and the matrices' part of it is the same).  Gate and
    // up of 128 experts of 768 x 2048 (us, tiles of 128 and of 64): 8192 tokens 581 and 748, 1024 160 and 150; 1200 rows by 4096 x
    // 4096 (160 and 304 tiles) 80 and 72.
    const int64_t experts = std::min(a.P, a.E), tall = GLU ? 128 : 256;
    const auto waves = [&](int n) { return (experts * ((a.P / experts + n - 1) / n) * ((a.rows + tall - 1) / tall) + sms - 1) / sms; };
    many = 3 * waves(kSumRows) < 2 * waves(kFewRows);
    a.N = many ? kSumRows : kFewRows;
  }
  if (pair) {
    // Pairs where a third of them have a tile; else smaller tiles of single CTAs, over which the columns can be split too.  One
    // matrix of 4096 x 4096 (us, pairs and single): 100 rows of y (8 tiles of pairs) 30 and 13, 300 (16) 31 and 26; two of
    // them with SwiGLU, 512 (32) 44 and 51.
    const int64_t experts = std::min(a.P, a.E), tall = GLU ? 256 : 512;
    const int64_t tiles = experts * ((a.P / experts + a.N - 1) / a.N) * ((a.rows + tall - 1) / tall);
    if (6 * tiles < sms) {
      pair = false;
      a.N = kFewRows;
    }
  }
  const int rows = (GLU ? 128 : 256) * (pair ? 2 : 1);
  a.mt = (a.rows + rows - 1) / rows;
  a.nk = (a.cols + (F8 ? 127 : 63)) / (F8 ? 128 : 64);
  a.w_next = a.w_eld != 0;
  a.u_next = a.u_eld != 0;
  a.nbuf = std::min(SUMS ? kAccumulators : 2, 512 / (2 * a.N));
  const int64_t most = std::min<int64_t>(a.P, (int64_t)a.P / a.N + a.E) * a.mt;   // tiles at most
  // Few tiles: the columns over clusters of as many CTAs as the SMs hold (one token by 4096 x 4096 9.8 us, unsplit 24.0; through
  // gate and up of eight experts of 768 x 2048 11.6 and 14.8).
  a.splits = 1;
  if (!pair && !many)   // (clusters that do not all run at once would take a second turn)
    for (int n = 8; n > 1 && a.splits == 1; n /= 2)
      if (most * n <= sms && a.nk >= 2 * n && most <= clusters_at_once<k_expert_tc<F8, GLU, false, SUMS ? kFewRows : 0>>(dev, n)) a.splits = n;
  a.sps = (a.nk + a.splits - 1) / a.splits;
  const size_t room = kTcShared - 1024 - sizeof(TcShared) - (a.splits > 1 ? (size_t)a.N * 1024 : 0);
  a.stages = std::min(kStagesMost, (int)(room / (kATile + (size_t)a.N * (pair ? 64 : 128))));
  a.chain = F8 ? 8 : 2;   // 32 additions, of bf16 8 (products of 8 bits leave less to cut off); twice that: errors 1.5 times, a tenth less time
  if constexpr (SUMS) {
    if (many) return launch_tc_as<F8, GLU, false, kSumRows>(a, wm, um, std::min<int64_t>(most, sms), dev, st);
    return launch_tc_as<F8, GLU, false, kFewRows>(a, wm, um, std::min<int64_t>(most, sms / a.splits), dev, st);
  } else {
    if (pair) return launch_tc_as<F8, GLU, true, 0>(a, wm, um, std::min<int64_t>({most, sms / 2, kPairsMost}), dev, st);
    return launch_tc_as<F8, GLU, false, 0>(a, wm, um, std::min<int64_t>(most, sms / a.splits), dev, st);
  }
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
  a.y_ld = g.y_ld;
  a.y_vec = g.y_type == BITSMOE_BF16 && on_boundaries(g.y, g.y_ld, 2, g.P);
  a.spin = debug_wait_clocks() > 0 ? debug_wait_clocks() : kWaitClocks;
  a.lose = debug_skip_arrival();
  a.lose_plan = debug_skip_plan();
  a.status = g.status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  a.x_vec = g.x_rows > 0 && on_boundaries(g.x, g.x_ld, f8 ? 1 : 2, g.x_rows);
  CUtensorMap wm, um;
  std::memset(&wm, 0, sizeof(wm));
  std::memset(&um, 0, sizeof(um));
  a.w_vec = tc_maps(a, f8, &wm, &um);
  const auto go = [&](auto f8_, auto glu) {
    constexpr bool kF8 = decltype(f8_)::value, kGlu = decltype(glu)::value;
    return g.y_type == BITSMOE_F32 ? launch_tc<kF8, kGlu, true>(a, wm, um, dev, sms, st) : launch_tc<kF8, kGlu, false>(a, wm, um, dev, sms, st);
  };
  constexpr std::true_type yes;
  constexpr std::false_type no;
  e = f8 ? (a.up ? go(yes, yes) : go(yes, no)) : (a.up ? go(no, yes) : go(no, no));
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
