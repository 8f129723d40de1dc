// Routing as lists of its own, and the weighted sum that ends a layer of experts.
//
//   experts[t] = the top_k largest logits of a token (ties to the lower expert; NaN and -inf never)
//   weights[t] = exp(l - l_max) / sum over the selected, or over all, of exp(l - l_max)
//   pairs      = the pairs t * top_k + j sorted by (expert, number), offsets where each expert's begin,
//                places the inverse
//   out[t]     = base[t] + sum_j weights[t][j] y[places[t][j]]
//
// The sort is by counting, and no result depends on the order of atomics: each 32 tokens set their bits in a word for
// each expert (a token picks an expert once), and a pair's rank in its expert is the count of the bits below its
// token's, plus those of the words before.  The chain of launches and dependent reads bounds it, not the logits' bytes:
// one token of 128 experts 3.5 us, 16384 tokens 16.4 (10.5 MB, 1.6 us at DRAM's rate), 8 of them selected.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "microscale.cuh"

namespace {
using namespace bmoe;

constexpr int kMaxExperts = 1024, kMaxTopK = 32;
constexpr int kRouteThreads = 1024;
constexpr int kWords = 4, kChunk = 32 * kWords;   // tokens of a block at a time: a bit of a warp's in each word
constexpr int kAloneTokens = kChunk;              // one block does all of at most so many

struct RouteArgs {
  const float* logits;
  int64_t ld;
  int T, E, k, renormalize;
  int per;               // tokens of a block (a multiple of 32)
  int32_t* experts;
  float* weights;
  int32_t* offsets;
  int32_t* pairs;
  int32_t* places;
  int32_t* counts;       // [blocks][E]
};

__device__ __forceinline__ float logit_of(uint32_t key) {   // order_key's inverse
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

// A token's logits: lane l holds those of experts l + 32 i.
template <int NE>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, uint32_t (&key)[NE]) {
  const float* row = a.logits + t * a.ld + lane;
#pragma unroll
  for (int i = 0; i < NE; ++i) key[i] = lane + 32 * i < a.E ? __float_as_uint(__ldg(row + 32 * i)) : 0xFF800000u;
}
// One token's selection by a warp: lane j < k gets the j-th expert (-1: none) and its weight.  list: the warp's own.
template <int NE>
__device__ __forceinline__ void select_token(const RouteArgs& a, int lane, uint32_t (&key)[NE], uint2* list, int& expert, float& weight) {
  constexpr uint32_t kNone = 0x007FFFFFu;   // -infinity's key, above NaN's
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    key[i] = order_key(__uint_as_float(key[i]));   // 0 where one cannot be selected
    if (key[i] <= kNone) key[i] = 0u;
  }
  expert = -1;
  float mine = 0.f, top = 0.f, sum = 0.f;
  // The top_k-th largest of the lanes' largest logits is not above the token's top_k-th largest: what is not below it are
  // the candidates, few more than top_k.  Where a lane each holds them, a candidate's rank is the count of better ones.
  uint32_t most = key[0];
#pragma unroll
  for (int i = 1; i < NE; ++i) most = max(most, key[i]);
  uint32_t sorted = most;   // by lane, descending
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int o = size / 2; o; o /= 2) {
      const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, sorted, o);
      const bool larger = ((lane & o) == 0) == ((lane & size) == 0);
      sorted = larger ? max(sorted, other) : min(sorted, other);
    }
  const uint32_t border = max(__shfl_sync(0xFFFFFFFFu, sorted, a.k - 1), 1u);
  const uint32_t first = __shfl_sync(0xFFFFFFFFu, sorted, 0);
  if (first == 0u) {
    weight = 0.f;
    return;
  }
  top = logit_of(first);
  if (!a.renormalize) {
#pragma unroll
    for (int i = 0; i < NE; ++i)
      if (key[i]) sum += expf(logit_of(key[i]) - top);
    sum = warp_sum(sum);
  }
  int n = 0;   // candidates
#pragma unroll
  for (int i = 0; i < NE; ++i) {
    const uint32_t who = __ballot_sync(0xFFFFFFFFu, key[i] >= border);
    const int at = n + __popc(who & ((1u << lane) - 1u));
    if (key[i] >= border && at < 32) list[at] = make_uint2(key[i], (uint32_t)(lane + 32 * i));
    n += __popc(who);
  }
  __syncwarp();
  if (n <= 32) {
    uint2 c = make_uint2(0u, 0xFFFFFFFFu);
    if (lane < n) c = list[lane];
    int rank = 0;
    for (int q = 0; q < n; ++q) {
      const uint2 d = list[q];
      rank += d.x > c.x || (d.x == c.x && d.y < c.y);
    }
    __syncwarp();
    if (lane < n && rank < a.k) list[rank] = c;
    __syncwarp();
    if (lane < min(n, a.k)) {
      expert = (int)list[lane].y;
      mine = logit_of(list[lane].x);
    }
    __syncwarp();   // (the list is the next token's)
  } else {
    // (many equal ones) each lane offers its largest logit, the first of equal ones; of the largest offers the lowest
    // expert's is taken
    for (int j = 0; j < a.k; ++j) {
      uint32_t offer = key[0];
      int at = lane;
#pragma unroll
      for (int i = 1; i < NE; ++i)
        if (key[i] > offer) {
          offer = key[i];
          at = lane + 32 * i;
        }
      const uint32_t best = __reduce_max_sync(0xFFFFFFFFu, offer);
      if (best == 0u) break;
      const int e = (int)__reduce_min_sync(0xFFFFFFFFu, offer == best ? (uint32_t)at : 0xFFFFFFFFu);
      if (lane == j) {
        expert = e;
        mine = logit_of(best);
      }
#pragma unroll
      for (int i = 0; i < NE; ++i)
        if (e == lane + 32 * i) key[i] = 0u;
    }
    __syncwarp();
  }
  weight = expert >= 0 ? expf(mine - top) : 0.f;
  if (a.renormalize) sum = warp_sum(weight);
  if (expert >= 0) weight /= sum;
}

// Exclusive sums of v[0 .. n) in place (n <= 1024, one block of 1024 threads); the whole sum is returned.
__device__ __forceinline__ int block_scan(int* v, int n, int* part) {
  const int i = threadIdx.x, lane = i & 31;
  const int x = i < n ? v[i] : 0;
  int s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, s, o);
    if (lane >= o) s += y;
  }
  if (lane == 31) part[i >> 5] = s;
  __syncthreads();
  if (i < 32) {
    const int q = part[i];
    int p = q;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, p, o);
      if (lane >= o) p += y;
    }
    part[i] = p - q;
    if (i == 31) part[32] = p;
  }
  __syncthreads();
  if (i < n) v[i] = part[i >> 5] + s - x;
  return part[32];
}

struct RouteShared {
  uint32_t mask[kWords][kMaxExperts];
  int count[kMaxExperts];
  uint16_t pick[kChunk * kMaxTopK];
  uint2 list[kRouteThreads / 32][32];
  int part[33];
};

// Tokens [first, last) of a block: selection, and each pair's rank among the block's pairs of its expert (into places, for
// now).  s.count[e]: the block's pairs of expert e.
template <int NE>
__device__ __forceinline__ void select_block(const RouteArgs& a, int first, int last, RouteShared& s) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  constexpr bool kAhead = NE <= 8;   // the next token's logits are requested before this one's are used
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
#pragma unroll
    for (int q = 0; q < kWords; ++q) s.mask[q][e] = 0u;
    s.count[e] = 0;
  }
  for (int t0 = first; t0 < last; t0 += kChunk) {
    const int n = min(last - t0, kChunk);
    uint32_t key[NE], next[kAhead ? NE : 1];
    if (kAhead && w < n) load_logits<NE>(a, t0 + w, lane, key);
    __syncthreads();
    for (int q = 0; w + 32 * q < n; ++q) {
      const int t = w + 32 * q;
      int expert;
      float weight;
      if constexpr (kAhead) {
        if (t + 32 < n) load_logits<NE>(a, t0 + t + 32, lane, next);
      } else {
        load_logits<NE>(a, t0 + t, lane, key);
      }
      select_token<NE>(a, lane, key, s.list[w], expert, weight);
      if (lane < a.k) {
        a.weights[(int64_t)(t0 + t) * a.k + lane] = weight;
        s.pick[t * a.k + lane] = (uint16_t)expert;
        if (expert >= 0) atomicOr(s.mask[q] + expert, 1u << w);
      }
      if constexpr (kAhead) {
#pragma unroll
        for (int i = 0; i < NE; ++i) key[i] = next[i];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n * a.k; i += kRouteThreads) {
      const int t = i / a.k, e = (int16_t)s.pick[i];
      int rank = -1;
      if (e >= 0) {
        rank = s.count[e] + __popc(s.mask[t >> 5][e] & ((1u << (t & 31)) - 1u));
        for (int q = 0; q < t >> 5; ++q) rank += __popc(s.mask[q][e]);
      }
      const int64_t p = (int64_t)t0 * a.k + i;
      a.experts[p] = e;
      a.places[p] = rank;
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kRouteThreads)
#pragma unroll
      for (int q = 0; q < kWords; ++q) {
        s.count[e] += __popc(s.mask[q][e]);
        s.mask[q][e] = 0u;
      }
  }
  __syncthreads();
}

// Place of pair p, of rank r among the block's of expert e, once base[e] is where the block's first one goes.
__device__ __forceinline__ void place_pair(const RouteArgs& a, int64_t p, int e, int r, const int* base) {
  if (e < 0) return;
  const int at = base[e] + r;
  a.places[p] = at;
  a.pairs[at] = (int)p;
}

template <int NE>
__global__ void __launch_bounds__(kRouteThreads) k_route_alone(const __grid_constant__ RouteArgs a) {
  __shared__ RouteShared s;
  select_block<NE>(a, 0, a.T, s);
  const int total = block_scan(s.count, a.E, s.part);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) a.offsets[e] = s.count[e];
  if (threadIdx.x == 0) a.offsets[a.E] = total;
  for (int p = total + threadIdx.x; p < a.T * a.k; p += kRouteThreads) a.pairs[p] = -1;
  for (int p = threadIdx.x; p < a.T * a.k; p += kRouteThreads) place_pair(a, p, a.experts[p], a.places[p], s.count);
}

// 16384 tokens of 128 experts are 128 blocks whose warps have four tokens each in turn: 8.6 us, issuing on two thirds of the
// cycles (the sort of the lanes' largest, the candidates' ranks).
template <int NE>
__global__ void __launch_bounds__(kRouteThreads) k_route_select(const __grid_constant__ RouteArgs a) {
  __shared__ RouteShared s;
  pdl_trigger();
  const int first = blockIdx.x * a.per;
  select_block<NE>(a, first, min(first + a.per, a.T), s);
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) a.counts[(int64_t)blockIdx.x * a.E + e] = s.count[e];
}

// Every block sums the counts itself: of the blocks before it, and of all.  (Launched while the selection runs.)
__global__ void __launch_bounds__(kRouteThreads) k_route_place(const __grid_constant__ RouteArgs a) {
  __shared__ int base[kMaxExperts], start[kMaxExperts];
  __shared__ int part[33];
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) base[e] = start[e] = 0;
  __syncthreads();
  pdl_wait();
  const int64_t first = (int64_t)blockIdx.x * a.per * a.k, last = min(first + (int64_t)a.per * a.k, (int64_t)a.T * a.k);
  // this thread's first pair, requested with the counts
  const int64_t p0 = first + threadIdx.x;
  const int e1 = p0 < last ? a.experts[p0] : -1, r1 = p0 < last ? a.places[p0] : 0;
  // threads take (expert, slice of the blocks), their counts requested sixteen at a time
  const int ex = (a.E + 31) / 32 * 32, slices = max(1, kRouteThreads / ex);
  const int slice = threadIdx.x / ex, e0 = threadIdx.x % ex;
  if (slice < slices && e0 < a.E) {
    int before = 0, all = 0;
    for (int b0 = slice; b0 < (int)gridDim.x; b0 += 16 * slices) {
      int c[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) c[i] = b0 + i * slices < (int)gridDim.x ? a.counts[(int64_t)(b0 + i * slices) * a.E + e0] : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        all += c[i];
        before += b0 + i * slices < (int)blockIdx.x ? c[i] : 0;
      }
    }
    atomicAdd(base + e0, before);
    atomicAdd(start + e0, all);
  }
  __syncthreads();
  const int total = block_scan(start, a.E, part);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
    base[e] += start[e];
    if (blockIdx.x == 0) a.offsets[e] = start[e];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[a.E] = total;
  for (int64_t p = total + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; p < (int64_t)a.T * a.k; p += (int64_t)gridDim.x * kRouteThreads)
    a.pairs[p] = -1;
  __syncthreads();
  place_pair(a, p0, e1, r1, base);
  for (int64_t p = p0 + kRouteThreads; p < last; p += kRouteThreads) place_pair(a, p, a.experts[p], a.places[p], base);
}

__global__ void k_route_none(int32_t* offsets, int E) {
  for (int e = threadIdx.x; e <= E; e += blockDim.x) offsets[e] = 0;
}

template <int NE>
cudaError_t launch_route(const RouteArgs& a, int blocks, cudaStream_t st) {
  if (blocks == 1) {
    k_route_alone<NE><<<1, kRouteThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  k_route_select<NE><<<blocks, kRouteThreads, 0, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kRouteThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_route_place, a);
}

// Tokens of a block, and blocks of a call: each block of the second launch reads blocks x E counts.
int route_per(int T) {
  const int most = 152;
  return T <= kAloneTokens ? T : ((T + most - 1) / most + 31) / 32 * 32;
}
int route_blocks(int T) { return T <= kAloneTokens ? 1 : (T + route_per(T) - 1) / route_per(T); }
bool route_sizes_ok(int T, int E, int k) {
  return T >= 0 && E >= 1 && E <= kMaxExperts && k >= 1 && k <= std::min(E, kMaxTopK) && (int64_t)T * k <= (1 << 24);
}

// ---------------------------------------------------------------------------
struct CombineArgs {
  const void* y;
  int64_t y_ld;
  int T, P, k, D;
  int shift;             // log2 of a token's threads
  const int32_t* places;
  const float* weights;
  const void* base;
  int64_t base_ld;
  void* out;
  int64_t out_ld;
};

// V elements of a row on 16-byte boundaries (V: 16 bytes of y's type; 8, 16 or 32 of the other's).
template <typename T, int V>
struct Piece {
  uint32_t w[V * sizeof(T) / 4];
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p) {
  Piece<T, V> r;
  if constexpr (V * sizeof(T) >= 16) {
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T)) / 16; ++i) {
      const uint4 x = reinterpret_cast<const uint4*>(p)[i];
      r.w[4 * i] = x.x, r.w[4 * i + 1] = x.y, r.w[4 * i + 2] = x.z, r.w[4 * i + 3] = x.w;
    }
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    r.w[0] = x.x, r.w[1] = x.y;
  }
  return r;
}
template <typename T, int V>
__device__ __forceinline__ float piece_at(const Piece<T, V>& r, int i) {
  if constexpr (sizeof(T) == 4) return __uint_as_float(r.w[i]);
  else return i & 1 ? bf16hi(r.w[i / 2]) : bf16lo(r.w[i / 2]);
}
template <typename T, int V>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[V]) {
  uint32_t w[V * sizeof(T) / 4];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[i], v[i + 1]);
      w[i / 2] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  if constexpr (V * sizeof(T) >= 16) {
#pragma unroll
    for (int i = 0; i < (int)(V * sizeof(T)) / 16; ++i)
      reinterpret_cast<uint4*>(p)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  } else {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

// A group of threads a token (2^shift of the block's 256), V columns a thread; the pieces of R rows are requested before the
// first is used (of one or two rows R is 2, and the registers leave room for twice the warps).  The rows' bytes bound it: 8192
// tokens of 8 rows of 2048 bf16 59 us, 5.7 TB/s.
constexpr int kCombineThreads = 256;
template <typename TY, typename TO, int V, int R, bool ONE>   // ONE: a block's threads have one token (its places are uniform)
__global__ void __launch_bounds__(kCombineThreads, R == 2 ? 6 : 3) k_combine(const __grid_constant__ CombineArgs a) {
  const int64_t t = ONE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (kCombineThreads >> a.shift) + (threadIdx.x >> a.shift);
  const int d = ONE ? (int)(blockIdx.y * kCombineThreads + threadIdx.x) * V
                    : (int)((blockIdx.y << a.shift) + (threadIdx.x & ((1 << a.shift) - 1))) * V;
  if (t >= a.T || d >= a.D) return;   // (D is a multiple of V)
  float s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = 0.f;
  Piece<TO, V> base;
  if (a.base) base = load_piece<TO, V>(static_cast<const TO*>(a.base) + t * a.base_ld + d);
  for (int j0 = 0; j0 < a.k; j0 += R) {
    Piece<TY, V> y[R];
    float w[R];
    int p[R];
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] = j0 + j < a.k ? __ldg(a.places + t * a.k + j0 + j) : -1;
#pragma unroll
    for (int j = 0; j < R; ++j)
      if ((unsigned)p[j] < (unsigned)a.P) {
        y[j] = load_piece<TY, V>(static_cast<const TY*>(a.y) + (int64_t)p[j] * a.y_ld + d);
        w[j] = __ldg(a.weights + t * a.k + j0 + j);
      }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if ((unsigned)p[j] < (unsigned)a.P) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = fmaf(w[j], piece_at<TY, V>(y[j], i), s[i]);
      }
  }
  if (a.base) {
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = piece_at<TO, V>(base, i) + s[i];
  }
  store_piece<TO, V>(static_cast<TO*>(a.out) + t * a.out_ld + d, s);
}

// Rows on any boundary: a warp 32 V columns of a token (V: 16 bytes of y's type), a lane's as the two aligned 16 bytes that hold
// them, of four rows requested before the first is shifted into place; the sums are turned in shared memory, so that
// neighbouring lanes store neighbouring elements.  8192 tokens of 8 rows of 2050 bf16, with a base, 92 us (an element a lane at a time 128).
template <typename TY, typename TO, bool ONE>   // ONE: a block's warps have one token
__global__ void __launch_bounds__(kCombineThreads) k_combine_any(const __grid_constant__ CombineArgs a) {
  constexpr int R = 4, V = 16 / sizeof(TY), kCols = 32 * V;
  __shared__ float turn[kCombineThreads / 32][kCols];
  const int lane = threadIdx.x & 31;
  const int chunks = (a.D + kCols - 1) / kCols;
  const int64_t task = (int64_t)blockIdx.x * (kCombineThreads / 32) + (threadIdx.x >> 5);
  const int64_t t = ONE ? (int64_t)blockIdx.x : task / chunks;
  const int chunk = ONE ? (int)(blockIdx.y * (kCombineThreads / 32) + (threadIdx.x >> 5)) : (int)(task - t * chunks);
  if (t >= a.T || chunk >= chunks) return;   // (whole warps)
  const int d0 = chunk * kCols, d = d0 + lane * V;
  const int bytes = min(a.D - d, V) * (int)sizeof(TY);   // (not above 0: nothing)
  float s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) s[i] = 0.f;
  const TO* base = static_cast<const TO*>(a.base) + t * a.base_ld;
  TO* out = static_cast<TO*>(a.out) + t * a.out_ld;
  float held[V];   // base, of the elements that the lane stores
#pragma unroll
  for (int i = 0; i < V; ++i) {
    held[i] = 0.f;
    if (a.base && d0 + 32 * i + lane < a.D) {
      if constexpr (sizeof(TO) == 4) held[i] = base[d0 + 32 * i + lane];
      else held[i] = __bfloat162float(base[d0 + 32 * i + lane]);
    }
  }
  int pn[R];   // of the next four rows, requested while these are on their way
  float wn[R];
  const auto take = [&](int j0) {
#pragma unroll
    for (int j = 0; j < R; ++j) {
      pn[j] = j0 + j < a.k ? __ldg(a.places + t * a.k + j0 + j) : -1;
      wn[j] = j0 + j < a.k ? __ldg(a.weights + t * a.k + j0 + j) : 0.f;
    }
  };
  take(0);
  for (int j0 = 0; j0 < a.k; j0 += R) {
    uint4 lo[R], hi[R];
    int p[R];
    float w[R];
    uint32_t off[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
      p[j] = (unsigned)pn[j] < (unsigned)a.P ? pn[j] : -1;
      w[j] = wn[j];
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      lo[j] = hi[j] = make_uint4(0u, 0u, 0u, 0u);
      const uint8_t* at = reinterpret_cast<const uint8_t*>(static_cast<const TY*>(a.y) + (int64_t)max(p[j], 0) * a.y_ld + d);
      off[j] = (uint32_t)(reinterpret_cast<uintptr_t>(at) & 15);
      const uint4* q = reinterpret_cast<const uint4*>(at - off[j]);
      if (p[j] >= 0 && bytes > 0) lo[j] = __ldg(q);
      if (p[j] >= 0 && (int)off[j] + bytes > 16) hi[j] = __ldg(q + 1);
    }
    if (j0 + R < a.k) take(j0 + R);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (p[j] < 0) continue;
      uint32_t v[8] = {lo[j].x, lo[j].y, lo[j].z, lo[j].w, hi[j].x, hi[j].y, hi[j].z, hi[j].w};
      if (off[j] & 8)
#pragma unroll
        for (int i = 0; i < 6; ++i) v[i] = v[i + 2];
      if (off[j] & 4)
#pragma unroll
        for (int i = 0; i < 5; ++i) v[i] = v[i + 1];
      if constexpr (sizeof(TY) == 2) {
        const uint32_t sh = (off[j] & 2) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __funnelshift_r(v[i], v[i + 1], sh);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float e;
        if constexpr (sizeof(TY) == 4) e = __uint_as_float(v[i]);
        else e = i & 1 ? bf16hi(v[i / 2]) : bf16lo(v[i / 2]);
        s[i] = fmaf(w[j], e, s[i]);   // (what lies past the columns is not stored)
      }
    }
  }
  float* mine = turn[threadIdx.x >> 5];
#pragma unroll
  for (int i = 0; i < V / 4; ++i) reinterpret_cast<float4*>(mine)[V / 4 * lane + i] = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int c = 32 * i + lane;
    if (d0 + c >= a.D) break;
    const float v = a.base ? held[i] + mine[c] : mine[c];
    if constexpr (sizeof(TO) == 4) out[d0 + c] = v;
    else out[d0 + c] = __float2bfloat16_rn(v);
  }
}

template <typename TY, typename TO>
cudaError_t launch_combine(CombineArgs a, cudaStream_t st) {
  constexpr int V = sizeof(TY) == 4 ? 4 : 8;
  const auto on = [&](const void* p, int64_t ld, int size) {
    const int64_t to = std::min(16, V * size);
    return reinterpret_cast<uintptr_t>(p) % to == 0 && (ld * size) % to == 0;
  };
  if (a.D % V || !on(a.y, a.y_ld, sizeof(TY)) || !on(a.out, a.T == 1 ? 0 : a.out_ld, sizeof(TO)) || !on(a.base, a.T == 1 ? 0 : a.base_ld, sizeof(TO))) {
    const int chunks = (a.D + 32 * V - 1) / (32 * V), per = kCombineThreads / 32;
    if (chunks > per / 2) k_combine_any<TY, TO, true><<<dim3((unsigned)a.T, (unsigned)((chunks + per - 1) / per)), kCombineThreads, 0, st>>>(a);
    else k_combine_any<TY, TO, false><<<(unsigned)(((int64_t)a.T * chunks + per - 1) / per), kCombineThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  const int pieces = a.D / V;
  a.shift = 0;
  while (a.shift < 8 && 1 << a.shift < pieces) ++a.shift;
  const int per = kCombineThreads >> a.shift;
  const auto go = [&](auto kern) {
    kern<<<dim3((unsigned)((a.T + per - 1) / per), (unsigned)((pieces + (1 << a.shift) - 1) >> a.shift)), kCombineThreads, 0, st>>>(a);
    return cudaGetLastError();
  };
  if (per == 1) return a.k <= 2 ? go(k_combine<TY, TO, V, 2, true>) : go(k_combine<TY, TO, V, 8, true>);
  return a.k <= 2 ? go(k_combine<TY, TO, V, 2, false>) : go(k_combine<TY, TO, V, 8, false>);
}

}  // namespace

extern "C" size_t bitsmoe_route_workspace_bytes(int T, int E, int top_k) {
  if (!route_sizes_ok(T, E, top_k) || route_blocks(T) == 1) return 0;
  return (size_t)route_blocks(T) * E * 4;
}

extern "C" int bitsmoe_route(const float* logits, int64_t ld, int T, int E, int top_k, int renormalize, int32_t* experts,
                             float* weights, int32_t* offsets, int32_t* pairs, int32_t* places, void* ws, size_t ws_bytes,
                             void* stream) {
  if (T < 0 || E < 1 || top_k < 1 || top_k > std::min(E, kMaxTopK) || ld < E) return BITSMOE_ERR_INVALID_ARG;
  if (!route_sizes_ok(T, E, top_k)) return BITSMOE_ERR_SHAPE;
  if (!offsets || (T > 0 && (!logits || !experts || !weights || !pairs || !places))) return BITSMOE_ERR_INVALID_ARG;
  const auto odd = [](const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (odd(logits, 4) || odd(experts, 4) || odd(weights, 4) || odd(offsets, 4) || odd(pairs, 4) || odd(places, 4) || odd(ws, 16))
    return BITSMOE_ERR_ALIGNMENT;
  const size_t need = bitsmoe_route_workspace_bytes(T, E, top_k);
  if (ws_bytes < need || (need && !ws)) return BITSMOE_ERR_WORKSPACE_TOO_SMALL;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (T == 0) {
    k_route_none<<<1, 256, 0, st>>>(offsets, E);
    e = cudaGetLastError();
  } else {
    const int blocks = route_blocks(T);
    const RouteArgs a{logits, ld, T, E, top_k, renormalize, route_per(T), experts, weights, offsets, pairs, places, static_cast<int32_t*>(ws)};
    e = E <= 32    ? launch_route<1>(a, blocks, st)
        : E <= 64  ? launch_route<2>(a, blocks, st)
        : E <= 128 ? launch_route<4>(a, blocks, st)
        : E <= 256 ? launch_route<8>(a, blocks, st)
        : E <= 512 ? launch_route<16>(a, blocks, st)
                   : launch_route<32>(a, blocks, st);
  }
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}

extern "C" int bitsmoe_expert_combine(const void* y, int y_type, int64_t y_ld, int P, const int32_t* places, const float* weights,
                                      int T, int top_k, int D, const void* base, int64_t base_ld, void* out, int out_type,
                                      int64_t out_ld, void* stream) {
  if (T < 0 || P < 0 || top_k < 1 || top_k > kMaxTopK || D < 1 || !dense_type_ok(y_type) || !dense_type_ok(out_type))
    return BITSMOE_ERR_INVALID_ARG;
  if (T > kMaxMicroRows || P > kMaxMicroRows || D > kMaxMicroCols) return BITSMOE_ERR_SHAPE;
  if (y_ld < D || out_ld < D || (base && base_ld < D)) return BITSMOE_ERR_INVALID_ARG;
  if (T == 0) return BITSMOE_OK;
  if ((!y && P > 0) || !places || !weights || !out) return BITSMOE_ERR_INVALID_ARG;
  if (base == out && base_ld != out_ld && T > 1) return BITSMOE_ERR_INVALID_ARG;
  const auto odd = [](const void* p, int to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (odd(y, dense_size(y_type)) || odd(out, dense_size(out_type)) || odd(base, dense_size(out_type)) || odd(places, 4) || odd(weights, 4))
    return BITSMOE_ERR_ALIGNMENT;
  CombineArgs a{y, y_ld, T, P, top_k, D, 0, places, weights, base, base_ld, out, out_ld};
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool yf = y_type == BITSMOE_F32, of = out_type == BITSMOE_F32;
  const cudaError_t e = yf ? (of ? launch_combine<float, float>(a, st) : launch_combine<float, __nv_bfloat16>(a, st))
                           : (of ? launch_combine<__nv_bfloat16, float>(a, st) : launch_combine<__nv_bfloat16, __nv_bfloat16>(a, st));
  return e == cudaSuccess ? BITSMOE_OK : record_cuda_error((int)e);
}
