// Tokens to their experts and back (pgc_route, pgc_spread, pgc_join, pgc_join_grad).
//
// A router chose k experts for each of T tokens: slot s = t k + j holds an
// expert or nothing.  Slots sorted by expert, in their order within one, give
//   place[s] = offsets[e] + number of slots before s that hold e,
// and, with rows[place[t, j]] the row that expert made of token t,
//   spread     rows[place[t, j]] = x[t]
//   join       y[t] = sum_j w[t, j] rows[place[t, j]]       (weights 1: the gradient of spread)
//   join_grad  drows[place[t, j]] = w[t, j] dy[t],  dw[t, j] = <dy[t], rows[place[t, j]]>.
// All three go through the rows token by token, so that a token's own row is
// read or written once.
#include <algorithm>
#include <initializer_list>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxExperts = 1024, kMaxChoices = 64;

// ---- sorting -------------------------------------------------------------------
// A CTA has consecutive slots, and each of its warps consecutive ones of these:
// counts per warp and expert, summed up over warps and CTAs before, say where a warp's
// first slot of each expert goes; within 32 slots a lane's rank is the number of
// lanes before it that hold the same expert.  Nothing depends on the order of atomics.

struct Route {
  const int32_t* choice;
  int32_t *place, *slot, *offsets;
  int32_t* counts;              // [CTAs][E]
  int n, E;                     // slots, experts
  int per;                      // slots of a CTA, a multiple of 32 kRouteWarps
};
__device__ __forceinline__ int expert_of(const Route& a, int s) {
  const int e = s < a.n ? a.choice[s] : -1;
  return e >= 0 && e < a.E ? e : -1;
}

constexpr int kRouteThreads = 512, kRouteWarps = kRouteThreads / 32;

// The exclusive running sum over the CTA's threads; total in *sum.
__device__ __forceinline__ int before_me(int v, int* red, int* sum) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int up = v;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int q = __shfl_up_sync(0xffffffffu, up, o);
    if (lane >= o) up += q;
  }
  if (lane == 31) red[warp] = up;
  __syncthreads();
  int base = 0, all = 0;
  for (int w = 0; w < kRouteWarps; ++w) {
    base += w < warp ? red[w] : 0;
    all += red[w];
  }
  __syncthreads();
  *sum = all;
  return base + up - v;
}
__device__ __forceinline__ void clear(int32_t* p, int n) {
  for (int i = threadIdx.x; i < n; i += kRouteThreads) p[i] = 0;
}

// Counts of every expert among a CTA's slots.
__global__ void __launch_bounds__(kRouteThreads) count_kernel(Route a) {
  __shared__ int32_t count[kMaxExperts];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  clear(count, a.E);
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * a.per, last = min(first + a.per, (int64_t)a.n);
  for (int64_t s = first + threadIdx.x; s < last; s += kRouteThreads) {
    const int e = expert_of(a, (int)s);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) a.counts[(int64_t)blockIdx.x * a.E + e] = count[e];
}

// kAlone: one CTA has all slots, and counts them itself.
template <bool kAlone>
__global__ void __launch_bounds__(kRouteThreads) place_kernel(Route a) {
  extern __shared__ int32_t next[];              // [kRouteWarps][E]: the row of a warp's next slot of an expert
  __shared__ int32_t total[kMaxExperts], base[kMaxExperts];
  __shared__ int red[kRouteWarps];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t cta = (int64_t)blockIdx.x * a.per, first = cta + (int64_t)warp * (a.per / kRouteWarps);
  const int64_t last = min(first + a.per / kRouteWarps, (int64_t)a.n);
  clear(next, kRouteWarps * a.E);
  clear(total, a.E);
  clear(base, a.E);
  __syncthreads();
  for (int64_t s = first + lane; s < last; s += 32) {
    const int e = expert_of(a, (int)s);
    if (e >= 0) atomicAdd(&next[warp * a.E + e], 1);
  }
  if (!kAlone) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    // counts of all CTAs, and of those before this one: as many threads to an expert as there are
    const int groups = max(kRouteThreads / a.E, 1), group = threadIdx.x / a.E;
    const int width = groups > 1 ? a.E : kRouteThreads;
    if (group < groups)
      for (int e = threadIdx.x - group * width; e < a.E; e += width) {
        int all = 0, before = 0;
#pragma unroll 8
        for (int b = group; b < (int)gridDim.x; b += groups) {
          const int c = __ldcg(a.counts + (int64_t)b * a.E + e);
          all += c;
          before += b < (int)blockIdx.x ? c : 0;
        }
        atomicAdd(&total[e], all);
        atomicAdd(&base[e], before);
      }
  }
  __syncthreads();
  // first row of every expert; a thread has two consecutive ones
  const int e0 = 2 * threadIdx.x;
  int c[2] = {0, 0};
  for (int i = 0; i < 2; ++i) {
    if (e0 + i >= a.E) continue;
    if (kAlone)
      for (int w = 0; w < kRouteWarps; ++w) c[i] += next[w * a.E + e0 + i];
    else
      c[i] = total[e0 + i];
  }
  int rows;
  int at = before_me(c[0] + c[1], red, &rows);
  for (int i = 0; i < 2; ++i) {
    if (e0 + i >= a.E) continue;
    if (blockIdx.x == 0) a.offsets[e0 + i] = at;
    base[e0 + i] += at;
    at += c[i];
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[a.E] = rows;
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) {
    int row = base[e];
    for (int w = 0; w < kRouteWarps; ++w) {
      const int count = next[w * a.E + e];
      next[w * a.E + e] = row;
      row += count;
    }
  }
  __syncthreads();
  for (int64_t s0 = first; s0 < last; s0 += 32) {
    const int64_t s = s0 + lane;
    const int e = s < last ? expert_of(a, (int)s) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    int row = -1;
    if (e >= 0) row = next[warp * a.E + e] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (e >= 0) {
      if (lane == __ffs(same) - 1) next[warp * a.E + e] += __popc(same);
      a.slot[row] = (int)s;
    }
    if (s < last) a.place[s] = row;
    __syncwarp();
  }
  // rows that no slot has
  for (int64_t i = rows + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; i < a.n; i += (int64_t)gridDim.x * kRouteThreads)
    a.slot[i] = -1;
}

// ---- rows ----------------------------------------------------------------------
// A row is read and written in pieces of W bytes, the most that all rows' starts
// allow, and single elements behind the last piece.

struct Move {
  const void* x;                // spread: tokens; join, join_grad: the experts' rows
  const void* dy;               // join_grad
  void* out;                    // spread: the experts' rows; join: tokens; join_grad: gradient of the experts' rows
  const int32_t* place;
  const float* weight;
  float* dweight;
  int64_t T, rows, ldx, ldy, ldo;
  int k, d;
  int chunks;                   // parts of a row, each a warp's
};

template <int W> struct RawOf;
template <> struct RawOf<16> { using T = uint4; };
template <> struct RawOf<8> { using T = uint2; };
template <> struct RawOf<4> { using T = uint32_t; };
template <> struct RawOf<2> { using T = uint16_t; };

template <typename E, int W>
struct Piece {
  using Raw = typename RawOf<W>::T;
  static constexpr int N = W / (int)sizeof(E);
  Raw raw;
  __device__ __forceinline__ void widen(float (&f)[N]) const {
    if constexpr (sizeof(E) == 4) {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = __uint_as_float(w[i]);
    } else if constexpr (W == 2) {
      f[0] = __uint_as_float((uint32_t)raw << 16);
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        f[i] = __uint_as_float(w[i / 2] << 16);
        f[i + 1] = __uint_as_float(w[i / 2] & 0xffff0000u);
      }
    }
  }
  __device__ __forceinline__ void narrow(const float (&f)[N]) {
    if constexpr (sizeof(E) == 4) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(f[i]);
    } else if constexpr (W == 2) {
      raw = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else {
      uint32_t* w = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
      for (int i = 0; i < N; i += 2) w[i / 2] = Elem<__nv_bfloat16>::two(pair(f[i], f[i + 1]));
    }
  }
};

// The rows of a token's slots: lane j has those of slots j and j + 32, -1 without one.
struct Places {
  int lo, hi;
  __device__ __forceinline__ Places(const Move& a, int64_t t) {
    const int lane = threadIdx.x % 32;
    lo = row(a, t, lane);
    hi = a.k > 32 ? row(a, t, lane + 32) : -1;
  }
  __device__ __forceinline__ static int row(const Move& a, int64_t t, int j) {
    const int r = j < a.k ? a.place[t * a.k + j] : -1;
    return r >= 0 && r < a.rows ? r : -1;
  }
  __device__ __forceinline__ int operator[](int j) const { return __shfl_sync(0xffffffffu, j < 32 ? lo : hi, j & 31); }
};
// The same for the weights (1 where there are none).
struct Weights {
  float lo, hi;
  __device__ __forceinline__ Weights(const Move& a, int64_t t) {
    const int lane = threadIdx.x % 32;
    lo = a.weight && lane < a.k ? a.weight[t * a.k + lane] : 1.f;
    hi = a.weight && lane + 32 < a.k ? a.weight[t * a.k + lane + 32] : 1.f;
  }
  __device__ __forceinline__ float operator[](int j) const { return __shfl_sync(0xffffffffu, j < 32 ? lo : hi, j & 31); }
};

template <int W>
constexpr int spread_pieces() { return W == 16 ? 4 : 8; }       // a lane has in flight

template <typename E, int W>
__global__ void __launch_bounds__(kThreads) spread_kernel(Move a) {
  constexpr int N = Piece<E, W>::N, U = spread_pieces<W>();
  using Raw = typename RawOf<W>::T;
  const int lane = threadIdx.x % 32;
  const int64_t unit = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  const int64_t t = unit / a.chunks;
  if (t >= a.T) return;
  const int chunk = (int)(unit - t * a.chunks), pieces = a.d / N, p0 = chunk * (32 * U) + lane;
  const E* x = static_cast<const E*>(a.x) + t * a.ldx;
  const Places at(a, t);
  Raw v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (p0 + 32 * u < pieces) v[u] = reinterpret_cast<const Raw*>(x)[p0 + 32 * u];
  const int rest = chunk == a.chunks - 1 && lane < a.d - pieces * N ? pieces * N + lane : -1;
  const E last = rest >= 0 ? x[rest] : E();
  for (int j = 0; j < a.k; ++j) {
    const int r = at[j];
    if (r < 0) continue;
    E* out = static_cast<E*>(a.out) + r * a.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p0 + 32 * u < pieces) reinterpret_cast<Raw*>(out)[p0 + 32 * u] = v[u];
    if (rest >= 0) out[rest] = last;
  }
}

template <int W>
constexpr int join_pieces() { return W == 16 ? 2 : 4; }
constexpr int kJoinAtOnce = 4;        // rows a lane has in flight

template <typename E, int W>
__global__ void __launch_bounds__(kThreads) join_kernel(Move a) {
  constexpr int N = Piece<E, W>::N, U = join_pieces<W>();
  using Raw = typename RawOf<W>::T;
  const int lane = threadIdx.x % 32;
  const int64_t unit = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  const int64_t t = unit / a.chunks;
  if (t >= a.T) return;
  const int chunk = (int)(unit - t * a.chunks), pieces = a.d / N, p0 = chunk * (32 * U) + lane;
  const int rest = chunk == a.chunks - 1 && lane < a.d - pieces * N ? pieces * N + lane : -1;
  const Places at(a, t);
  const Weights w(a, t);
  float sum[U][N], sum_rest = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < N; ++i) sum[u][i] = 0.f;
  for (int j0 = 0; j0 < a.k; j0 += kJoinAtOnce) {
    Piece<E, W> v[kJoinAtOnce][U];
    int r[kJoinAtOnce];
    float wj[kJoinAtOnce];
#pragma unroll
    for (int q = 0; q < kJoinAtOnce; ++q) {
      r[q] = j0 + q < a.k ? at[j0 + q] : -1;
      wj[q] = j0 + q < a.k ? w[j0 + q] : 0.f;
      if (r[q] < 0) continue;
      const E* x = static_cast<const E*>(a.x) + r[q] * a.ldx;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p0 + 32 * u < pieces) v[q][u].raw = reinterpret_cast<const Raw*>(x)[p0 + 32 * u];
    }
#pragma unroll
    for (int q = 0; q < kJoinAtOnce; ++q) {
      if (r[q] < 0) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (p0 + 32 * u >= pieces) continue;
        float f[N];
        v[q][u].widen(f);
#pragma unroll
        for (int i = 0; i < N; ++i) sum[u][i] = fmaf(wj[q], f[i], sum[u][i]);
      }
      if (rest >= 0) sum_rest = fmaf(wj[q], Elem<E>::get(static_cast<const E*>(a.x) + r[q] * a.ldx + rest), sum_rest);
    }
  }
  E* out = static_cast<E*>(a.out) + t * a.ldo;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (p0 + 32 * u >= pieces) continue;
    Piece<E, W> v;
    v.narrow(sum[u]);
    reinterpret_cast<Raw*>(out)[p0 + 32 * u] = v.raw;
  }
  if (rest >= 0) Elem<E>::put(out + rest, sum_rest);
}

constexpr int kGradAtOnce = 8;
// A token per warp (G = 32) or CTA: the products with its own row are summed over all of it.
template <typename E, int W, int G>
__global__ void __launch_bounds__(kThreads) join_grad_kernel(Move a) {
  constexpr int N = Piece<E, W>::N;
  using Raw = typename RawOf<W>::T;
  __shared__ float red[kWarps][kMaxChoices];
  const int lane = threadIdx.x % 32, tid = threadIdx.x % G, warp = threadIdx.x / 32;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + warp : blockIdx.x;
  if (t >= a.T) return;
  const int pieces = a.d / N, rest = tid < a.d - pieces * N ? pieces * N + tid : -1;
  const E* dy = static_cast<const E*>(a.dy) + t * a.ldy;
  const Places at(a, t);
  const Weights w(a, t);
  for (int j0 = 0; j0 < a.k; j0 += kGradAtOnce) {
    const E* x[kGradAtOnce];
    E* out[kGradAtOnce];
    float wj[kGradAtOnce], sum[kGradAtOnce];
#pragma unroll
    for (int q = 0; q < kGradAtOnce; ++q) {
      const int r = j0 + q < a.k ? at[j0 + q] : -1;
      wj[q] = j0 + q < a.k ? w[j0 + q] : 0.f;
      x[q] = r >= 0 ? static_cast<const E*>(a.x) + r * a.ldx : nullptr;
      out[q] = r >= 0 ? static_cast<E*>(a.out) + r * a.ldo : nullptr;
      sum[q] = 0.f;
    }
    for (int p = tid; p < pieces; p += G) {
      Piece<E, W> v[kGradAtOnce], own;
      own.raw = reinterpret_cast<const Raw*>(dy)[p];
#pragma unroll
      for (int q = 0; q < kGradAtOnce; ++q)
        if (x[q]) v[q].raw = reinterpret_cast<const Raw*>(x[q])[p];
      float d[N];
      own.widen(d);
#pragma unroll
      for (int q = 0; q < kGradAtOnce; ++q) {
        if (!x[q]) continue;
        float f[N];
        v[q].widen(f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          sum[q] = fmaf(d[i], f[i], sum[q]);
          f[i] = wj[q] * d[i];
        }
        v[q].narrow(f);
        reinterpret_cast<Raw*>(out[q])[p] = v[q].raw;
      }
    }
    if (rest >= 0) {
      const float d = Elem<E>::get(dy + rest);
#pragma unroll
      for (int q = 0; q < kGradAtOnce; ++q) {
        if (!x[q]) continue;
        sum[q] = fmaf(d, Elem<E>::get(x[q] + rest), sum[q]);
        Elem<E>::put(out[q] + rest, wj[q] * d);
      }
    }
#pragma unroll
    for (int q = 0; q < kGradAtOnce; ++q) {
      sum[q] = warp_sum(sum[q]);
      if (lane == 0 && j0 + q < a.k) {
        if (G == 32) a.dweight[t * a.k + j0 + q] = sum[q];
        else red[warp][j0 + q] = sum[q];
      }
    }
  }
  if (G == 32) return;
  __syncthreads();
  if (threadIdx.x < a.k) {
    float sum = 0.f;
    for (int i = 0; i < kWarps; ++i) sum += red[i][threadIdx.x];
    a.dweight[t * a.k + threadIdx.x] = sum;
  }
}

// ---- host --------------------------------------------------------------------

constexpr int64_t kFarPitch = int64_t(1) << 31;
constexpr size_t kPlainSmem = 36 * 1024;         // beside 8 KB of fixed size, without asking

int check_sizes(int64_t tokens, int32_t k) {
  if (tokens < 0 || k < 1 || tokens > INT32_MAX / k) return PGC_EINVAL;
  return k > kMaxChoices ? PGC_ENOTSUP : PGC_OK;
}
// Rows of d elements: `count` of them at p, each `ld` behind the last.
bool bad_rows(const void* p, int64_t count, int64_t d, int64_t ld, uintptr_t size) {
  return ld < d || ld > kFarPitch || (count && !p) || (uintptr_t)p % size;
}
int check_move(int32_t dtype, int64_t tokens, int32_t k, int64_t d, int64_t rows, const int32_t* place) {
  if (dtype != PGC_F32 && dtype != PGC_BF16) return PGC_EINVAL;
  if (tokens < 0 || k < 1 || tokens > INT32_MAX / k || d < 1 || d > INT32_MAX || rows < 0 || rows > INT32_MAX) return PGC_EINVAL;
  return (tokens && !place) || (uintptr_t)place % 4 ? PGC_EINVAL : PGC_OK;
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 148;
  return n;
}

// CTAs of a large sort: 1024 slots each at least.  Up to 8192 slots one CTA does it all.
constexpr int kAloneSlots = 8192, kMostRouteCtas = 128;
int route_ctas(int64_t n) { return (int)std::min<int64_t>((n + 1023) / 1024, kMostRouteCtas); }

// The most bytes that divide every row's start.
int width_of(std::initializer_list<uintptr_t> starts) {
  uintptr_t all = 16;
  for (const uintptr_t p : starts) all |= p;
  return (int)(all & (~all + 1));
}
// f.template operator()<E, W>()
template <typename F>
cudaError_t by_width(int32_t dtype, int width, F f) {
  using H = __nv_bfloat16;
  if (dtype == PGC_F32) {
    if (width >= 16) return f.template operator()<float, 16>();
    if (width >= 8) return f.template operator()<float, 8>();
    return f.template operator()<float, 4>();
  }
  if (width >= 16) return f.template operator()<H, 16>();
  if (width >= 8) return f.template operator()<H, 8>();
  if (width >= 4) return f.template operator()<H, 4>();
  return f.template operator()<H, 2>();
}
// Warps for T rows in chunks of 32 U pieces, and the chunks; too many warps for a grid of CTAs are refused by the launch.
unsigned grid_of(Move& a, int n, int u) {
  a.chunks = std::max((a.d / n + 32 * u - 1) / (32 * u), 1);
  return (unsigned)((a.T * a.chunks + kWarps - 1) / kWarps);
}
struct Spread {
  Move a;
  cudaStream_t st;
  template <typename E, int W> cudaError_t operator()() {
    const unsigned grid = grid_of(a, Piece<E, W>::N, spread_pieces<W>());
    spread_kernel<E, W><<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
};
struct Join {
  Move a;
  cudaStream_t st;
  template <typename E, int W> cudaError_t operator()() {
    const unsigned grid = grid_of(a, Piece<E, W>::N, join_pieces<W>());
    join_kernel<E, W><<<grid, kThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
};
// A warp per token where there are tokens for the SMs' warps, else a CTA.
struct JoinGrad {
  Move a;
  cudaStream_t st;
  template <typename E, int W> cudaError_t operator()() {
    if (a.T >= sm_count() * 32) join_grad_kernel<E, W, 32><<<(unsigned)((a.T + kWarps - 1) / kWarps), kThreads, 0, st>>>(a);
    else join_grad_kernel<E, W, kThreads><<<(unsigned)a.T, kThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
};

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_route_workspace(int64_t tokens, int32_t k, int32_t experts, int64_t *bytes) {
  if (!bytes || tokens < 0 || k < 1 || tokens > INT32_MAX / k || experts < 1) return PGC_EINVAL;
  if (experts > kMaxExperts || k > kMaxChoices) return PGC_ENOTSUP;
  const int64_t n = tokens * k;
  *bytes = n <= kAloneSlots ? 16 : (int64_t)route_ctas(n) * experts * 4;
  return PGC_OK;
}

int pgc_route(int64_t tokens, int32_t k, int32_t experts, const int32_t *choice, int32_t *place, int32_t *slot,
              int32_t *offsets, void *workspace, int64_t workspace_bytes, void *stream) {
  int64_t need = 0;
  const int rc = pgc_route_workspace(tokens, k, experts, &need);
  if (rc) return rc;
  if (!offsets || (tokens && (!choice || !place || !slot)) || !workspace) return PGC_EINVAL;
  if ((uintptr_t)choice % 4 || (uintptr_t)place % 4 || (uintptr_t)slot % 4 || (uintptr_t)offsets % 4 || (uintptr_t)workspace % 16)
    return PGC_EINVAL;
  if (workspace_bytes < need) return PGC_ESCRATCH;
  const int64_t n = tokens * k;
  const cudaStream_t st = (cudaStream_t)stream;
  const int ctas = n <= kAloneSlots ? 1 : route_ctas(n), grain = 32 * kRouteWarps;
  const int64_t per = ((n + ctas - 1) / ctas + grain - 1) / grain * grain;
  const Route a{choice, place, slot, offsets, static_cast<int32_t*>(workspace), (int)n, experts, (int)per};
  const size_t smem = (size_t)kRouteWarps * experts * 4;
  const auto kernel = ctas == 1 ? place_kernel<true> : place_kernel<false>;
  if (smem > kPlainSmem) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRouteWarps * kMaxExperts * 4);
    if (e != cudaSuccess) return report_cuda(e);
  }
  if (ctas > 1) {
    count_kernel<<<ctas, kRouteThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return report_cuda(e);
  }
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kRouteThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = ctas > 1 ? 1 : 0;
  return report_cuda(cudaLaunchKernelEx(&cfg, kernel, a));
}

int pgc_spread(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *x, int64_t ld, const int32_t *place,
               int64_t rows, void *out, int64_t out_ld, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(x, tokens, d, ld, size) || bad_rows(out, rows, d, out_ld, size)) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens || !rows) return rc;
  Move a{};
  a.x = x; a.out = out; a.place = place; a.T = tokens; a.rows = rows; a.ldx = ld; a.ldo = out_ld; a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  const int width = width_of({(uintptr_t)x, (uintptr_t)out, (uintptr_t)ld * size, (uintptr_t)out_ld * size});
  return report_cuda(by_width(dtype, width, Spread{a, st}));
}

int pgc_join(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *rows_in, int64_t ld, int64_t rows,
             const int32_t *place, const float *weight, void *out, int64_t out_ld, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(rows_in, rows, d, ld, size) || bad_rows(out, tokens, d, out_ld, size) || (uintptr_t)weight % 4) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens) return rc;
  Move a{};
  a.x = rows_in; a.out = out; a.place = place; a.weight = weight; a.T = tokens; a.rows = rows; a.ldx = ld; a.ldo = out_ld;
  a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  const int width = width_of({(uintptr_t)rows_in, (uintptr_t)out, (uintptr_t)ld * size, (uintptr_t)out_ld * size});
  return report_cuda(by_width(dtype, width, Join{a, st}));
}

int pgc_join_grad(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *dy, int64_t dy_ld, const void *rows_in,
                  int64_t ld, int64_t rows, const int32_t *place, const float *weight, void *drows, int64_t drows_ld,
                  float *dweight, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(dy, tokens, d, dy_ld, size) || bad_rows(rows_in, rows, d, ld, size) || bad_rows(drows, rows, d, drows_ld, size))
    return PGC_EINVAL;
  if ((tokens && (!weight || !dweight)) || (uintptr_t)weight % 4 || (uintptr_t)dweight % 4) return PGC_EINVAL;
  if (drows && drows == rows_in && drows_ld != ld) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens) return rc;
  Move a{};
  a.x = rows_in; a.dy = dy; a.out = drows; a.place = place; a.weight = weight; a.dweight = dweight;
  a.T = tokens; a.rows = rows; a.ldx = ld; a.ldy = dy_ld; a.ldo = drows_ld; a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  const int width = width_of({(uintptr_t)dy, (uintptr_t)rows_in, (uintptr_t)drows, (uintptr_t)dy_ld * size,
                              (uintptr_t)ld * size, (uintptr_t)drows_ld * size});
  return report_cuda(by_width(dtype, width, JoinGrad{a, st}));
}

}  // extern "C"
