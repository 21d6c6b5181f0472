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
#pragma unroll 4
  for (int64_t s = first + threadIdx.x; s < last; s += kRouteThreads) {
    const int e = expert_of(a, (int)s);
    if (e >= 0) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kRouteThreads) a.counts[(int64_t)blockIdx.x * a.E + e] = count[e];
}

// counts[c][e] becomes what CTAs before c count, and counts[CTAs][e] what all do: 32 experts a CTA, CTAs
// in sixteen parts, a warp each, whose counts stay in registers between their sum and their places.
constexpr int kMostRouteCtas = 256, kPartCtas = kMostRouteCtas / kRouteWarps;
__global__ void __launch_bounds__(kRouteThreads) prefix_kernel(Route a, int ctas) {
  __shared__ int32_t sum[kRouteWarps][32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, e = blockIdx.x * 32 + lane;
  const int per = (ctas + kRouteWarps - 1) / kRouteWarps, first = warp * per;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int32_t c[kPartCtas], all = 0;
#pragma unroll
  for (int i = 0; i < kPartCtas; ++i) {
    c[i] = i < per && first + i < ctas && e < a.E ? __ldcg(a.counts + (int64_t)(first + i) * a.E + e) : 0;
    all += c[i];
  }
  sum[warp][lane] = all;
  __syncthreads();
  if (e >= a.E) return;
  int32_t before = 0;
  for (int w = 0; w < warp; ++w) before += sum[w][lane];
#pragma unroll
  for (int i = 0; i < kPartCtas; ++i)
    if (i < per && first + i < ctas) {
      a.counts[(int64_t)(first + i) * a.E + e] = before;
      before += c[i];
    }
  if (warp == kRouteWarps - 1) a.counts[(int64_t)ctas * a.E + e] = before;
}

// kAlone: one CTA has all slots, and counts them itself.
template <bool kAlone>
__global__ void __launch_bounds__(kRouteThreads) place_kernel(Route a) {
  extern __shared__ int32_t next[];              // [kRouteWarps][E]: the row of a warp's next slot of an expert
  __shared__ int32_t base[kMaxExperts];
  __shared__ int red[kRouteWarps];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t cta = (int64_t)blockIdx.x * a.per, first = cta + (int64_t)warp * (a.per / kRouteWarps);
  const int64_t last = min(first + a.per / kRouteWarps, (int64_t)a.n);
  clear(next, kRouteWarps * a.E);
  __syncthreads();
#pragma unroll 4
  for (int64_t s = first + lane; s < last; s += 32) {
    const int e = expert_of(a, (int)s);
    if (e >= 0) atomicAdd(&next[warp * a.E + e], 1);
  }
  if (!kAlone) asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();
  // first row of every expert; a thread has two consecutive ones
  const int e0 = 2 * threadIdx.x;
  int c[2] = {0, 0};
  for (int i = 0; i < 2; ++i) {
    if (e0 + i >= a.E) continue;
    if (kAlone)
      for (int w = 0; w < kRouteWarps; ++w) c[i] += next[w * a.E + e0 + i];
    else
      c[i] = __ldcg(a.counts + (int64_t)gridDim.x * a.E + e0 + i);
  }
  int rows;
  int at = before_me(c[0] + c[1], red, &rows);
  for (int i = 0; i < 2; ++i) {
    if (e0 + i >= a.E) continue;
    if (blockIdx.x == 0) a.offsets[e0 + i] = at;
    base[e0 + i] = at + (kAlone ? 0 : __ldcg(a.counts + (int64_t)blockIdx.x * a.E + e0 + i));
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
  int ahead = first + lane < last ? expert_of(a, (int)(first + lane)) : -1;
  for (int64_t s0 = first; s0 < last; s0 += 32) {
    const int64_t s = s0 + lane;
    const int e = ahead;
    ahead = s + 32 < last ? expert_of(a, (int)s + 32) : -1;
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
// A lane has pieces of W bytes of a row: 16 where every row starts on 16 bytes, else 4, or 2 where bf16
// rows start between two words.  (16-byte pieces put together from the two that hold them were slower: 90
// instructions a piece, 109 us where 4-byte pieces take 55: join of 10000 x 6 x 1001 fp32.)  What is left
// behind the last piece is taken by single elements.  All three kernels are bound by memory:
// at 16 bytes they move 6.1 to 6.6 TB/s (bf16, 16384 x 8 x 2048: spread 95 us, join 95, gradient 174), at 4 bytes
// fp32 5.1 to 5.8, at 2 bytes 3.2 to 5.0.  16 bytes and 4, bf16: join 8192 x 4 x 5120 67 and 78 us, gradient
// 174 and 199, spread 95 both.

struct Move {
  const void* x;                // spread: tokens; join, join_grad: the experts' rows
  const void* dy;               // join_grad
  void* out;                    // spread: the experts' rows; join: tokens; join_grad: gradient of the experts' rows
  const int32_t* place;
  const float* weight;
  float* dweight;
  int64_t T, rows, ldx, ldy, ldo;
  int k, d;
  int chunks;                   // spread: parts of a row, each a warp's
};

template <typename E, int W>
struct Access;
template <typename E>
struct Access<E, 16> {
  static constexpr int N = Elem<E>::N;
  using Raw = uint4;
  __device__ __forceinline__ static void widen(const Raw& v, float (&f)[N]) {
    Pair h[4];
    Elem<E>::widen(v, h);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) split(h[i], f[2 * i], f[2 * i + 1]);
  }
  __device__ __forceinline__ static Raw narrow(const float (&f)[N]) {
    Pair h[4];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) h[i] = pair(f[2 * i], f[2 * i + 1]);
    return Elem<E>::narrow(h);
  }
};
template <>
struct Access<float, 4> {
  static constexpr int N = 1;
  using Raw = float;
  __device__ __forceinline__ static void widen(Raw v, float (&f)[1]) { f[0] = v; }
  __device__ __forceinline__ static Raw narrow(const float (&f)[1]) { return f[0]; }
};
template <>
struct Access<__nv_bfloat16, 4> {
  static constexpr int N = 2;
  using Raw = uint32_t;
  __device__ __forceinline__ static void widen(Raw v, float (&f)[2]) {
    f[0] = __uint_as_float(v << 16);
    f[1] = __uint_as_float(v & 0xffff0000u);
  }
  __device__ __forceinline__ static Raw narrow(const float (&f)[2]) { return Elem<__nv_bfloat16>::two(pair(f[0], f[1])); }
};
template <>
struct Access<__nv_bfloat16, 2> {
  static constexpr int N = 1;
  using Raw = uint16_t;
  __device__ __forceinline__ static void widen(Raw v, float (&f)[1]) { f[0] = bf16_bits_to_float(v); }
  __device__ __forceinline__ static Raw narrow(const float (&f)[1]) { return __bfloat16_as_ushort(__float2bfloat16_rn(f[0])); }
};
template <typename A, typename E>
__device__ __forceinline__ typename A::Raw load(const E* x) { return *reinterpret_cast<const typename A::Raw*>(x); }
template <typename A, typename E>
__device__ __forceinline__ void store(E* x, const typename A::Raw& v) { *reinterpret_cast<typename A::Raw*>(x) = v; }

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
  // -1 behind the last slot
  __device__ __forceinline__ int operator[](int j) const {
    const int r = __shfl_sync(0xffffffffu, j < 32 ? lo : hi, j & 31);
    return j < kMaxChoices ? r : -1;
  }
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

// Pieces that a lane has in flight: two or four (10000 x 6 x 1001 fp32: 47 us, 52 with half as many; 16384 x 8 x 2048 bf16: 94.5 us,
// 96.5 with twice as many, and few tokens make more warps: 8 x 8 x 2048 2.3 us on the GPU, 3.3).
template <int W>
constexpr int spread_pieces() { return W == 16 ? 2 : 4; }

template <typename E, int W>
__global__ void __launch_bounds__(kThreads) spread_kernel(Move a) {
  using A = Access<E, W>;
  constexpr int N = A::N, U = spread_pieces<W>();
  const int lane = threadIdx.x % 32;
  const int64_t unit = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32;
  const int64_t t = unit / a.chunks;
  if (t >= a.T) return;
  const int chunk = (int)(unit - t * a.chunks), pieces = a.d / N, p0 = chunk * (32 * U) + lane;
  const int rest = chunk == a.chunks - 1 && lane < a.d - pieces * N ? pieces * N + lane : -1;
  const E* x = static_cast<const E*>(a.x) + t * a.ldx;
  const Places at(a, t);
  typename A::Raw v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (p0 + 32 * u < pieces) v[u] = load<A>(x + (p0 + 32 * u) * N);
  const E last = rest >= 0 ? x[rest] : E();
  for (int j = 0; j < a.k; ++j) {
    const int r = at[j];
    if (r < 0) continue;
    E* out = static_cast<E*>(a.out) + r * a.ldo;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p0 + 32 * u < pieces) store<A>(out + (p0 + 32 * u) * N, v[u]);
    if (rest >= 0) out[rest] = last;
  }
}

// Rows that a lane has in flight (Q: four, or two where k is no more), and pieces of each: 16384 x 8 x 2048 bf16 95 us, 99 with two
// rows, 158 with eight; 30000 x 2 x 2048 60 us, 63 with four rows of two pieces; 30000 x 2 x 1001 fp32 57, 62 with four of eight;
// 30000 x 2 x 2002 bf16, whose sums are two a piece, 59, with 16 pieces 142.
template <typename E, int W, int Q>
constexpr int join_pieces() { return W == 16 ? (Q == 2 ? 3 : 2) : Q == 4 ? 8 : W > (int)sizeof(E) ? 12 : 16; }

// A token per warp (G = 32) or CTA, in a loop over its row: a warp for each part of a row
// spent its time on the places and weights (8192 x 4 x 5120 bf16: 98 us, 58 this way).
template <typename E, int W, int Q, int G>
__global__ void __launch_bounds__(kThreads, 4) join_kernel(Move a) {
  using A = Access<E, W>;
  constexpr int N = A::N, U = join_pieces<E, W, Q>();
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x;
  if (t >= a.T) return;
  E* out = static_cast<E*>(a.out) + t * a.ldo;
  const int pieces = a.d / N, rest = a.d - pieces * N;
  const Places at(a, t);
  const Weights w(a, t);
  for (int p0 = 0; p0 < pieces; p0 += G * U) {
    const int first = p0 + tid;
    float sum[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < N; ++i) sum[u][i] = 0.f;
    for (int j0 = 0; j0 < a.k; j0 += Q) {
      typename A::Raw v[Q][U];
      int r[Q];
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        r[q] = at[j0 + q];
        if (r[q] < 0) continue;
        const E* x = static_cast<const E*>(a.x) + r[q] * a.ldx + first * N;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (first + u * G < pieces) v[q][u] = load<A>(x + u * G * N);
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        const float wj = w[j0 + q];
        if (r[q] < 0) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (first + u * G >= pieces) continue;
          float f[N];
          A::widen(v[q][u], f);
#pragma unroll
          for (int i = 0; i < N; ++i) sum[u][i] = fmaf(wj, f[i], sum[u][i]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (first + u * G < pieces) store<A>(out + (first + u * G) * N, A::narrow(sum[u]));
  }
  if (rest && (G == 32 || threadIdx.x < 32)) {
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int r = at[j];
      const float wj = w[j];
      if (r >= 0 && tid < rest) sum = fmaf(wj, Elem<E>::get(static_cast<const E*>(a.x) + r * a.ldx + pieces * N + tid), sum);
    }
    if (tid < rest) Elem<E>::put(out + pieces * N + tid, sum);
  }
}

// Pieces of a row that a lane has in flight, with Q rows: as many as registers allow.  30000 x 2 x 2048 bf16 94 us, 101 with one
// of 16 bytes; 15000 x 4 x 1001 fp32 88, 98 with three of 4; 10000 x 6 x 1001 90, 93 with three, 97 with eight; 8000 x 8 x 1001 104, 109 with four.
template <int W, int Q>
constexpr int grad_pieces() { return W == 16 ? (Q <= 4 ? 2 : 1) : Q == 8 ? 3 : Q == 6 ? 5 : 8; }

// A token per warp or CTA: the products with its own row are summed over all of it.  Q rows at
// once: the least of 2, 4, 6 and 8 that takes k, or 8 (65536 x 2 x 1024 bf16: 101 us, 137 with 8), for which three CTAs an
// SM matter more than registers (16384 x 8 x 2048 bf16: 175 us, 226 with two).  In place too: a lane reads what it writes before it does.
template <typename E, int W, int Q, int G>
__global__ void __launch_bounds__(kThreads, Q == 2 ? 4 : 3) join_grad_kernel(Move a) {
  using A = Access<E, W>;
  constexpr int N = A::N, U = grad_pieces<W, Q>();
  __shared__ float red[kWarps][kMaxChoices];
  const int lane = threadIdx.x % 32, tid = threadIdx.x % G, warp = threadIdx.x / 32;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + warp : blockIdx.x;
  if (t >= a.T) return;
  const int pieces = a.d / N, rest = tid < a.d - pieces * N ? pieces * N + tid : -1;
  const E* dy = static_cast<const E*>(a.dy) + t * a.ldy;
  const Places at(a, t);
  const Weights w(a, t);
  for (int j0 = 0; j0 < a.k; j0 += Q) {
    int r[Q];
    float wj[Q], sum[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      r[q] = at[j0 + q];
      wj[q] = w[j0 + q];
      sum[q] = 0.f;
    }
    for (int p = tid; p < pieces; p += G * U) {
      typename A::Raw own[U], v[Q][U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p + u * G < pieces) own[u] = load<A>(dy + (p + u * G) * N);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (r[q] < 0) continue;
        const E* x = static_cast<const E*>(a.x) + r[q] * a.ldx + p * N;
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (p + u * G < pieces) v[q][u] = load<A>(x + u * G * N);
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (r[q] < 0) continue;
        E* out = static_cast<E*>(a.out) + r[q] * a.ldo + p * N;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (p + u * G >= pieces) continue;
          float d[N], f[N];
          A::widen(own[u], d);
          A::widen(v[q][u], f);
#pragma unroll
          for (int i = 0; i < N; ++i) {
            sum[q] = fmaf(d[i], f[i], sum[q]);
            f[i] = wj[q] * d[i];
          }
          store<A>(out + u * G * N, A::narrow(f));
        }
      }
    }
    if (rest >= 0) {
      const float d = Elem<E>::get(dy + rest);
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        if (r[q] < 0) continue;
        sum[q] = fmaf(d, Elem<E>::get(static_cast<const E*>(a.x) + r[q] * a.ldx + rest), sum[q]);
        Elem<E>::put(static_cast<E*>(a.out) + r[q] * a.ldo + rest, wj[q] * d);
      }
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
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
constexpr int64_t kMostWidth = 1 << 30;         // an index of elements that steps beyond a row stays an int
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
  if (tokens < 0 || k < 1 || tokens > INT32_MAX / k || d < 1 || d > kMostWidth || rows < 0 || rows > INT32_MAX) return PGC_EINVAL;
  return (tokens && !place) || (uintptr_t)place % 4 ? PGC_EINVAL : PGC_OK;
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 148;
  return n;
}

// CTAs of a sort: one does up to 2048 slots (2.6 us for 64 on the GPU; 5.3 for 2048, three kernels 6.3; 14.8 for 8000, three kernels 6.3);
// above, each has 1024 at least.  65536 x 8 of 256: 14.8 us, 34.2 where every CTA read all counts itself.
constexpr int kAloneSlots = 2048;
int route_ctas(int64_t n) {
  return n <= kAloneSlots ? 1 : (int)std::min<int64_t>((n + 1023) / 1024, kMostRouteCtas);
}

// The pieces that all rows' starts allow.
int width_of(std::initializer_list<uintptr_t> starts) {
  uintptr_t all = 0;
  for (const uintptr_t p : starts) all |= p;
  return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 2;
}
// A token is a warp's where there are tokens for the SMs' warps, else a CTA's: join 8192 x 4 x 5120 67 us by warps, 74 by CTAs, 65536 x 2 x
// 1024 70 and 208; 1000 x 8 x 2048 13 and 9, its gradient 16 and 13.  Between them it costs: 3000 x 4 x 5120 29.4
// by CTAs, 26.9 by warps.
bool by_warps(const Move& a) { return a.T >= sm_count() * 32; }
unsigned grid_of(const Move& a, bool warps) { return (unsigned)(warps ? (a.T + kWarps - 1) / kWarps : a.T); }

template <typename E, int W>
cudaError_t launch_spread(Move a, cudaStream_t st) {
  const int most = 32 * spread_pieces<W>();
  a.chunks = std::max((a.d / Access<E, W>::N + most - 1) / most, 1);
  spread_kernel<E, W><<<(unsigned)((a.T * a.chunks + kWarps - 1) / kWarps), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}
template <typename E, int W, int G>
auto join_of(int k) { return k <= 2 ? join_kernel<E, W, 2, G> : join_kernel<E, W, 4, G>; }
template <typename E, int W>
cudaError_t launch_join(const Move& a, cudaStream_t st) {
  const bool warps = by_warps(a);
  (warps ? join_of<E, W, 32>(a.k) : join_of<E, W, kThreads>(a.k))<<<grid_of(a, warps), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}
template <typename E, int W, int G>
auto join_grad_of(int k) {
  return k <= 2 ? join_grad_kernel<E, W, 2, G> : k <= 4 ? join_grad_kernel<E, W, 4, G> : k <= 6 ? join_grad_kernel<E, W, 6, G> : join_grad_kernel<E, W, 8, G>;
}
template <typename E, int W>
cudaError_t launch_join_grad(const Move& a, cudaStream_t st) {
  const bool warps = by_warps(a);
  (warps ? join_grad_of<E, W, 32>(a.k) : join_grad_of<E, W, kThreads>(a.k))<<<grid_of(a, warps), kThreads, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_route_workspace(int64_t tokens, int32_t k, int32_t experts, int64_t *bytes) {
  if (!bytes || tokens < 0 || k < 1 || tokens > INT32_MAX / k || experts < 1) return PGC_EINVAL;
  if (experts > kMaxExperts || k > kMaxChoices) return PGC_ENOTSUP;
  const int64_t ctas = route_ctas(tokens * k);
  *bytes = ctas == 1 ? 16 : (ctas + 1) * experts * 4;
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
  const int ctas = route_ctas(n), grain = 32 * kRouteWarps;
  const int64_t per = ((n + ctas - 1) / ctas + grain - 1) / grain * grain;
  const Route a{choice, place, slot, offsets, static_cast<int32_t*>(workspace), (int)n, experts, (int)per};
  const size_t smem = (size_t)kRouteWarps * experts * 4;
  const auto kernel = ctas == 1 ? place_kernel<true> : place_kernel<false>;
  if (smem > kPlainSmem) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRouteWarps * kMaxExperts * 4);
    if (e != cudaSuccess) return report_cuda(e);
  }
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kRouteThreads);
  cfg.stream = st;
  cfg.attrs = &attr;
  if (ctas > 1) {
    count_kernel<<<ctas, kRouteThreads, 0, st>>>(a);
    cudaError_t e = cudaGetLastError();
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(experts + 31) / 32);
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, prefix_kernel, a, ctas);
    if (e != cudaSuccess) return report_cuda(e);
  }
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.dynamicSmemBytes = smem;
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
  if (dtype == PGC_BF16)
    return report_cuda(width == 16 ? launch_spread<__nv_bfloat16, 16>(a, st)
                       : width == 4 ? launch_spread<__nv_bfloat16, 4>(a, st) : launch_spread<__nv_bfloat16, 2>(a, st));
  return report_cuda(width == 16 ? launch_spread<float, 16>(a, st) : launch_spread<float, 4>(a, st));
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
  if (dtype == PGC_BF16)
    return report_cuda(width == 16 ? launch_join<__nv_bfloat16, 16>(a, st)
                       : width == 4 ? launch_join<__nv_bfloat16, 4>(a, st) : launch_join<__nv_bfloat16, 2>(a, st));
  return report_cuda(width == 16 ? launch_join<float, 16>(a, st) : launch_join<float, 4>(a, st));
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
  if (dtype == PGC_BF16)
    return report_cuda(width == 16 ? launch_join_grad<__nv_bfloat16, 16>(a, st)
                       : width == 4 ? launch_join_grad<__nv_bfloat16, 4>(a, st) : launch_join_grad<__nv_bfloat16, 2>(a, st));
  return report_cuda(width == 16 ? launch_join_grad<float, 16>(a, st) : launch_join_grad<float, 4>(a, st));
}

}  // extern "C"
