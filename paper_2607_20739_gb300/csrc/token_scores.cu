// Token scores (pgc_token_scores, pgc_token_scores_grad): the log probability of
// a row's target, the row's entropy and its k likeliest classes, and the
// gradient of the first two.
//
// With q_v = (x_v - m) / tau - L the log probability of class v (m the largest
// logit, L = log sum_v exp((x_v - m) / tau)) and p = exp q:
//   logp = q_y,   H = -sum_v p_v q_v = L - sum_v e_v z_v / sum_v e_v,  z = (x - m) / tau, e = exp z,
//   d logp / d x_v = ([v = y] - p_v) / tau,   d H / d x_v = -p_v (q_v + H) / tau.
// Every term of H is positive, so nothing cancels.
//
// Long rows are bound by memory: one pass makes the sums and finds a bound that the k likeliest classes reach, and
// only the few parts of a row that reach it are read again (4096 x 131072 bf16, k = 20: 189 us, 5.7 TB/s; the pass
// alone 165, without alternatives 158; pushing what may be among the k while the pass runs took 255 to 277).  Short
// rows are bound by their own instructions, few rows by latencies.  The gradient is one pass (2000 x 50001 fp32: 122 us,
// 6.5 TB/s read and written; 115 where a row in eight has no target and is only written).
#include <algorithm>
#include <cmath>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

using Key = unsigned long long;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;            // 16-byte pieces a thread has in flight
constexpr int kMaxCluster = 8;
constexpr int kMostTop = 64;
// Up to as many alternatives of a warp's row come from a bound that sorts the lanes' maxima; more from one that counts those of four
// parts a lane: 65536 x 2000 bf16, k = 16: 113 us, 125 by counts; 1000, k = 20: 87, 83 by sorting; k = 32: 105, 325; 20000 x 8192 fp32: 173, 305.
constexpr int kFewTop = 16;

struct Scores {
  const void* x;
  void* g;
  const int32_t* y;           // NULL: every row takes part, without a target
  int64_t T, ld, ldg;
  int32_t V, k;
  float inv_tau, c;           // 1 / tau, log2(e) / tau
  float *logp, *entropy, *top_logp;
  int32_t* top;
  float2* stats;
};

// ---- sums ------------------------------------------------------------------------
// Exponents are base 2 and relative to M = fl(m c), as in row_slice.cuh, with
// w = sum of 2^z z beside s = sum of 2^z: H = ln 2 (log2 s - w / s) whatever M is.

struct Part {
  float m = -INFINITY, M = -kFar, s = 0.f, w = 0.f;
};
__device__ __forceinline__ void raise(Part& o, float top, float c) {
  if (top > o.m) {
    const float M = ref_of(top, c), d = o.M - M, f = ex2(d);
    o.w = f * fmaf(d, o.s, o.w);
    o.s *= f;
    o.m = top;
    o.M = M;
  }
}
// 2^z z where 2^z has run out: masked classes have z = -inf.
__device__ __forceinline__ float times_log(float e, float z) { return e * fmaxf(z, -1e4f); }
__device__ __forceinline__ void add_one(Part& o, float f, float c) {
  raise(o, f, c);
  const float z = fmaf(f, c, -o.M), e = ex2(z);
  o.s += e;
  o.w += times_log(e, z);
}
// A piece with -inf as -2^100 (NaN stays NaN), so that 2^z z is 0 there and not NaN: one instruction for
// two bf16.  An element below -2^100 adds nothing but with a c below 2^-70, where such a row is summed apart (part_extreme).
template <typename E>
__device__ __forceinline__ uint4 above(uint4 v);
template <>
__device__ __forceinline__ uint4 above<__nv_bfloat16>(uint4 v) {
  auto at_least = [](uint32_t w) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0xf180f180u));
    return r;
  };
  return make_uint4(at_least(v.x), at_least(v.y), at_least(v.z), at_least(v.w));
}
template <>
__device__ __forceinline__ uint4 above<float>(uint4 v) {
  auto at_least = [](uint32_t w) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(__uint_as_float(w)), "f"(-0x1p100f));
    return __float_as_uint(r);
  };
  return make_uint4(at_least(v.x), at_least(v.y), at_least(v.z), at_least(v.w));
}
template <typename E, int U>
__device__ __forceinline__ void add_pieces(Part& o, const uint4 (&v)[U], float c) {
  constexpr int H = Elem<E>::N / 2;
  raise(o, Elem<E>::top(v), c);
  const Pair c2 = pair(c, c), M2 = pair(-o.M, -o.M);
  Pair sum[2] = {0, 0}, log[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < U; ++u) {
    Pair f[H];
    Elem<E>::widen(above<E>(v[u]), f);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      const Pair z = fma2(f[i], c2, M2), e = ex2_2(z);
      sum[i % 2] = add2(sum[i % 2], e);
      log[i % 2] = fma2(e, z, log[i % 2]);
    }
  }
  float lo, hi;
  split(add2(sum[0], sum[1]), lo, hi);
  o.s += lo + hi;
  split(add2(log[0], log[1]), lo, hi);
  o.w += lo + hi;
}
__device__ __forceinline__ Part warp_merge(const Part& o, float c) {
  Part r;
  r.m = warp_max(o.m);
  r.M = ref_of(r.m, c);
  const float d = o.M - r.M, f = ex2(d);
  r.s = warp_sum(o.s * f);
  r.w = warp_sum(f * fmaf(d, o.s, o.w));
  return r;
}
// The same relative to m itself: how CTAs' parts of a row are joined, whatever their M.
__device__ __forceinline__ float3 at_m(const Part& o, float c) {
  const float r = fmaf(o.m, c, -o.M), f = ex2(-r);
  return make_float3(o.m, o.s * f, f * fmaf(-r, o.s, o.w));
}

template <int G>
__device__ __forceinline__ void sync_group() {
  if (G == 32) __syncwarp();
  else __syncthreads();
}

// ---- the k largest ---------------------------------------------------------------
// Every lane knows the largest of its elements, and of up to eight parts of them (4096 x 131072 bf16, k = 20: 190 us,
// 199 with four parts and 207 with sixteen).  The r-th largest of a warp's 32, with r = k over the group's warps, is reached by
// r elements of this warp, the least of the warps' such bounds by k of the row: only what reaches it can be among
// the k largest.  (A bound from the ranks of all 256 maxima is tighter and slower: 241 us.)  The parts that do, a few more than k,
// are read again (from the L2 cache, as a rule), and what reaches the bound there is ranked.  Keys order by value and
// then by the lower class; no two are equal.  Finding parts, reading and ranking them took 12, 10 and 8 us
// when the whole took 195.

__device__ __forceinline__ Key key_of(float f, unsigned v) {
  const uint32_t b = __float_as_uint(f + 0.f);              // zeros of both signs are equal
  return (Key)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - v);
}
__device__ __forceinline__ int class_of(Key q) { return (int)(0xffffffffu - (uint32_t)q); }
__device__ __forceinline__ float value_of(Key q) {
  const uint32_t b = (uint32_t)(q >> 32);
  return __uint_as_float(b ^ (b & 0x80000000u ? 0x80000000u : 0xffffffffu));
}

template <int G>
struct Top {
  static constexpr int kKeys = G * 8 + kMostTop;            // the ones kept and a step of eight each
  static constexpr int kFewKeys = G == 32 ? 160 : 2 * G;     // more are equal ones, as a rule
  static constexpr int kParts = 8;
  Key key[kKeys];
  Key best[kMostTop];                                          // largest first, 0 where there is none
  alignas(16) float most[kParts * G];                       // by parts, then threads
  uint16_t hot[kParts * G];
  Key red[G / 32];
  float warp_bound[G / 32];
  float bound;
  int keys, hots;
};

// The n-th largest of the lanes' values, n = 1 .. 32: they are sorted.
__device__ __forceinline__ float warp_nth(float v, int n) {
  const int lane = threadIdx.x % 32;
#pragma unroll
  for (int size = 2; size <= 32; size *= 2)
#pragma unroll
    for (int o = size / 2; o > 0; o /= 2) {
      const float other = __shfl_xor_sync(0xffffffffu, v, o);
      v = ((lane & o) == 0) == ((lane & size) == 0) ? fmaxf(v, other) : fminf(v, other);
    }
  return __shfl_sync(0xffffffffu, v, n - 1);
}
// The least of the warp's values, 32 times N of them, that are at least the largest number of 16 bits, found bit by bit,
// which k of them reach.  -infinity where fewer than k are above it.
template <int N>
__device__ __forceinline__ float warp_reached(const float (&v)[N], int k) {
  uint32_t key[N], found = 0, least = 0xffffffffu;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t b = __float_as_uint(v[i]);
    key[i] = b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u);
  }
  for (uint32_t bit = 1u << 31; bit >= 1u << 16; bit >>= 1) {
    const uint32_t next = found | bit;
    int n = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) n += __popc(__ballot_sync(0xffffffffu, key[i] >= next));
    if (n < k) continue;
    found = next;
    if (n == k) break;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) least = min(least, key[i] >= found ? key[i] : least);
  least = __reduce_min_sync(0xffffffffu, least);
  return __uint_as_float(least ^ (least & 0x80000000u ? 0x80000000u : 0xffffffffu));
}
template <int G>
__device__ __forceinline__ float least_bound(const Top<G>& sh) {
  float bound = INFINITY;
#pragma unroll
  for (int w = 0; w < G / 32; ++w) bound = fminf(bound, sh.warp_bound[w]);
  return bound;
}

// f(j) for j = 0 .. n - 1, n up to 64: a thread each, or two of a warp.
template <int G, typename F>
__device__ __forceinline__ void for_top(int n, int tid, F f) {
  if (tid < n) f(tid);
  if (G == 32 && tid + 32 < n) f(tid + 32);
}

// The k largest of n keys into sh.best, by all threads of the group: each one's rank, or, of more than two a
// thread of a CTA, one after another.
template <int G>
__device__ __forceinline__ void rank_keys(Top<G>& sh, const Key* keys, int n, int k, int tid) {
  for_top<G>(k, tid, [&](int j) { sh.best[j] = 0; });
  sync_group<G>();
  if (n <= (G == 32 ? Top<G>::kKeys : 2 * G)) {
    for (int i = tid; i < n; i += G) {
      const Key mine = keys[i];
      int rank = 0;
#pragma unroll 4
      for (int j = 0; j < n; ++j) rank += keys[j] > mine;
      if (rank < k) sh.best[rank] = mine;
    }
    sync_group<G>();
    return;
  }
  Key before = ~0ull;
  for (int j = 0; j < k; ++j) {
    Key most = 0;
    for (int i = tid; i < n; i += G) {
      const Key q = keys[i];
      if (q < before && q > most) most = q;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Key q = __shfl_xor_sync(0xffffffffu, most, o);
      most = q > most ? q : most;
    }
    if (G > 32) {
      __syncthreads();
      if (tid % 32 == 0) sh.red[tid / 32] = most;
      __syncthreads();
      for (int i = 0; i < G / 32; ++i) most = sh.red[i] > most ? sh.red[i] : most;
    }
    before = most;
    if (tid == 0) sh.best[j] = most;
    if (most == 0) break;
  }
  sync_group<G>();
}
template <typename E>
__device__ __forceinline__ void each(const uint4& v, float (&f)[8]) {
  Pair h[4];
  Elem<E>::widen(v, h);
#pragma unroll
  for (int i = 0; i < Elem<E>::N / 2; ++i) split(h[i], f[2 * i], f[2 * i + 1]);
}
// A slice's pieces in steps of one a thread, keeping the k largest so far: for rows where more different elements
// reach the bound than there are places (rising ones: 4096 x 131072 bf16, k = 64: 640 us, other rows 213).
template <typename E, int G>
__device__ __noinline__ void top_in_steps(const E* x, Slice s, int tid, int k, Top<G>& sh) {
  constexpr int N = Elem<E>::N;
  const int body = s.first + s.head, rest = body + s.pieces * N;
  Key least = 0;                                             // a key has to be larger
  int n = 0;
  sync_group<G>();
  if (tid == 0) sh.keys = 0;
  sync_group<G>();
  auto push = [&](float f, int v) {
    if (!(f > -INFINITY)) return;
    const Key q = key_of(f, (unsigned)v);
    if (q > least) sh.key[atomicAdd(&sh.keys, 1)] = q;
  };
  for (int i0 = -G; i0 < s.pieces; i0 += G) {
    if (i0 < 0) {
      if (tid < s.head + (s.last - rest)) {
        const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
        push(Elem<E>::get(x + v), v);
      }
    } else if (i0 + tid < s.pieces) {
      float f[8];
      each<E>(load16(reinterpret_cast<const uint4*>(x + body) + i0 + tid), f);
#pragma unroll
      for (int j = 0; j < N; ++j) push(f[j], body + (i0 + tid) * N + j);
    }
    sync_group<G>();
    n = sh.keys;
    if (n > kMostTop) {
      rank_keys<G>(sh, sh.key, n, k, tid);
      n = 0;
      for (int j = 0; j < k; ++j) n += sh.best[j] != 0;
      if (n == k) least = sh.best[k - 1];
      sync_group<G>();
      for_top<G>(n, tid, [&](int j) { sh.key[j] = sh.best[j]; });
      if (tid == 0) sh.keys = n;
    }
    sync_group<G>();
  }
  rank_keys<G>(sh, sh.key, n, k, tid);
}

// The slice read again: the bound is the k-th largest of all the threads' largest elements, and only
// threads that have met it, about k of them, hold alternatives.
template <typename E, int G>
__device__ __noinline__ void top_again(const E* x, Slice s, int tid, int k, float most, Top<G>& sh) {
  constexpr int N = Elem<E>::N;
  sync_group<G>();
  sh.most[tid] = most;
  if (tid == 0) sh.keys = sh.hots = 0;
  sync_group<G>();
  int rank = 0;
#pragma unroll 8
  for (int i = 0; i < G; i += 4) {
    const float4 o = *reinterpret_cast<const float4*>(sh.most + i);
    rank += (o.x > most || (o.x == most && i < tid)) + (o.y > most || (o.y == most && i + 1 < tid)) +
            (o.z > most || (o.z == most && i + 2 < tid)) + (o.w > most || (o.w == most && i + 3 < tid));
  }
  if (rank == k - 1 || (k > G && tid == 0)) sh.bound = k > G ? -INFINITY : most;
  sync_group<G>();
  const float bound = sh.bound;
  auto push = [&](float f, int v) {
    if (!(f >= bound && f > -INFINITY)) return;
    const int at = atomicAdd(&sh.keys, 1);
    if (at < Top<G>::kKeys) sh.key[at] = key_of(f, (unsigned)v);
  };
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (most >= bound && most > -INFINITY) {
    sh.hot[atomicAdd(&sh.hots, 1)] = (uint16_t)tid;
    if (tid < s.head + (s.last - rest)) {
      const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
      push(Elem<E>::get(x + v), v);
    }
  }
  sync_group<G>();
  const unsigned per = (unsigned)(s.pieces + G - 1) / G, items = per * (unsigned)sh.hots;
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  for (unsigned i = tid; i < items; i += G * kUnroll) {
    uint4 v[kUnroll];
    int at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const unsigned item = i + u * G, h = item / per;
      at[u] = item < items ? (int)(sh.hot[h] + (item - h * per) * G) : s.pieces;
      v[u] = at[u] < s.pieces ? load16(p + at[u]) : no_piece(Elem<E>::kLowest);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (at[u] >= s.pieces) continue;
      const uint4 one[1] = {v[u]};
      if (!(Elem<E>::top(one) >= bound)) continue;
      float f[8];
      each<E>(v[u], f);
#pragma unroll
      for (int j = 0; j < N; ++j) push(f[j], body + at[u] * N + j);
    }
  }
  sync_group<G>();
  const int n = sh.keys;
  if (n <= Top<G>::kKeys) rank_keys<G>(sh, sh.key, n, k, tid);
  else top_in_steps<E, G>(x, s, tid, k, sh);
}

// Groups of pieces in a part.
template <int G>
__device__ __forceinline__ int groups_of_part(const Slice& s) {
  return ((s.pieces + G * kUnroll - 1) / (G * kUnroll) + Top<G>::kParts - 1) / Top<G>::kParts;
}
// A warp's row whose pieces stay in registers until their bound is known.
template <int G>
__device__ __forceinline__ bool at_once(const Slice& s) { return G == 32 && s.pieces > 0 && s.pieces <= G * kUnroll; }
template <int G>
__device__ __forceinline__ void push(float f, int v, float bound, Top<G>& sh) {
  if (!(f >= bound)) return;
  const int at = atomicAdd(&sh.keys, 1);
  if (at < Top<G>::kKeys) sh.key[at] = key_of(f, (unsigned)v);
}
template <typename E, int G>
__device__ __forceinline__ void push_piece(const uint4& piece, int first, float bound, Top<G>& sh) {
  float f[8];
  each<E>(piece, f);
#pragma unroll
  for (int j = 0; j < Elem<E>::N; ++j) push(f[j], first + j, bound, sh);
}
// Which of the elements of kUnroll pieces reach the bound, a bit each, and where a bit's element is.  (A bf16 pair is
// compared at once; the bound is a bf16 number there.)
template <typename E>
struct Reach;
template <>
struct Reach<float> {
  __device__ __forceinline__ static uint32_t bits(const uint4 (&v)[kUnroll], float bound) {
    uint32_t r = 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) r |= __uint_as_float(w[j]) >= bound ? 1u << (4 * u + j) : 0u;
    }
    return r;
  }
  __device__ __forceinline__ static int piece(int bit) { return bit / 4; }
  __device__ __forceinline__ static int element(int bit) { return bit % 4; }
};
template <>
struct Reach<__nv_bfloat16> {
  __device__ __forceinline__ static uint32_t bits(const uint4 (&v)[kUnroll], float bound) {
    const __nv_bfloat162 b = __float2bfloat162_rn(bound);
    uint32_t r = 0;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) r |= __hge2_mask(*reinterpret_cast<const __nv_bfloat162*>(&w[j]), b) & 0x00010001u << (4 * u + j);
    }
    return r;
  }
  __device__ __forceinline__ static int piece(int bit) { return bit % 16 / 4; }
  __device__ __forceinline__ static int element(int bit) { return bit % 4 * 2 + bit / 16; }
};
// Those elements' keys, read again one by one, as they are few; first(u): the class that piece u starts with.
template <typename E, int G, typename F>
__device__ __forceinline__ void push_pieces(const E* x, const uint4 (&v)[kUnroll], float bound, Top<G>& sh, F first) {
  uint32_t bits = Reach<E>::bits(v, bound);
  if (!bits) return;
  int at = atomicAdd(&sh.keys, __popc(bits));
  for (; bits && at < Top<G>::kKeys; bits &= bits - 1, ++at) {
    const int bit = __ffs(bits) - 1, c = first(Reach<E>::piece(bit)) + Reach<E>::element(bit);
    sh.key[at] = key_of(Elem<E>::get(x + c), (unsigned)c);
  }
}

// Where most parts reach the bound, by elements that are equal, as a rule: classes masked by a number, fewer than k
// others left.  What lies above the bound is taken from the whole slice, and what is missing to k from the
// lowest classes that have met it (4096 x 131072 bf16, 10 classes left, k = 20: 308 us, 1205 in steps; others 189).
template <typename E, int G>
__device__ __noinline__ void top_of_ties(const E* x, Slice s, int tid, int k, float bound, Top<G>& sh) {
  constexpr int N = Elem<E>::N;
  const int body = s.first + s.head, rest = body + s.pieces * N;
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  sync_group<G>();
  if (tid == 0) sh.keys = 0;
  sync_group<G>();
  auto put = [&](bool take, float f, int v) {
    if (!take) return;
    const int at = atomicAdd(&sh.keys, 1);
    if (at < Top<G>::kKeys) sh.key[at] = key_of(f, (unsigned)v);
  };
  const int edge = tid < s.head ? s.first + tid : rest + tid - s.head;       // an element beside the pieces
  const bool has_edge = tid < s.head + (s.last - rest);
  const float at_edge = has_edge ? Elem<E>::get(x + edge) : -INFINITY;
  put(at_edge > bound, at_edge, edge);
  for (int i0 = tid; i0 < s.pieces; i0 += G * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = i0 + u * G < s.pieces ? load16(p + i0 + u * G) : no_piece(Elem<E>::kLowest);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint4 one[1] = {v[u]};
      if (!(Elem<E>::top(one) > bound)) continue;
      float f[8];
      each<E>(v[u], f);
#pragma unroll
      for (int j = 0; j < N; ++j) put(f[j] > bound, f[j], body + (i0 + u * G) * N + j);
    }
  }
  sync_group<G>();
  const int above = sh.keys;
  int n = above;
  if (n > Top<G>::kKeys) {
    top_in_steps<E, G>(x, s, tid, k, sh);
    return;
  }
  // elements of consecutive classes, thread after thread
  auto append = [&](const float (&f)[8], int first) {
    int mine = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) mine += f[j] == bound;
    int up = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int q = __shfl_up_sync(0xffffffffu, up, o);
      if (tid % 32 >= o) up += q;
    }
    if (tid % 32 == 31) sh.red[tid / 32] = up;
    sync_group<G>();
    int at = n + up - mine;
    for (int w = 0; w < G / 32; ++w) {
      at += w < tid / 32 ? (int)sh.red[w] : 0;
      n += (int)sh.red[w];
    }
    sync_group<G>();
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (f[j] == bound) {
        if (at < k) sh.key[at] = key_of(f[j], (unsigned)(first + j));
        ++at;
      }
  };
  auto one = [&](bool has, float f, int v) {
    float all[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) all[j] = j || !has ? NAN : f;
    append(all, v);
  };
  sync_group<G>();
  if (n < k) one(tid < s.head, at_edge, edge);
  for (int i0 = 0; i0 < s.pieces && n < k; i0 += G) {
    float f[8];
    each<E>(i0 + tid < s.pieces ? load16(p + i0 + tid) : no_piece(Elem<E>::kLowest), f);
    append(f, body + (i0 + tid) * N);
  }
  if (n < k) one(tid >= s.head && has_edge, at_edge, edge);
  sync_group<G>();
  rank_keys<G>(sh, sh.key, above < k ? min(n, k) : above, k, tid);
}

// A slice's sums in one pass, its parts' largest elements and the warps' bounds.
// kMany: more alternatives than a warp has lanes.
template <typename E, int G, bool kMany>
__device__ __forceinline__ Part scan(const E* x, const Slice& s, int tid, float c, int k, Top<G>& sh) {
  constexpr int N = Elem<E>::N;
  Part o;
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (tid < s.head + (s.last - rest)) add_one(o, Elem<E>::get(x + (tid < s.head ? s.first + tid : rest + tid - s.head)), c);
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  const int groups = groups_of_part<G>(s);
  float most = -INFINITY, each_most[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) each_most[u] = -INFINITY;
  uint4 v[kUnroll];
  for (int i0 = 0, part = 0, left = groups; i0 < s.pieces; i0 += G * kUnroll) {
    const int i = i0 + tid;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) v[u] = i + u * G < s.pieces ? load16(p + i + u * G) : no_piece(Elem<E>::kLowest);
    add_pieces<E>(o, v, c);
    if (kMany) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint4 one[1] = {v[u]};
        each_most[u] = fmaxf(each_most[u], Elem<E>::top(one));
      }
    }
    if (!k || at_once<G>(s)) continue;
    most = fmaxf(most, Elem<E>::top(v));
    if (--left == 0 || i0 + G * kUnroll >= s.pieces) {
      sh.most[part++ * G + tid] = most;
      most = -INFINITY;
      left = groups;
    }
  }
  if (k) {
    const float bound = kMany ? warp_reached(each_most, k) : warp_nth(o.m, (k + G / 32 - 1) / (G / 32));
    if (tid % 32 == 0) sh.warp_bound[tid / 32] = bound;
    if (tid == 0) sh.keys = sh.hots = 0;
    if (G == 32) __syncwarp();
    if (at_once<G>(s) && bound > -INFINITY) {
      push_pieces<E, G>(x, v, bound, sh, [&](int u) { return body + (tid + u * G) * N; });
    }
  }
  return o;
}
// The k largest, after scan and a barrier behind it.
template <typename E, int G>
__device__ __forceinline__ void scan_top(const E* x, const Slice& s, int tid, int k, const Part& o, Top<G>& sh) {
  constexpr int N = Elem<E>::N;
  const float bound = least_bound(sh);
  if (bound == -INFINITY) {
    top_again<E, G>(x, s, tid, k, o.m, sh);
    return;
  }
  const int body = s.first + s.head, rest = body + s.pieces * N, groups = groups_of_part<G>(s);
  const int parts = s.pieces && !at_once<G>(s) ? ((s.pieces + G * kUnroll - 1) / (G * kUnroll) + groups - 1) / groups : 0;
  if (o.m >= bound) {
    for (int q = 0; q < parts; ++q)
      if (sh.most[q * G + tid] >= bound) sh.hot[atomicAdd(&sh.hots, 1)] = (uint16_t)(q * G + tid);
    if (tid < s.head + (s.last - rest)) {
      const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
      push(Elem<E>::get(x + v), v, bound, sh);
    }
  }
  sync_group<G>();
  // (A warp's row of one part or two never has so many for k from 32 on, one in registers for any k: equal elements show there
  // only when their keys are too many.  65536 x 2000 bf16, k = 40: 176 us, 603 with 10 classes left and the others at the lowest number;
  // 600, k = 20: 84, 174.)
  if (sh.hots > max(parts * G / 2, 2 * k)) {
    top_of_ties<E, G>(x, s, tid, k, bound, sh);
    return;
  }
  const unsigned per = groups * kUnroll, items = per * (unsigned)sh.hots;
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  for (unsigned i = tid; i < items; i += G * kUnroll) {
    uint4 v[kUnroll];
    int at[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const unsigned item = i + u * G, h = item / per;
      at[u] = s.pieces;
      if (item < items) at[u] = (int)((sh.hot[h] / G * per + (item - h * per)) * G + sh.hot[h] % G);
      if (at[u] < s.pieces) v[u] = load16(p + at[u]);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (at[u] >= s.pieces) continue;
      const uint4 one[1] = {v[u]};
      if (Elem<E>::top(one) >= bound) push_piece<E, G>(v[u], body + at[u] * N, bound, sh);
    }
  }
  sync_group<G>();
  const int n = sh.keys;
  if (n <= Top<G>::kFewKeys) rank_keys<G>(sh, sh.key, n, k, tid);
  else top_of_ties<E, G>(x, s, tid, k, bound, sh);
}

// ---- a row -------------------------------------------------------------------------

__device__ __forceinline__ int cluster_ranks() {
  int n;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
__device__ __forceinline__ int cluster_rank() {
  int n;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(n));
  return n;
}

template <int G>
struct Shared {
  Top<G> top;
  float4 part[G / 32];
};
// What the CTAs of a cluster hand to its first one.
struct Gathered {
  float3 part[kMaxCluster];
  Key key[kMaxCluster * kMostTop];
};

// s and w of a slice whose exponents leave the range of the fast path, relative to its m.
template <typename E, int G>
__device__ __noinline__ float3 part_extreme(const E* x, Slice s, int tid, float m, float c, float4* red) {
  float sum = 0.f, log = 0.f;
  for (unsigned v = s.first + tid; v < (unsigned)s.last; v += G) {
    const float f = Elem<E>::get(x + v), z = f == -INFINITY ? f : (f - m) * c, e = exp2f(z);
    sum += e;
    log += times_log(e, z);
  }
  sum = warp_sum(sum);
  log = warp_sum(log);
  if (G > 32) {
    __syncthreads();
    if (tid % 32 == 0) red[tid / 32] = make_float4(0.f, 0.f, sum, log);
    __syncthreads();
    sum = log = 0.f;
    for (int i = 0; i < G / 32; ++i) {
      sum += red[i].z;
      log += red[i].w;
    }
  }
  return make_float3(m, sum, log);
}

template <typename E, int G, bool kMany>
__device__ __forceinline__ float3 row_part(const E* x, const Slice& s, int tid, const Scores& a, Part& o, Shared<G>& sh) {
  float4* red = sh.part;
  o = scan<E, G, kMany>(x, s, tid, a.c, a.k, sh.top);
  Part q = warp_merge(o, a.c);
  if (G == 32) __syncwarp();
  if (G > 32) {
    const int lane = tid % 32;
    if (lane == 0) red[tid / 32] = make_float4(q.m, q.M, q.s, q.w);
    __syncthreads();
    q = Part();
    if (lane < G / 32) {
      const float4 r = red[lane];
      q.m = r.x; q.M = r.y; q.s = r.z; q.w = r.w;
    }
    q = warp_merge(q, a.c);
  }
  // so small a c that an element below -2^100 may count, or so large that x c overflowed
  const bool slow = is_extreme(q.m, a.c) || a.c < 0x1p-70f || (isnan(q.w) && !isnan(q.s));
  return slow ? part_extreme<E, G>(x, s, tid, q.m, a.c, red) : at_m(q, a.c);
}

// m, L and H of a row from the sums relative to m.
__device__ __forceinline__ float3 finish(const float3& q) {
  if (q.x == -INFINITY) return make_float3(q.x, NAN, NAN);
  return make_float3(q.x, logf(q.y), logf(q.y) - kLn2 * (q.z / q.y));
}
// Row t's results, by lane `tid` of the threads that have them all.
template <int G>
__device__ __forceinline__ void write_row(const Scores& a, int64_t t, float3 r, float xy, const Key* best, int tid) {
  for_top<G>(a.k, tid, [&](int j) {
    const Key q = best[j];
    a.top[t * a.k + j] = q ? class_of(q) : -1;
    a.top_logp[t * a.k + j] = q ? (value_of(q) - r.x) * a.inv_tau - r.y : -INFINITY;
  });
  if (tid) return;
  if (a.logp) a.logp[t] = (xy - r.x) * a.inv_tau - r.y;
  a.entropy[t] = r.z;
  a.stats[t] = make_float2(r.x, r.y);
}
template <int G>
__device__ __forceinline__ void write_none(const Scores& a, int64_t t, int tid) {
  for_top<G>(a.k, tid, [&](int j) {
    a.top[t * a.k + j] = -1;
    a.top_logp[t * a.k + j] = -INFINITY;
  });
  if (tid) return;
  if (a.logp) a.logp[t] = 0.f;
  a.entropy[t] = 0.f;
  a.stats[t] = make_float2(0.f, 0.f);
}

// A row per warp (G = 32), CTA or cluster of CTAs.  Five CTAs an SM (16384 x 32768 bf16, k = 5: 194 us; 198 with four, 267 with six);
// warps in fp32 four (20000 x 8192, k = 20: 148, 160 with five).
template <typename E, int G, bool kMany>
__global__ void __launch_bounds__(kThreads, G == 32 && sizeof(E) == 4 ? 4 : 5) scores_kernel(Scores a) {
  extern __shared__ __align__(16) unsigned char raw[];
  Shared<G>& sh = reinterpret_cast<Shared<G>*>(raw)[G == 32 ? threadIdx.x / 32 : 0];
  const int rank = G == 32 ? 0 : cluster_rank(), ranks = G == 32 ? 1 : cluster_ranks();
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x / ranks;
  if (t >= a.T) return;
  const int32_t y = a.y ? a.y[t] : 0;
  if (y < 0) {
    if (rank == 0) write_none<G>(a, t, tid);
    return;
  }
  // a CTA's shared memory may be written by another one of its cluster only once it runs
  if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  const float xy = a.y && y < a.V ? Elem<E>::get(x + y) : NAN;
  const Slice s = slice_of(x, a.V, rank, ranks);
  Part mine;
  float3 q = row_part<E, G, kMany>(x, s, tid, a, mine, sh);
  if (a.k) scan_top<E, G>(x, s, tid, a.k, mine, sh.top);
  if (ranks == 1) {
    write_row<G>(a, t, finish(q), xy, sh.top.best, tid);
    return;
  }
  Gathered& all = *reinterpret_cast<Gathered*>(raw + (sizeof(Shared<G>) + 15) / 16 * 16);
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  auto first = [](const void* p) {                           // the same place in the cluster's first CTA
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(smem_u32(p)));
    return at;
  };
  if (tid == 0) {
    const uint32_t at = first(&all.part[rank]);
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(q.x) : "memory");
    asm volatile("st.shared::cluster.f32 [%0 + 4], %1;" ::"r"(at), "f"(q.y) : "memory");
    asm volatile("st.shared::cluster.f32 [%0 + 8], %1;" ::"r"(at), "f"(q.z) : "memory");
  }
  if (tid < a.k)
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(first(&all.key[rank * a.k + tid])), "l"(sh.top.best[tid]) : "memory");
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank) return;
  // parts relative to their own m: 2^((m_i - m) c) each
  float m = -INFINITY, sum = 0.f, log = 0.f;
  for (int i = 0; i < ranks; ++i) m = fmaxf(m, all.part[i].x);
  for (int i = 0; i < ranks; ++i) {
    const float3 p = all.part[i];
    const float d = p.x == m ? 0.f : fmaxf((p.x - m) * a.c, -1e4f), f = ex2(d);
    sum += p.y * f;
    log += f * fmaf(d, p.y, p.z);
  }
  if (a.k) {
    for (int i = tid; i < ranks * a.k; i += G) sh.top.key[i] = all.key[i];
    __syncthreads();
    rank_keys<G>(sh.top, sh.top.key, ranks * a.k, a.k, tid);
  }
  write_row<G>(a, t, finish(make_float3(m, sum, log)), xy, sh.top.best, tid);
}

// ---- short rows --------------------------------------------------------------------
// Rows of up to L R classes in the registers of L lanes, so that a warp has 32 / L rows at once:
// what a row costs there is its own instructions and one load's latency, not its bytes (131072 x 100 bf16, which are 3.9 us of
// memory: 12.0 us from a graph, 28 with k = 5, 43 with k = 20, 2.6 to 3.1 instructions a cycle and SM of 4; by calls, which the host
// makes in 20 us, in pieces 66 and, with k = 20, 393).  Elements are single ones, or (P = 2: bf16
// rows of even length and pitch that start on 4 bytes) two neighbours.
template <int L, int P>
__device__ __forceinline__ int short_at(int l, int j) { return P * (l + j / P * L) + j % P; }
template <typename E, int L, int R, int P>
__device__ __forceinline__ void short_load(const E* x, int l, int V, bool taken, float (&v)[R]) {
#pragma unroll
  for (int j = 0; j < R; j += P) {
    const int e = short_at<L, P>(l, j);
    if constexpr (P == 2) {
      const uint32_t w = taken && e < V ? *reinterpret_cast<const uint32_t*>(x + e) : Elem<E>::kLowest;
      v[j] = __uint_as_float(w << 16);
      v[j + 1] = __uint_as_float(w & 0xffff0000u);
    } else {
      v[j] = taken && e < V ? Elem<E>::get(x + e) : -INFINITY;
    }
  }
}
template <int L>
__device__ __forceinline__ float group_add(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Keys of a short row: 32 bits for bf16 logits, whose classes are below 2^16.  0: no alternative.
template <typename E>
struct ShortKey {
  using T = Key;
  __device__ __forceinline__ static T of(float f, int v) { return f > -INFINITY ? key_of(f, (unsigned)v) : 0; }
  __device__ __forceinline__ static int at(T q) { return class_of(q); }
  __device__ __forceinline__ static float value(T q) { return value_of(q); }
};
template <>
struct ShortKey<__nv_bfloat16> {
  using T = uint32_t;
  __device__ __forceinline__ static T of(float f, int v) {
    const uint32_t b = __float_as_uint(f + 0.f);
    return f > -INFINITY ? ((b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) & 0xffff0000u) | (0xffffu - v) : 0;
  }
  __device__ __forceinline__ static int at(T q) { return (int)(0xffffu - (q & 0xffffu)); }
  __device__ __forceinline__ static float value(T q) {
    return __uint_as_float((q ^ (q & 0x80000000u ? 0x80000000u : 0xffffffffu)) & 0xffff0000u);
  }
};
// Odd-even merge sort (Batcher) of a power of two of keys, largest first.
template <typename T, int R>
__device__ __forceinline__ void sort_down(T (&q)[R]) {
#pragma unroll
  for (int p = 1; p < R; p *= 2)
#pragma unroll
    for (int d = p; d >= 1; d /= 2)
#pragma unroll
      for (int i = 0; i + d < R; ++i)
        if (i >= d % p && (i - d % p) % (2 * d) < d && i / (2 * p) == (i + d) / (2 * p)) {
          const T one = q[i], two = q[i + d];
          q[i] = one > two ? one : two;
          q[i + d] = one > two ? two : one;
        }
}
template <typename E, int L, int R, int P>
__global__ void __launch_bounds__(kThreads) short_scores_kernel(Scores a) {
  const int lane = threadIdx.x % 32, l = lane % L;
  const int64_t t = (blockIdx.x * (int64_t)kWarps + threadIdx.x / 32) * (32 / L) + lane / L;
  const int32_t y = t < a.T ? a.y ? a.y[t] : 0 : -1;
  const bool taken = y >= 0;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  float v[R];
  short_load<E, L, R, P>(x, l, a.V, taken, v);
  const float xy = taken && a.y && y < a.V ? Elem<E>::get(x + y) : NAN;
  float m = v[0];
#pragma unroll
  for (int j = 1; j < R; ++j) m = fmaxf(m, v[j]);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float sum = 0.f, log = 0.f;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const float z = (v[j] - m) * a.c, e = ex2(z);
    sum += e;
    log += times_log(e, z);
  }
  sum = group_add<L>(sum);
  log = group_add<L>(log);
  const float3 r = taken ? finish(make_float3(m, sum, log)) : make_float3(0.f, 0.f, 0.f);
  if (l == 0 && t < a.T) {
    if (a.logp) a.logp[t] = taken ? (xy - r.x) * a.inv_tau - r.y : 0.f;
    a.entropy[t] = r.z;
    a.stats[t] = make_float2(r.x, r.y);
  }
  if (!a.k) return;
  // A lane's keys, sorted, lie in its column of shared memory; the group's largest head is taken k times, and L of
  // them are written at once.
  using Short = typename ShortKey<E>::T;
  __shared__ Short list[R * kThreads];
  Short key[R];
#pragma unroll
  for (int j = 0; j < R; ++j) key[j] = ShortKey<E>::of(v[j], short_at<L, P>(l, j));
  sort_down(key);
#pragma unroll
  for (int j = 1; j < R; ++j) list[j * kThreads + threadIdx.x] = key[j];
  Short head = key[0], kept = 0;
  int next = 1;
  for (int i = 0; i < a.k; ++i) {
    Short best = head;
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) {
      const Short other = __shfl_xor_sync(0xffffffffu, best, o);
      best = other > best ? other : best;
    }
    if (best != 0 && head == best) {
      head = next < R ? list[next * kThreads + threadIdx.x] : 0;
      ++next;
    }
    if (l == i % L) kept = best;
    const int first = i / L * L;
    if ((i % L == L - 1 || i == a.k - 1) && t < a.T && first + l <= i) {
      a.top[t * a.k + first + l] = kept ? ShortKey<E>::at(kept) : -1;
      a.top_logp[t * a.k + first + l] = kept ? (ShortKey<E>::value(kept) - r.x) * a.inv_tau - r.y : -INFINITY;
    }
  }
}

// ---- gradient ----------------------------------------------------------------------

// -p (a + b (q + H)) / tau is 2^z (at0 + at_z z) with z = x c - M, as q is linear in z.
struct Slope {
  float m, M, c, at0, at_z, at_y;
  int y;
  bool extreme;
  float L, H, a, b, inv_tau;          // extreme rows
};
__device__ __forceinline__ Slope slope_of(float2 st, float H, float a, float b, float inv_tau, float c, int y) {
  Slope r;
  r.m = st.x; r.c = c; r.y = y;
  r.M = ref_of(st.x, c);
  r.extreme = is_extreme(st.x, c);
  r.L = st.y; r.H = H; r.a = a; r.b = b; r.inv_tau = inv_tau;
  const float l2 = fmaf(st.x, c, -r.M) + st.y * kLog2e;       // log2 of the sum at M
  const float scale = -inv_tau * exp2f(-l2);
  r.at0 = scale * fmaf(b, fmaf(-kLn2, l2, H), a);
  r.at_z = scale * b * kLn2;
  r.at_y = a * inv_tau;
  return r;
}
__device__ __forceinline__ float slope_at(float x, bool target, const Slope& r) {
  if (r.extreme) {
    const float q = (x - r.m) * r.inv_tau - r.L;
    return (-expf(q) * fmaf(r.b, fmaxf(q + r.H, -1e4f), r.a) + (target ? r.a : 0.f)) * r.inv_tau;
  }
  const float z = fmaxf(fmaf(x, r.c, -r.M), -1e4f);
  return fmaf(ex2(z), fmaf(z, r.at_z, r.at0), target ? r.at_y : 0.f);
}
template <typename E>
__device__ __forceinline__ void slope_piece(const uint4& v, E* out, bool wide, const Slope& r) {
  constexpr int N = Elem<E>::N;
  Pair f[N / 2];
  Elem<E>::widen(v, f);
  const Pair c2 = pair(r.c, r.c), M2 = pair(-r.M, -r.M), k0 = pair(r.at0, r.at0), kz = pair(r.at_z, r.at_z);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    float lo, hi;
    split(fma2(f[i], c2, M2), lo, hi);
    const Pair z = pair(fmaxf(lo, -1e4f), fmaxf(hi, -1e4f));
    f[i] = mul2(ex2_2(z), fma2(z, kz, k0));
  }
  if (wide) {
    store16(reinterpret_cast<uint4*>(out), Elem<E>::narrow(f));
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      float lo, hi;
      split(f[i], lo, hi);
      Elem<E>::put(out + 2 * i, lo);
      Elem<E>::put(out + 2 * i + 1, hi);
    }
  }
}

// What a row's derivatives ask for: zeros where they are 0, NaN where there is no gradient, or a slope.
struct RowSlope {
  bool filled;
  float fill;
  Slope r;
};
__device__ __forceinline__ RowSlope row_slope(const Scores& a, int64_t t, int32_t y, const float* dlogp, const float* dentropy) {
  const float da = dlogp && y >= 0 ? dlogp[t] : 0.f, db = dentropy && y >= 0 ? dentropy[t] : 0.f;
  const float2 st = a.stats[t];
  const float H = db != 0.f ? a.entropy[t] : 0.f;
  const bool none = da == 0.f && db == 0.f;
  RowSlope q;
  q.filled = none || isnan(da) || isnan(db) || isnan(st.y) || isnan(H) || (da != 0.f && y >= a.V);
  q.fill = none ? 0.f : NAN;
  q.r = slope_of(st, H, da, db, a.inv_tau, a.c, da != 0.f ? y : -1);
  return q;
}

// A row, or one of its `parts`, per group: nothing is exchanged between them.  In place too: a thread
// reads what it writes before it does, and the target's logit, which the thread of its piece writes again.
template <typename E, int G>
__global__ void __launch_bounds__(kThreads) scores_grad_kernel(Scores a, int parts, const float* dlogp, const float* dentropy) {
  constexpr int N = Elem<E>::N;
  const int rank = G == 32 ? 0 : blockIdx.x % parts, ranks = G == 32 ? 1 : parts;
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x / parts;
  if (t >= a.T) return;
  const int32_t y = a.y ? a.y[t] : 0;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const Slice s = slice_of(x, a.V, rank, ranks);
  const RowSlope row = row_slope(a, t, y, dlogp, dentropy);
  if (row.filled) {
    slice_fill<E, G>(g, s.first, s.last, tid, row.fill);
    return;
  }
  const Slope& r = row.r;
  const int target = r.y;
  const float xy = target >= 0 ? Elem<E>::get(x + target) : 0.f;
  if (r.extreme) {
    for (unsigned v = s.first + tid; v < (unsigned)s.last; v += G)
      Elem<E>::put(g + v, slope_at(Elem<E>::get(x + v), (int)v == target, r));
    return;
  }
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (tid < s.head + (s.last - rest)) {
    const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
    Elem<E>::put(g + v, slope_at(Elem<E>::get(x + v), v == target, r));
  }
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  for (int i = tid; i < s.pieces; i += G * kUnroll) {
    uint4 v[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i + u * G < s.pieces) v[u] = load16(p + i + u * G);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i + u * G < s.pieces) slope_piece<E>(v[u], g + body + (i + u * G) * N, wide, r);
  }
  const int at = target - body;
  if (target >= 0 && at >= 0 && at < s.pieces * N && at / N % G == tid) Elem<E>::put(g + target, slope_at(xy, true, r));
}

// Short rows: 131072 x 100 bf16 18.6 us from a graph (memory 7.8; the log probability's alone 14.2), 65536 x 512 39 (20; 27): 2.5 to 2.7
// instructions a cycle and SM of 4, compares and selects of every element's extreme case and target among them.
template <typename E, int L, int R, int P>
__global__ void __launch_bounds__(kThreads) short_scores_grad_kernel(Scores a, const float* dlogp, const float* dentropy) {
  const int lane = threadIdx.x % 32, l = lane % L;
  const int64_t t = (blockIdx.x * (int64_t)kWarps + threadIdx.x / 32) * (32 / L) + lane / L;
  if (t >= a.T) return;
  const int32_t y = a.y ? a.y[t] : 0;
  const RowSlope row = row_slope(a, t, y, dlogp, dentropy);
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  float v[R];
  short_load<E, L, R, P>(static_cast<const E*>(a.x) + t * a.ld, l, a.V, !row.filled, v);
  const bool words = reinterpret_cast<uintptr_t>(g) % 4 == 0;
#pragma unroll
  for (int j = 0; j < R; j += P) {
    const int e = short_at<L, P>(l, j);
    if (e >= a.V) continue;
    float d[P];
#pragma unroll
    for (int i = 0; i < P; ++i) d[i] = row.filled ? row.fill : slope_at(v[j + i], e + i == row.r.y, row.r);
    if constexpr (P == 2) {
      if (words) {
        *reinterpret_cast<uint32_t*>(g + e) = Elem<E>::two(pair(d[0], d[1]));
        continue;
      }
    }
#pragma unroll
    for (int i = 0; i < P; ++i) Elem<E>::put(g + e + i, d[i]);
  }
}

// ---- host --------------------------------------------------------------------

int check(const pgc_logits* z, bool grad) {
  if (!z) return PGC_EINVAL;
  if (z->dtype != PGC_F32 && z->dtype != PGC_BF16) return PGC_EINVAL;
  if (z->rows < 0 || z->rows > INT32_MAX || z->classes < 1 || z->classes > INT32_MAX) return PGC_EINVAL;
  if (!(z->temperature > 0.f) || !std::isfinite(z->temperature) || !std::isfinite(1.f / z->temperature * kLog2e)) return PGC_EINVAL;
  const uintptr_t size = z->dtype == PGC_BF16 ? 2 : 4;
  const int64_t far = int64_t(1) << 31;
  if (z->ld < z->classes || z->ld > far || (z->rows && !z->x)) return PGC_EINVAL;
  if ((uintptr_t)z->x % size || (uintptr_t)z->target % 4) return PGC_EINVAL;
  if (!grad) return PGC_OK;
  if (z->grad_ld < z->classes || z->grad_ld > far || (z->rows && !z->grad)) return PGC_EINVAL;
  if ((uintptr_t)z->grad % size || (z->grad == z->x && z->grad_ld != z->ld)) return PGC_EINVAL;
  return PGC_OK;
}
Scores scores_of(const pgc_logits* z) {
  Scores a{};
  a.x = z->x; a.g = z->grad; a.y = z->target; a.T = z->rows; a.ld = z->ld; a.ldg = z->grad_ld;
  a.V = (int32_t)z->classes;
  a.inv_tau = 1.f / z->temperature;
  a.c = a.inv_tau * kLog2e;
  return a;
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 148;
  return n;
}

// A warp takes a row of up to 4 KB; where there are rows for all warps, up to 24 KB (36621 x 8192 bf16: 101 us, 163 by CTAs; the
// gradient's 183, 206; up to 72 KB no gain: 16384 x 32768 bf16 171 and 173, gradient 313 and 336), and with alternatives, whose
// barriers a CTA waits at, up to 72 KB (20000 x 32768, k = 5: 239 us, 284 by CTAs; fp32 of 8192, k = 20: 149, 209) or, above
// 12 of them, 48 KB (20000 x 24000, k = 32: 261, 284; 32768, k = 32: 349, 318).  Few long rows are split over a
// cluster while the SMs hold more CTAs and a part stays above 4 KB (one row of 131072, k = 20: 9.0 us on the
// GPU, 13.1 by one CTA).  Where these bounds cost: 8192 x 32768 fp32, k = 5: 193 us by CTAs, 183 by warps; 64 x 32768, k = 20: 8.4 us by clusters, 7.9
// by CTAs.
constexpr int64_t kWarpRowBytes = 4 * 1024, kWarpManyRowsBytes = 24 * 1024, kWarpFewTopBytes = 72 * 1024, kWarpTopBytes = 48 * 1024;
constexpr int kWarpFewTop = 12;
struct Shape {
  bool warp;
  int ranks;
  unsigned grid;
};
Shape shape_of(const pgc_logits* z, int k) {
  const int64_t bytes = z->classes * (z->dtype == PGC_BF16 ? 2 : 4), sms = sm_count();
  const int64_t many = k == 0 ? kWarpManyRowsBytes : k <= kWarpFewTop ? kWarpFewTopBytes : kWarpTopBytes;
  Shape s{bytes <= kWarpRowBytes || (bytes <= many && z->rows >= 32 * sms), 1, 0};
  if (s.warp) {
    s.grid = (unsigned)((z->rows + kWarps - 1) / kWarps);
    return s;
  }
  while (s.ranks < kMaxCluster && z->rows * s.ranks * 2 <= 2 * sms && bytes / (s.ranks * 2) >= kWarpRowBytes) s.ranks *= 2;
  s.grid = (unsigned)(z->rows * s.ranks);
  return s;
}

// Rows of bf16 whose elements can be taken in pairs, and rows that are held in registers: up to 128
// classes by 8 lanes, 256 by 16, 512 by 32.  Their limit, with both sides in us for 65536 rows (registers, then pieces):
// 512 bf16, k = 5: 58, 60; k = 12: 74, 65; k = 20: 91, 85; k = 64: 183, 717; 301 bf16, one by one, k = 12: 72, 69; k = 20: 89, 95;
// 256 bf16, k = 12: 38, 64; 256 fp32, k = 5: 56, 56; k = 12: 70, 62; k = 20: 85, 81; k = 64: 165, 441; 130 fp32, k = 12: 68, 66; k = 20: 83, 87;
// 100 fp32, k = 12: 36, 56; 512 fp32, whose keys have 64 bits, k = 5: 109, 60; k = 64: 347, 160.  Without alternatives as in the losses.
bool in_pairs(const pgc_logits* z) { return z->classes % 2 == 0 && z->ld % 2 == 0 && (uintptr_t)z->x % 4 == 0; }
bool short_rows(const pgc_logits* z, int k) {
  const bool wide = z->dtype == PGC_F32;
  if (!k) return z->classes <= (wide || in_pairs(z) ? 512 : 256);
  return z->classes <= (wide ? 256 : 512) / (k > 8 && k <= kFewTop ? 2 : 1);
}
unsigned short_grid(const pgc_logits* z) {
  const int64_t rows = kWarps * (z->classes <= 128 ? 4 : z->classes <= 256 ? 2 : 1);
  return (unsigned)((z->rows + rows - 1) / rows);
}
// f.template operator()<E, L, R, P>()
template <typename F>
cudaError_t by_width(const pgc_logits* z, F f) {
  const int64_t V = z->classes;
  if (z->dtype == PGC_F32) {
    if (V <= 16) return f.template operator()<float, 8, 2, 1>();
    if (V <= 64) return f.template operator()<float, 8, 8, 1>();
    if (V <= 128) return f.template operator()<float, 8, 16, 1>();
    if (V <= 256) return f.template operator()<float, 16, 16, 1>();
    return f.template operator()<float, 32, 16, 1>();
  }
  using H = __nv_bfloat16;
  const bool two = in_pairs(z);
  if (V <= 16) return f.template operator()<H, 8, 2, 1>();
  if (V <= 64) return two ? f.template operator()<H, 8, 8, 2>() : f.template operator()<H, 8, 8, 1>();
  if (V <= 128) return two ? f.template operator()<H, 8, 16, 2>() : f.template operator()<H, 8, 16, 1>();
  if (V <= 256) return two ? f.template operator()<H, 16, 16, 2>() : f.template operator()<H, 16, 16, 1>();
  return two ? f.template operator()<H, 32, 16, 2>() : f.template operator()<H, 32, 16, 1>();
}
struct ShortScores {
  const pgc_logits* z;
  Scores a;
  cudaStream_t st;
  template <typename E, int L, int R, int P> cudaError_t operator()() {
    short_scores_kernel<E, L, R, P><<<short_grid(z), kThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
};
struct ShortGrad {
  const pgc_logits* z;
  Scores a;
  const float *dlogp, *dentropy;
  cudaStream_t st;
  template <typename E, int L, int R, int P> cudaError_t operator()() {
    short_scores_grad_kernel<E, L, R, P><<<short_grid(z), kThreads, 0, st>>>(a, dlogp, dentropy);
    return cudaGetLastError();
  }
};

template <typename E>
cudaError_t launch_scores(const Scores& a, const Shape& s, cudaStream_t st) {
  const auto kernel = !s.warp ? scores_kernel<E, kThreads, false> : a.k > kFewTop ? scores_kernel<E, 32, true> : scores_kernel<E, 32, false>;
  size_t smem = s.warp ? sizeof(Shared<32>) * kWarps : sizeof(Shared<kThreads>);
  if (s.ranks > 1) smem = (smem + 15) / 16 * 16 + sizeof(Gathered);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)s.ranks;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(s.grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = s.ranks > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

// The gradient takes a longer row in parts of 32 KB at least, few rows in as many as a cluster would have CTAs: 2000 x 50001 fp32
// 122 us, 132 in whole rows, 136 in parts of 16 KB; 4096 x 131072 bf16 310, 323, 357.
constexpr int64_t kGradPartBytes = 32 * 1024;
template <typename E>
cudaError_t launch_grad(const Scores& a, const Shape& s, const float* dlogp, const float* dentropy, cudaStream_t st) {
  const int64_t bytes = a.V * (int64_t)sizeof(E), most = INT32_MAX / a.T;
  const int parts = s.warp ? 1 : (int)std::min(std::max<int64_t>(s.ranks, bytes / kGradPartBytes), most);
  const unsigned grid = s.warp ? s.grid : (unsigned)(a.T * parts);
  if (s.warp) scores_grad_kernel<E, 32><<<grid, kThreads, 0, st>>>(a, parts, dlogp, dentropy);
  else scores_grad_kernel<E, kThreads><<<grid, kThreads, 0, st>>>(a, parts, dlogp, dentropy);
  return cudaGetLastError();
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_token_scores(const pgc_logits *z, int32_t k, float *logp, float *entropy, int32_t *top, float *top_logp,
                     float *stats, void *stream) {
  const int rc = check(z, false);
  if (rc) return rc;
  if (k < 0) return PGC_EINVAL;
  if (k > kMostTop) return PGC_ENOTSUP;
  if (z->rows && (!entropy || !stats || (k && (!top || !top_logp)) || !z->target != !logp)) return PGC_EINVAL;
  if ((uintptr_t)logp % 4 || (uintptr_t)entropy % 4 || (uintptr_t)top % 4 || (uintptr_t)top_logp % 4 || (uintptr_t)stats % 8)
    return PGC_EINVAL;
  if (!z->rows) return PGC_OK;
  Scores a = scores_of(z);
  a.k = k; a.logp = logp; a.entropy = entropy; a.top = top; a.top_logp = top_logp;
  a.stats = reinterpret_cast<float2*>(stats);
  const cudaStream_t st = (cudaStream_t)stream;
  if (short_rows(z, k)) return report_cuda(by_width(z, ShortScores{z, a, st}));
  const Shape s = shape_of(z, k);
  return report_cuda(z->dtype == PGC_BF16 ? launch_scores<__nv_bfloat16>(a, s, st) : launch_scores<float>(a, s, st));
}

int pgc_token_scores_grad(const pgc_logits *z, const float *stats, const float *entropy, const float *dlogp,
                          const float *dentropy, void *stream) {
  const int rc = check(z, true);
  if (rc) return rc;
  if (z->rows && (!stats || (dentropy && !entropy) || (dlogp && !z->target) || (!dlogp && !dentropy))) return PGC_EINVAL;
  if ((uintptr_t)stats % 8 || (uintptr_t)entropy % 4 || (uintptr_t)dlogp % 4 || (uintptr_t)dentropy % 4) return PGC_EINVAL;
  if (!z->rows) return PGC_OK;
  Scores a = scores_of(z);
  a.stats = reinterpret_cast<float2*>(const_cast<float*>(stats));
  a.entropy = const_cast<float*>(entropy);
  const cudaStream_t st = (cudaStream_t)stream;
  if (short_rows(z, 0)) return report_cuda(by_width(z, ShortGrad{z, a, dlogp, dentropy, st}));
  const Shape s = shape_of(z, 0);
  return report_cuda(z->dtype == PGC_BF16 ? launch_grad<__nv_bfloat16>(a, s, dlogp, dentropy, st)
                                          : launch_grad<float>(a, s, dlogp, dentropy, st));
}

}  // extern "C"
