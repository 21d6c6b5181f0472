// One row of logits, or a CTA's share of it, read and written in 16-byte
// pieces by a group of threads: the running maximum and sum of its softmax in
// one pass, and the pass that writes coef ([v = y] - p_v) / tau.
//
// Exponents are base 2 with c = log2(e) / tau: 2^(x c - M) for the float
// M = fl(m c).  x c - M is one FMA, rounded once; that M is not m c itself
// does no harm, as any M close to it serves: its residue r = m c - M (exact,
// one FMA) is taken out of the logarithm of the sum.  M is held above -1e38, so that a
// thread that has met nothing but -inf (or the type's lowest value, as masks
// write it) adds 0 instead of NaN; a whole row of such values, or one whose
// products overflow, is `extreme` and goes through (x - m) c in place of it.
#pragma once

#include "dev_common.cuh"

namespace pgc {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename E>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int N = 4;    // elements of a piece
  static constexpr uint32_t kLowest = 0xff800000u;   // -inf throughout
  __device__ static float get(const float* p) { return *p; }
  __device__ static void put(float* p, float v) { *p = v; }
  __device__ static void widen(const uint4& r, float* o) {
    o[0] = __uint_as_float(r.x); o[1] = __uint_as_float(r.y); o[2] = __uint_as_float(r.z); o[3] = __uint_as_float(r.w);
  }
  __device__ static uint4 narrow(const float* o) {
    return make_uint4(__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
  }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr uint32_t kLowest = 0xff80ff80u;
  __device__ static float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  __device__ static void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
  __device__ static void widen(const uint4& r, float* o) { Vec<uint16_t, 8>::widen(r, o); }
  __device__ static uint32_t two(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
  __device__ static uint4 narrow(const float* o) {
    return make_uint4(two(o[0], o[1]), two(o[2], o[3]), two(o[4], o[5]), two(o[6], o[7]));
  }
};

__device__ __forceinline__ uint4 load16(const uint4* p) { return __ldcg(p); }
__device__ __forceinline__ void store16(uint4* p, const uint4& v) { __stcs(p, v); }

// Elements [first, last) of a row: `head` single ones up to a 16-byte
// boundary, pieces, and a rest behind them.
struct Slice {
  int first, last, head, pieces;
};
// The share of CTA `rank` of `ranks` in a row that starts at x: whole pieces
// but for the row's ends.
template <typename E>
__device__ __forceinline__ Slice slice_of(const E* x, int n, int rank, int ranks) {
  constexpr int N = Elem<E>::N;
  const int off = (int)((reinterpret_cast<uintptr_t>(x) / sizeof(E)) % N);
  const int head = min(n, (N - off) % N), pieces = (n - head) / N;
  if (ranks == 1) return Slice{0, n, head, pieces};
  const int p0 = (int)((int64_t)pieces * rank / ranks), p1 = (int)((int64_t)pieces * (rank + 1) / ranks);
  Slice s;
  s.first = rank ? head + p0 * N : 0;
  s.last = rank == ranks - 1 ? n : head + p1 * N;
  s.head = rank ? 0 : head;
  s.pieces = p1 - p0;
  return s;
}

// Running maximum and sum: s = sum of 2^(x c - M), M = max(fl(m c), -1e38).
struct Online {
  float m = -INFINITY, M = -1e38f, s = 0.f;
};
__device__ __forceinline__ float ref_of(float m, float c) { return fmaxf(m * c, -1e38f); }
template <int K>
__device__ __forceinline__ void add_all(Online& o, const float (&f)[K], float c) {
  float top = f[0];
#pragma unroll
  for (int i = 1; i < K; ++i) top = fmaxf(top, f[i]);
  if (top > o.m) {
    const float M = ref_of(top, c);
    o.s *= ex2(o.M - M);
    o.m = top;
    o.M = M;
  }
  float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < K; ++i) part[i % 4] += ex2(fmaf(f[i], c, -o.M));
  o.s += (part[0] + part[1]) + (part[2] + part[3]);
}
__device__ __forceinline__ Online warp_merge(Online o, float c) {
  Online r;
  r.m = warp_max(o.m);
  r.M = ref_of(r.m, c);
  r.s = warp_sum(o.s * ex2(o.M - r.M));
  return r;
}

// This thread's part (tid of G) of a slice's maximum and sum.
template <typename E, int G, int U>
__device__ __forceinline__ Online slice_stats(const E* x, const Slice& s, int tid, float c) {
  constexpr int N = Elem<E>::N;
  Online o;
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (tid < s.head + (s.last - rest)) {
    const float f[1] = {Elem<E>::get(x + (tid < s.head ? s.first + tid : rest + tid - s.head))};
    add_all(o, f, c);
  }
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  for (int i = tid; i < s.pieces; i += G * U) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      v[u] = i + u * G < s.pieces ? load16(p + i + u * G)
                                  : make_uint4(Elem<E>::kLowest, Elem<E>::kLowest, Elem<E>::kLowest, Elem<E>::kLowest);
    float f[U * N];
#pragma unroll
    for (int u = 0; u < U; ++u) Elem<E>::widen(v[u], f + u * N);
    add_all(o, f, c);
  }
  return o;
}

// What the gradient pass needs of a row.
struct RowGrad {
  float m, M, c;
  float scale;    // -coef / tau times 2^-(log2 of the sum at M)
  float at_y;     // coef / tau, added at y
  int y;
  bool extreme;
  float l2;       // log2 of the sum at m (extreme rows)
  float k;        // -coef / tau (extreme rows)
};
// A row whose largest logit, or its product with c, leaves the range of the fast path.
__device__ __forceinline__ bool is_extreme(float m, float c) { return !(fabsf(m) < 1e37f && fabsf(m * c) < 1e37f); }

__device__ __forceinline__ RowGrad row_grad(float m, float L, float coef, float inv_tau, float c, int y) {
  RowGrad g;
  g.m = m;
  g.c = c;
  g.M = ref_of(m, c);
  g.y = y;
  g.at_y = coef * inv_tau;
  g.k = -g.at_y;
  g.extreme = is_extreme(m, c);
  g.l2 = L * kLog2e;
  g.scale = g.k * exp2f(-(fmaf(m, c, -g.M) + g.l2));
  return g;
}

template <typename E, int G>
__device__ __forceinline__ void slice_fill(E* g, int first, int last, int tid, float value) {
  constexpr int N = Elem<E>::N;
  const int off = (int)((reinterpret_cast<uintptr_t>(g + first) / sizeof(E)) % N);
  const int head = min(last - first, (N - off) % N), pieces = (last - first - head) / N;
  const int rest = first + head + pieces * N;
  if (tid < head) Elem<E>::put(g + first + tid, value);
  if (tid < last - rest) Elem<E>::put(g + rest + tid, value);
  float f[N];
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = value;
  const uint4 v = Elem<E>::narrow(f);
  uint4* p = reinterpret_cast<uint4*>(g + first + head);
  for (int i = tid; i < pieces; i += G) store16(p + i, v);
}

template <typename E>
__device__ __noinline__ void slice_grad_extreme(const E* x, E* g, int first, int last, int tid, int threads, RowGrad r) {
  for (int v = first + tid; v < last; v += threads) {
    const float p = exp2f((Elem<E>::get(x + v) - r.m) * r.c - r.l2);
    Elem<E>::put(g + v, r.k * p + (v == r.y ? r.at_y : 0.f));
  }
}

template <typename E, int G, int U>
__device__ __forceinline__ void slice_grad(const E* x, E* g, const Slice& s, int tid, const RowGrad& r) {
  constexpr int N = Elem<E>::N;
  if (r.extreme) {
    slice_grad_extreme(x, g, s.first, s.last, tid, G, r);
    return;
  }
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (tid < s.head + (s.last - rest)) {
    const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
    Elem<E>::put(g + v, fmaf(ex2(fmaf(Elem<E>::get(x + v), r.c, -r.M)), r.scale, v == r.y ? r.at_y : 0.f));
  }
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  for (int i = tid; i < s.pieces; i += G * U) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * G < s.pieces) v[u] = load16(p + i + u * G);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = i + u * G;
      if (j >= s.pieces) break;
      float f[N];
      Elem<E>::widen(v[u], f);
#pragma unroll
      for (int q = 0; q < N; ++q) f[q] = ex2(fmaf(f[q], r.c, -r.M)) * r.scale;
      const unsigned at = (unsigned)(r.y - (body + j * N));
      if (at < (unsigned)N) {
#pragma unroll
        for (int q = 0; q < N; ++q) f[q] += at == q ? r.at_y : 0.f;
      }
      E* out = g + body + j * N;
      if (wide) {
        store16(reinterpret_cast<uint4*>(out), Elem<E>::narrow(f));
      } else {
#pragma unroll
        for (int q = 0; q < N; ++q) Elem<E>::put(out + q, f[q]);
      }
    }
  }
}

}  // namespace pgc
