// One row of logits, or a CTA's share of it, read and written in 16-byte
// pieces by a group of threads: the running maximum and sum of its softmax in
// one pass, and the pass that writes coef ([v = y] - p_v) / tau.
//
// Exponents are base 2 with c = log2(e) / tau: 2^(x c - M) for the float
// M = fl(m c).  x c - M is one FMA, rounded once; that M is not m c itself
// does no harm, as any M close to it serves: its residue r = m c - M (exact,
// one FMA) is taken out of the logarithm of the sum.  M is held above -1e8: down to
// there the residue is below 2^3, further down it would pass the range of 2^x.  A
// thread that has met nothing above -1e8 (-inf, or the large negative
// numbers that masks write) adds 2^(x c + 1e8), which is 0 or at most 2^3, and its sum is valid for that
// M; a whole row of such values, or one of products above 1e8, is `extreme` and
// goes through (x - m) c in place of it.
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

// A sum with its rounding errors kept beside it (two-sum): the double unit is
// slow enough here to hold up a row.
struct Sum {
  float s = 0.f, e = 0.f;
  __device__ void add(float v) {
    const float t = s + v, b = t - s;
    e += (s - (t - b)) + (v - b);
    s = t;
  }
  __device__ void add(const Sum& o) {
    add(o.s);
    e += o.e;
  }
  // infinities leave no error behind
  __device__ float value() const { return isfinite(s) ? s + e : s; }
};

__device__ __forceinline__ Sum shuffle_down(const Sum& v, int o) {
  Sum q;
  q.s = __shfl_down_sync(0xffffffffu, v.s, o);
  q.e = __shfl_down_sync(0xffffffffu, v.e, o);
  return q;
}
// The block's sum, in thread 0 (red: one per warp).
__device__ __forceinline__ Sum block_sum(Sum v, Sum* red) {
  const int lane = threadIdx.x % 32, warps = blockDim.x / 32;
  for (int o = 16; o > 0; o >>= 1) v.add(shuffle_down(v, o));
  __syncthreads();
  if (lane == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  if (threadIdx.x < 32) {
    v = lane < warps ? red[lane] : Sum();
    for (int o = 16; o > 0; o >>= 1) v.add(shuffle_down(v, o));
  }
  return v;
}

// Two floats side by side: one instruction does both (add, multiply, FMA).
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi) {
  Pair p;
  asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(lo), "f"(hi));
  return p;
}
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ Pair ex2_2(Pair a) {
  float lo, hi;
  split(a, lo, hi);
  return pair(ex2(lo), ex2(hi));
}

template <typename E>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int N = 4;    // elements of a piece
  static constexpr uint32_t kLowest = 0xff800000u;   // -inf throughout
  __device__ static float get(const float* p) { return *p; }
  __device__ static void put(float* p, float v) { *p = v; }
  __device__ static void widen(const uint4& r, Pair* o) {
    o[0] = pair(__uint_as_float(r.x), __uint_as_float(r.y));
    o[1] = pair(__uint_as_float(r.z), __uint_as_float(r.w));
  }
  __device__ static uint4 narrow(const Pair* o) {
    float a, b, c, d;
    split(o[0], a, b);
    split(o[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  }
  // the largest element of U pieces
  template <int U>
  __device__ static float top(const uint4 (&v)[U]) {
    float m = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      m = fmaxf(fmaxf(m, __uint_as_float(v[u].x)), __uint_as_float(v[u].y));
      m = fmaxf(fmaxf(m, __uint_as_float(v[u].z)), __uint_as_float(v[u].w));
    }
    return m;
  }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr uint32_t kLowest = 0xff80ff80u;
  __device__ static float get(const __nv_bfloat16* p) { return __bfloat162float(*p); }
  __device__ static void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
  __device__ static Pair wide(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  __device__ static void widen(const uint4& r, Pair* o) {
    o[0] = wide(r.x); o[1] = wide(r.y); o[2] = wide(r.z); o[3] = wide(r.w);
  }
  __device__ static uint32_t two(Pair p) {
    float lo, hi;
    split(p, lo, hi);
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&b);
  }
  __device__ static uint4 narrow(const Pair* o) { return make_uint4(two(o[0]), two(o[1]), two(o[2]), two(o[3])); }
  __device__ static uint32_t top2(uint32_t a, uint32_t b) {
    uint32_t m;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(m) : "r"(a), "r"(b));
    return m;
  }
  template <int U>
  __device__ static float top(const uint4 (&v)[U]) {
    uint32_t m = kLowest;
#pragma unroll
    for (int u = 0; u < U; ++u) m = top2(m, top2(top2(v[u].x, v[u].y), top2(v[u].z, v[u].w)));
    return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
};
__device__ __forceinline__ uint4 no_piece(uint32_t lowest) { return make_uint4(lowest, lowest, lowest, lowest); }

__device__ __forceinline__ uint4 load16(const uint4* p) { return __ldcg(p); }
__device__ __forceinline__ void store16(uint4* p, const uint4& v) { __stcs(p, v); }

// Elements [first, last) of a row: `head` single ones up to a 16-byte
// boundary, pieces, and a rest behind them.  A row has up to 2^31 - 1 elements:
// an index of single elements that steps beyond the last one is unsigned, as
// int would turn negative there; pieces are at most 2^29.
struct Slice {
  int first, last, head, pieces;
};
// The part of CTA `rank` of `ranks` in a row that starts at x: the pieces in
// parts that differ by one at most, and the row's ends.
template <typename E>
__device__ __forceinline__ Slice slice_of(const E* x, int n, int rank, int ranks) {
  constexpr int N = Elem<E>::N;
  const int off = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(E)) & (N - 1);
  const int head = min(n, (N - off) & (N - 1)), pieces = (n - head) / N;
  if (ranks == 1) return Slice{0, n, head, pieces};
  const int part = (unsigned)pieces / (unsigned)ranks, more = pieces - part * ranks;
  const int p0 = rank * part + min(rank, more), p1 = p0 + part + (rank < more ? 1 : 0);
  Slice s;
  s.first = rank ? head + p0 * N : 0;
  s.last = rank == ranks - 1 ? n : head + p1 * N;
  s.head = rank ? 0 : head;
  s.pieces = p1 - p0;
  return s;
}

// Running maximum and sum: s = sum of 2^(x c - M), M = max(fl(m c), -kFar).
constexpr float kFar = 1e8f;
struct Online {
  float m = -INFINITY, M = -kFar, s = 0.f;
};
__device__ __forceinline__ float ref_of(float m, float c) { return fmaxf(m * c, -kFar); }
__device__ __forceinline__ void raise(Online& o, float top, float c) {
  if (top > o.m) {
    const float M = ref_of(top, c);
    o.s *= ex2(o.M - M);
    o.m = top;
    o.M = M;
  }
}
__device__ __forceinline__ void add_one(Online& o, float f, float c) {
  raise(o, f, c);
  o.s += ex2(fmaf(f, c, -o.M));
}
template <typename E, int U>
__device__ __forceinline__ void add_exps(Pair (&sum)[2], const uint4 (&v)[U], Pair c2, Pair M2) {
  constexpr int H = Elem<E>::N / 2;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    Pair f[H];
    Elem<E>::widen(v[u], f);
#pragma unroll
    for (int i = 0; i < H; ++i) sum[i % 2] = add2(sum[i % 2], ex2_2(fma2(f[i], c2, M2)));
  }
}
template <typename E, int U>
__device__ __forceinline__ void add_pieces(Online& o, const uint4 (&v)[U], float c) {
  raise(o, Elem<E>::top(v), c);
  Pair sum[2] = {0, 0};
  add_exps<E>(sum, v, pair(c, c), pair(-o.M, -o.M));
  float lo, hi;
  split(add2(sum[0], sum[1]), lo, hi);
  o.s += lo + hi;
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
  if (tid < s.head + (s.last - rest)) add_one(o, Elem<E>::get(x + (tid < s.head ? s.first + tid : rest + tid - s.head)), c);
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  for (int i = tid; i < s.pieces; i += G * U) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = i + u * G < s.pieces ? load16(p + i + u * G) : no_piece(Elem<E>::kLowest);
    add_pieces<E>(o, v, c);
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
// A row whose largest logit leaves the range of the fast path: beyond kFar
// 2^(residue of m c) would soon overflow, and M is no longer fl(m c).
__device__ __forceinline__ bool is_extreme(float m, float c) { return !(fabsf(m) < 1e37f && fabsf(m * c) < kFar); }

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
  Pair f[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) f[i] = pair(value, value);
  const uint4 v = Elem<E>::narrow(f);
  uint4* p = reinterpret_cast<uint4*>(g + first + head);
  for (int i = tid; i < pieces; i += G) store16(p + i, v);
}

template <typename E>
__device__ __noinline__ void slice_grad_extreme(const E* x, E* g, int first, int last, int tid, int threads, RowGrad r) {
  for (unsigned v = first + tid; v < (unsigned)last; v += threads) {
    const float p = exp2f((Elem<E>::get(x + v) - r.m) * r.c - r.l2);
    Elem<E>::put(g + v, r.k * p + ((int)v == r.y ? r.at_y : 0.f));
  }
}

// A piece's gradient but for the target's part; `wide`: out is 16-byte aligned.
template <typename E>
__device__ __forceinline__ void put_piece(const uint4& v, E* out, bool wide, const RowGrad& r) {
  constexpr int N = Elem<E>::N;
  Pair f[N / 2];
  Elem<E>::widen(v, f);
  const Pair c2 = pair(r.c, r.c), M2 = pair(-r.M, -r.M), k2 = pair(r.scale, r.scale);
#pragma unroll
  for (int i = 0; i < N / 2; ++i) f[i] = mul2(ex2_2(fma2(f[i], c2, M2)), k2);
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
__device__ __forceinline__ float grad_at(float x, bool target, const RowGrad& r) {
  return fmaf(ex2(fmaf(x, r.c, -r.M)), r.scale, target ? r.at_y : 0.f);
}
// The target's element, written again by the thread that wrote its piece.
template <typename E, int G>
__device__ __forceinline__ void put_target(E* g, const Slice& s, int tid, float xy, const RowGrad& r) {
  const int at = r.y - (s.first + s.head);
  if (at >= 0 && at < s.pieces * Elem<E>::N && at / Elem<E>::N % G == tid) Elem<E>::put(g + r.y, grad_at(xy, true, r));
}

// xy: the target's logit, read before any of the row's gradient is written
template <typename E, int G, int U>
__device__ __forceinline__ void slice_grad(const E* x, E* g, const Slice& s, int tid, float xy, const RowGrad& r) {
  constexpr int N = Elem<E>::N;
  if (r.extreme) {
    slice_grad_extreme(x, g, s.first, s.last, tid, G, r);
    return;
  }
  const int body = s.first + s.head, rest = body + s.pieces * N;
  if (tid < s.head + (s.last - rest)) {
    const int v = tid < s.head ? s.first + tid : rest + tid - s.head;
    Elem<E>::put(g + v, grad_at(Elem<E>::get(x + v), v == r.y, r));
  }
  const uint4* p = reinterpret_cast<const uint4*>(x + body);
  const bool wide = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  for (int i = tid; i < s.pieces; i += G * U) {
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * G < s.pieces) v[u] = load16(p + i + u * G);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i + u * G < s.pieces) put_piece<E>(v[u], g + body + (i + u * G) * N, wide, r);
  }
  put_target<E, G>(g, s, tid, xy, r);
}

// ---- a row kept in shared memory ---------------------------------------------
// Every thread copies its own pieces (tid, tid + G, ...) with cp.async, in two
// groups, and reads only those: no barrier is needed between the copies, the
// reads and the copies of the next row into the places just read.  A thread has
// `most` places (even, the same for every row of a launch); the ones behind
// the row's last piece hold -inf, which adds nothing.  Rows differ by one piece
// at most, so only the last two places can be such ones.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_close() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint4 read16(uint32_t at) {
  uint4 v;
  asm ("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}

template <typename E>
struct Held {
  const E* x;         // row
  Slice s;
  float edge;         // this thread's element outside the pieces (tid < edges)
  int edge_at;        // its index, or -1
};
template <typename E>
__device__ __forceinline__ Held<E> hold(const E* x, const Slice& s, int tid) {
  Held<E> h{x, s, 0.f, -1};
  const int rest = s.first + s.head + s.pieces * Elem<E>::N;
  if (tid < s.head + (s.last - rest)) {
    h.edge_at = tid < s.head ? s.first + tid : rest + tid - s.head;
    h.edge = Elem<E>::get(x + h.edge_at);
  }
  return h;
}
// Piece i of a row into its place; behind the last one stands what adds nothing.
template <typename E>
__device__ __forceinline__ void copy_piece(uint32_t at, const uint4* p, int i, int pieces) {
  if (i < pieces) copy16(at + i * 16, p + i);
  else asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at + i * 16), "r"(Elem<E>::kLowest) : "memory");
}
template <typename E, int G>
__device__ __forceinline__ void copy_last(uint32_t at, const uint4* p, int tid, int pieces, int most) {
  copy_piece<E>(at, p, (most - 2) * G + tid, pieces);
  copy_piece<E>(at, p, (most - 1) * G + tid, pieces);
}
// Places of the first of the two groups.
__device__ __forceinline__ int first_group(int most) { return most / 4 * 2; }

template <typename E, int G>
__device__ __forceinline__ void copy_row(const Held<E>& h, uint32_t at, int tid, int most) {
  const uint4* p = reinterpret_cast<const uint4*>(h.x + h.s.first + h.s.head);
  const int half = first_group(most);
#pragma unroll 2
  for (int k = 0; k < half; ++k) copy16(at + tid * 16 + k * (G * 16), p + tid + k * G);
  copies_close();
#pragma unroll 2
  for (int k = half; k < most - 2; ++k) copy16(at + tid * 16 + k * (G * 16), p + tid + k * G);
  copy_last<E, G>(at, p, tid, h.s.pieces, most);
  copies_close();
}

template <typename E, int G>
__device__ __forceinline__ Online held_stats(const Held<E>& h, uint32_t at, int tid, float c, int most) {
  Online o;
  at += tid * 16;
  const int half = first_group(most);
  copies_wait<1>();
#pragma unroll 1
  for (int k = 0; k < most; k += 2) {
    if (k == half) copies_wait<0>();
    const uint4 v[2] = {read16(at), read16(at + G * 16)};
    at += 2 * G * 16;
    add_pieces<E>(o, v, c);
  }
  if (h.edge_at >= 0) add_one(o, h.edge, c);
  return o;
}
// Sum of exponentials at the maximum m, of an extreme row.
template <typename E, int G>
__device__ __noinline__ float held_sum_extreme(Held<E> h, uint32_t at, int tid, float m, float c) {
  constexpr int N = Elem<E>::N;
  float s = h.edge_at >= 0 ? exp2f((h.edge - m) * c) : 0.f;
  for (int i = tid; i < h.s.pieces; i += G) {
    Pair f[N / 2];
    Elem<E>::widen(read16(at + i * 16), f);
    for (int q = 0; q < N / 2; ++q) {
      float lo, hi;
      split(f[q], lo, hi);
      s += exp2f((lo - m) * c) + exp2f((hi - m) * c);
    }
  }
  return s;
}

template <typename E, int G>
__device__ __noinline__ void held_grad_extreme(Held<E> h, E* g, uint32_t at, int tid, RowGrad r) {
  constexpr int N = Elem<E>::N;
  const int body = h.s.first + h.s.head;
  if (h.edge_at >= 0)
    Elem<E>::put(g + h.edge_at, r.k * exp2f((h.edge - r.m) * r.c - r.l2) + (h.edge_at == r.y ? r.at_y : 0.f));
  for (int i = tid; i < h.s.pieces; i += G) {
    Pair f[N / 2];
    Elem<E>::widen(read16(at + i * 16), f);
    for (int j = 0; j < N; ++j) {
      float two[2];
      split(f[j / 2], two[0], two[1]);
      Elem<E>::put(g + body + i * N + j,
                   r.k * exp2f((two[j % 2] - r.m) * r.c - r.l2) + (body + i * N + j == r.y ? r.at_y : 0.f));
    }
  }
}

// The gradient of the held row, and (kCopy) the next row's copies into its place.
template <typename E, int G, bool kWide, bool kCopy>
__device__ __forceinline__ void held_grad_loop(const Held<E>& h, E* out, uint32_t at, int tid, const RowGrad& r, int most,
                                               const uint4* p, int next_pieces) {
  constexpr int N = Elem<E>::N;
  const uint32_t row_at = at;
  const uint4* row_p = p;
  at += tid * 16;
  out += tid * N;
  p += tid;
  const int half = first_group(most);
#pragma unroll 1
  for (int k = 0; k < most - 2; k += 2) {
    if (k == half) copies_close();
    const uint4 v0 = read16(at), v1 = read16(at + G * 16);
    if (kCopy) {
      copy16(at, p);
      copy16(at + G * 16, p + G);
    }
    put_piece<E>(v0, out, kWide, r);
    put_piece<E>(v1, out + G * N, kWide, r);
    at += 2 * G * 16;
    p += 2 * G;
    out += 2 * G * N;
  }
  if (half == most - 2) copies_close();
  const int i = (most - 2) * G + tid;
  const uint4 v0 = read16(at), v1 = read16(at + G * 16);
  if (kCopy) copy_last<E, G>(row_at, row_p, tid, next_pieces, most);
  copies_close();
  if (i < h.s.pieces) put_piece<E>(v0, out, kWide, r);
  if (i + G < h.s.pieces) put_piece<E>(v1, out + G * N, kWide, r);
}
template <typename E, int G>
__device__ __forceinline__ void held_grad(const Held<E>& h, E* g, uint32_t at, int tid, float xy, const RowGrad& r,
                                          int most, bool copy, const Held<E>& next) {
  if (h.edge_at >= 0) Elem<E>::put(g + h.edge_at, grad_at(h.edge, h.edge_at == r.y, r));
  E* out = g + h.s.first + h.s.head;
  const uint4* p = reinterpret_cast<const uint4*>(next.x + next.s.first + next.s.head);
  if (((reinterpret_cast<uintptr_t>(h.x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0) {
    if (copy) held_grad_loop<E, G, true, true>(h, out, at, tid, r, most, p, next.s.pieces);
    else held_grad_loop<E, G, true, false>(h, out, at, tid, r, most, p, 0);
  } else {
    if (copy) held_grad_loop<E, G, false, true>(h, out, at, tid, r, most, p, next.s.pieces);
    else held_grad_loop<E, G, false, false>(h, out, at, tid, r, most, p, 0);
  }
  put_target<E, G>(g, h.s, tid, xy, r);
}

}  // namespace pgc
