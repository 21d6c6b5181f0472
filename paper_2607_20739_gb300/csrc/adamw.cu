// AdamW over many tensors (pgc_adamw_step), moments in 32 bits or in 8.
//
//   g = grad * grad_scale
//   m' = beta1 m + (1 - beta1) g,   v' = beta2 v + (1 - beta2) g^2
//   p' = p (1 - lr decay) - lr (m' / (1 - beta1^t)) / (sqrt(v' / (1 - beta2^t)) + eps)
//
// Moments in 8 bits.  256 elements (a block) have one scale, a power of two, so
// that a value on a code's place stays on one whatever its block's largest
// element does.  A first moment is an 8-bit float of 4 bits of exponent and 3 of fraction times the
// scale; a second moment, which has no sign, has 16 codes an octave in the upper
// 8 octaves and 8 in the 16 below; its code 0 is kept for zero, so that no
// parameter whose gradient is small beside its neighbours' is divided by
// eps alone.  What lies between two codes goes up or down by chance, in proportion: to the nearest
// code a second moment would never leave its own (a step changes it by
// 1 - beta2, 0.001 say, and codes are 0.04 apart).
#include <algorithm>
#include <atomic>
#include <cmath>

#include <cuda_fp16.h>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlock = 256;           // elements with one scale, and what a warp takes at once: eight a lane

struct Tensor {
  void* p;
  const void* g;
  __nv_bfloat16* copy;
  void *m, *v;
  float *ms, *vs;
  int64_t n;                          // its sign bit set: not all of its arrays allow four elements at once
};
struct Rates {
  float lr, decay;
  const float* lr_at;
  const int64_t* step_at;
  const float* scale_at;
  float b1, b2, omb1, omb2, eps;      // omb: one minus beta
  float log_b1, log_b2;
  float size, rc1, rc2;               // lr / (1 - beta1^t), 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float keep;                         // 1 - lr decay
  float one;                          // 1
  uint32_t seed, step_lo;
};
constexpr int kMost = 240;            // tensors of a launch: what its arguments have room for
struct Table {
  Tensor t[kMost];
  uint32_t first[kMost + 1];          // blocks before each
  uint32_t ordinal[kMost];
  int count;
};

// What every element of a step has in common.
struct Step {
  float size, rc2, keep, scale;
  uint32_t key;                       // of seed and step
};

// 32 bits scattered, one to one: products by odd numbers (digits of square roots) and shifts.
constexpr uint32_t kOdd1 = 0x6A09E667u, kOdd2 = 0xBB67AE85u;
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
  h = (h ^ (h >> 16)) * kOdd1;
  h = (h ^ (h >> 15)) * kOdd2;
  return h ^ (h >> 16);
}

__device__ __forceinline__ Step step_of(const Rates& r) {
  Step s{r.size, r.rc2, r.keep, r.scale_at ? *r.scale_at : 1.f, 0};
  uint32_t t = r.step_lo;
  if (r.step_at || r.lr_at) {
    const float lr = r.lr_at ? *r.lr_at : r.lr;
    float rc1 = r.rc1;
    if (r.step_at) {
      const int64_t at = *r.step_at;
      t = (uint32_t)at;
      rc1 = -1.f / expm1f((float)at * r.log_b1);
      s.rc2 = 1.f / sqrtf(-expm1f((float)at * r.log_b2));
    }
    s.size = lr * rc1;
    s.keep = 1.f - lr * r.decay;
  }
  s.key = mix(mix(r.seed) + t);
  return s;
}

// Two elements at once.  Products and sums are rounded one by one, in this order, whatever kernel: the
// codes of a step are then the same wherever it is computed.  The assembler makes an FMA of a packed
// product and sum although both ask for their own rounding, so the sum is an FMA with a 1 that it does not know.
__device__ __forceinline__ Pair both(float f) { return pair(f, f); }
__device__ __forceinline__ Pair decay_to(Pair old, float keep, Pair now, float share, float one) {
  return fma2(mul2(old, both(keep)), both(one), mul2(now, both(share)));
}
__device__ __forceinline__ float root(float v) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float over(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// kExact: with so small an eps a v below the smallest normal float still counts.
template <bool kExact>
__device__ __forceinline__ Pair param(Pair p, Pair m, Pair v, const Step& s, float eps) {
  float v0, v1;
  split(v, v0, v1);
  if (kExact) {
    float p0, p1, m0, m1;
    split(p, p0, p1);
    split(m, m0, m1);
    return pair(p0 * s.keep - s.size * m0 / (sqrtf(v0) * s.rc2 + eps), p1 * s.keep - s.size * m1 / (sqrtf(v1) * s.rc2 + eps));
  }
  split(fma2(pair(root(v0), root(v1)), both(s.rc2), both(eps)), v0, v1);
  return fma2(mul2(m, both(-s.size)), pair(over(v0), over(v1)), mul2(p, both(s.keep)));
}

// A CTA has consecutive blocks of all tensors' in a row, as many as every other: its parts of tensors, one
// after another.
struct Share {
  uint32_t at, end;             // blocks
  int tensor;
  __device__ __forceinline__ explicit Share(const Table& a) {
    const uint64_t all = a.first[a.count];
    at = (uint32_t)(all * blockIdx.x / gridDim.x);
    end = (uint32_t)(all * (blockIdx.x + 1) / gridDim.x);
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (a.first[mid] <= at) lo = mid;
      else hi = mid;
    }
    tensor = lo;
  }
  // The next part: its tensor, the first of its blocks there and how many; 2^31 elements of a tensor are never
  // crossed, so that an index within a part is 32 bits, and the upper half of an element's the same in all of it.
  __device__ __forceinline__ bool next(const Table& a, int* of, uint32_t* block, uint32_t* count) {
    if (at >= end) return false;
    while (at >= a.first[tensor + 1]) ++tensor;
    *of = tensor;
    *block = at - a.first[tensor];
    constexpr uint32_t kSide = 1u << 23;
    *count = min(min(end, a.first[tensor + 1]) - at, kSide - *block % kSide);
    at += *count;
    return true;
  }
};

// Four elements at once, as two pairs; eight of a block are a lane's: 4 l .. 4 l + 3 and the same behind the first 128.
struct Four {
  Pair a, b;
};
__device__ __forceinline__ Four load4(const float* p) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  return Four{pair(v.x, v.y), pair(v.z, v.w)};
}
__device__ __forceinline__ Four load4(const __nv_bfloat16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return Four{Elem<__nv_bfloat16>::wide(v.x), Elem<__nv_bfloat16>::wide(v.y)};
}
__device__ __forceinline__ void store4(float* p, Pair a, Pair b) {
  float4 v;
  split(a, v.x, v.y);
  split(b, v.z, v.w);
  *reinterpret_cast<float4*>(p) = v;
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, Pair a, Pair b) {
  using H = Elem<__nv_bfloat16>;
  *reinterpret_cast<uint2*>(p) = make_uint2(H::two(a), H::two(b));
}
constexpr int kEach = kBlock / 32, kPairs = kEach / 2;
__device__ __forceinline__ int place_of(int lane, int j) { return 4 * lane + j % 4 + j / 4 * 128; }

// A lane's eight elements of the block at p; `all`: all there, and four at once allowed.
template <typename E>
__device__ __forceinline__ void load8(const E* p, int lane, int64_t left, bool all, Pair (&f)[kPairs]) {
  if (all) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const Four v = load4(p + place_of(lane, 4 * h));
      f[2 * h] = v.a;
      f[2 * h + 1] = v.b;
    }
  } else {
    float g[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) g[j] = place_of(lane, j) < left ? Elem<E>::get(p + place_of(lane, j)) : 0.f;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) f[j] = pair(g[2 * j], g[2 * j + 1]);
  }
}
template <typename E>
__device__ __forceinline__ void store8(E* p, int lane, int64_t left, bool all, const Pair (&f)[kPairs]) {
  if (all) {
#pragma unroll
    for (int h = 0; h < 2; ++h) store4(p + place_of(lane, 4 * h), f[2 * h], f[2 * h + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      float lo, hi;
      split(f[j / 2], lo, hi);
      if (place_of(lane, j) < left) Elem<E>::put(p + place_of(lane, j), j % 2 ? hi : lo);
    }
  }
}

// A block a warp at a time; memory bounds it (403 M fp32: 1657 us, 6.8 TB/s; 72 M bf16: 249).
template <typename P, typename G, bool kExact>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  const Step s = step_of(r);
  const int lane = threadIdx.x % 32;
  Share share(a);
  int of;
  uint32_t block, count;
  while (share.next(a, &of, &block, &count)) {
    const Tensor& t = a.t[of];
    const int64_t n = t.n & INT64_MAX;
    for (uint32_t b = threadIdx.x / 32; b < count; b += kWarps) {
      const int64_t i = ((int64_t)block + b) * kBlock, left = n - i;
      const bool all = t.n >= 0 && left >= kBlock;
      Pair p[kPairs], g[kPairs], m[kPairs], v[kPairs];
      load8(static_cast<const G*>(t.g) + i, lane, left, all, g);
      load8(static_cast<const float*>(t.m) + i, lane, left, all, m);
      load8(static_cast<const float*>(t.v) + i, lane, left, all, v);
      load8(static_cast<const P*>(t.p) + i, lane, left, all, p);
#pragma unroll
      for (int j = 0; j < kPairs; ++j) {
        const Pair q = mul2(g[j], both(s.scale));
        m[j] = decay_to(m[j], r.b1, q, r.omb1, r.one);
        v[j] = decay_to(v[j], r.b2, mul2(q, q), r.omb2, r.one);
        p[j] = param<kExact>(p[j], m[j], v[j], s, r.eps);
      }
      store8(static_cast<float*>(t.m) + i, lane, left, all, m);
      store8(static_cast<float*>(t.v) + i, lane, left, all, v);
      store8(static_cast<P*>(t.p) + i, lane, left, all, p);
      if (t.copy) store8(t.copy + i, lane, left, all, p);
    }
  }
}

// ---- moments in 8 bits ---------------------------------------------------------

// Codes of four elements, and their values before the scale.  What follows counts instructions: at
// 10 bytes an element (bf16 parameters and gradients) an SM has 55 issue slots for it while its share of memory moves, and
// its unit of compares, shifts and logic half as many.  So shifts to the left are products, choices maxima, and a
// second moment's values a table; what is rare (a value below the lowest code, a block without a scale) is put right
// behind a branch.  About 53 instructions an element are left (82 as first written), and they are the bound: 72 M in 133 us, 5.4 TB/s.
// With fp32 parameters memory is: 403 M with copies in 950 us, 6.8 TB/s.
__device__ __forceinline__ Four decode_m(uint32_t codes) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(codes));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return Four{pair(x.x, x.y), pair(y.x, y.y)};
}
// (c + 865) 2^20 below 127, (c + 1857) 2^19 from there on, as the bits of a float; 0 for 0.
__device__ __forceinline__ float decode_v(uint32_t c) {
  const uint32_t low = c * (1u << 20) + (865u << 20);
  return __uint_as_float(min(max(c, 127u) * (0u - (1u << 19)) + (low + (127u << 19)), 0u - c));
}
// The chances of a first and a second moment, 16 bits each, where the encodings want them: in the two
// middle bytes, over half a step.  h: before the last step of mix, h ^ h >> 16, whose upper half is h's.
struct Chances {
  uint32_t m, v;
};
__device__ __forceinline__ Chances chances_of(uint32_t h) {
  Chances c;
  c.v = __byte_perm(h, 0x80, 0x7324);                      // 0x80, the bytes 2 and 3 of h, 0
  c.m = __byte_perm(h, 0x40000000, 0x7104) ^ c.v;           // 0x80, those of h ^ h >> 16, 0x40
  return c;
}
// The code in the upper byte.  y = |m| / scale, below 2^8: twenty bits below a code's last place
// decide.  Codes are linear below 2^-6, where y + 2^-6 has their bits; the larger of the two places is the right one.
__device__ __forceinline__ uint32_t encode_m(float y, uint32_t chance) {
  const int w = __viaddmax_s32(__float_as_int(__fadd_rz(y, 0x1p-6f)), -(1 << 23), __float_as_int(y));
  return (uint32_t)w * 16u + chance;                        // - (120 << 23) 16 is 0x40 in the upper byte
}
// Sixteen codes an octave from 2^-3 on, eight below: again the larger place.  y as bits, those of code 1 at least.
constexpr int kLowestCode = 866 << 20;
__device__ __forceinline__ uint32_t encode_v(int y, uint32_t chance) {
  return (uint32_t)(__viaddmax_s32(y, -(1857 << 20), -(865 << 20)) + y) * 16u + chance;
}
// The upper bytes of four words.
__device__ __forceinline__ uint32_t bytes4(const uint32_t (&c)[4]) {
  return __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
}
// A lane's eight codes of the block at p, four a word, one by one.
__device__ __forceinline__ void load_codes(const uint8_t* p, int lane, int64_t left, uint32_t (&c)[2]) {
  c[0] = c[1] = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j)
    if (place_of(lane, j) < left) c[j / 4] |= (uint32_t)p[place_of(lane, j)] << (j % 4 * 8);
}
__device__ __forceinline__ void store_codes(uint8_t* p, int lane, int64_t left, const uint32_t (&c)[2]) {
#pragma unroll
  for (int j = 0; j < kEach; ++j)
    if (place_of(lane, j) < left) p[place_of(lane, j)] = (uint8_t)(c[j / 4] >> (j % 4 * 8));
}

// The arrays of a tensor from a part's first element on.
template <typename P, typename G>
struct Arrays {
  P* p;
  const G* g;
  __nv_bfloat16* copy;
  uint8_t *m, *v;
  float *ms, *vs;
  __device__ __forceinline__ Arrays(const Tensor& t, int64_t block) {
    const int64_t i = block * kBlock;
    p = static_cast<P*>(t.p) + i;
    g = static_cast<const G*>(t.g) + i;
    copy = t.copy ? t.copy + i : nullptr;
    m = static_cast<uint8_t*>(t.m) + i;
    v = static_cast<uint8_t*>(t.v) + i;
    ms = t.ms + block;
    vs = t.vs + block;
  }
};
// Blocks on their way: each warp copies its own next ones into a ring of places in shared memory (cp.async) and
// waits for nobody else's.  Loads to registers of one block a warp are too few bytes in flight for the memory's
// latency (72 M bf16: 242 us as first written, 185 with three places, 154 with four).  Now 100 M fp32 with bf16 gradients and copies
// take 242 us with four, 256 with three, 242 with six; with fp32 gradients 244, and 324 with six, whose memory leaves room for two CTAs.
constexpr int kPlaces = 4;
template <typename P, typename G>
struct Place {
  static constexpr int kG = 2 * kBlock, kP = kG + kBlock * (int)sizeof(G), kScales = kP + kBlock * (int)sizeof(P), kBytes = kScales + 16;
  // by the warp; o: the block's first element in the part
  __device__ __forceinline__ static void fetch(uint32_t at, const Arrays<P, G>& u, uint32_t o, int lane) {
    copy16(at + 16 * lane, (lane < 16 ? u.m + 16 * lane : u.v + 16 * lane - kBlock) + o);
#pragma unroll
    for (int q = 0; q < (int)sizeof(G) / 2; ++q)
      copy16(at + kG + 16 * lane + 512 * q, reinterpret_cast<const char*>(u.g + o) + 16 * lane + 512 * q);
#pragma unroll
    for (int q = 0; q < (int)sizeof(P) / 2; ++q)
      copy16(at + kP + 16 * lane + 512 * q, reinterpret_cast<const char*>(u.p + o) + 16 * lane + 512 * q);
    if (lane < 2)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + kScales + 4 * lane), "l"((lane ? u.vs : u.ms) + o / kBlock) : "memory");
  }
};

// One block's step: p, and codes and scales by a warp; its largest magnitudes are two warp reductions.
template <bool kExact>
__device__ __forceinline__ void step8(Pair (&p)[kPairs], const Pair (&g)[kPairs], uint32_t (&mc)[2], uint32_t (&vc)[2], float& ms, float& vs,
                                      const Step& s, const Rates& r, uint32_t index, uint32_t key, const float* values) {
  Pair m[kPairs], v[kPairs];
  float mt = 0.f;
  uint32_t vt = 0;                                       // as bits: NaN is above infinity
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const Four of_m = decode_m(mc[h]);
    m[2 * h] = of_m.a;
    m[2 * h + 1] = of_m.b;
#pragma unroll
    for (int j = 2 * h; j < 2 * h + 2; ++j) {
      const uint32_t c0 = __byte_perm(vc[h], 0, 0x4440 + j % 2 * 2), c1 = __byte_perm(vc[h], 0, 0x4441 + j % 2 * 2);
      const Pair q = mul2(g[j], both(s.scale));
      // + 0: a zero without a sign
      m[j] = add2(decay_to(mul2(m[j], both(ms)), r.b1, q, r.omb1, r.one), both(0.f));
      v[j] = decay_to(mul2(pair(values[c0], values[c1]), both(vs)), r.b2, mul2(q, q), r.omb2, r.one);
      p[j] = param<kExact>(p[j], m[j], v[j], s, r.eps);
      float lo, hi;
      split(m[j], lo, hi);
      mt = fmaxf(fmaxf(mt, fabsf(lo)), fabsf(hi));
      split(v[j], lo, hi);
      vt = __vimax3_u32(vt, __float_as_uint(lo), __float_as_uint(hi));
    }
  }
  // Scales as bits.  A block's largest exponents are 16 to 254, or its codes are zeros and the scale is
  // 0 or NaN.  An m' that is NaN has a v' that is, or an old scale that was.
  const uint32_t m_top = __reduce_max_sync(0xffffffffu, __float_as_uint(mt)) & 0x7f800000u;
  const uint32_t v_top = __reduce_max_sync(0xffffffffu, vt) & 0x7f800000u;
  constexpr uint32_t kLow = 16u << 23, kRange = 239u << 23;
  const bool usual = m_top - kLow < kRange && v_top - kLow < kRange && !isnan(ms);
  const float mo = __uint_as_float((261u << 23) - m_top), vo = __uint_as_float((258u << 23) - v_top);
  const float old_ms = ms;
  ms = __uint_as_float(m_top - (7u << 23));
  vs = __uint_as_float(v_top - (4u << 23));
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // the first step of mix is that of all four but for the last two bits of an index
    uint32_t first = (index + 128 * h) ^ key;
    first ^= first >> 16;
    uint32_t cm[4], cv[4], of_v[4];
    int y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      uint32_t x = (first ^ j) * kOdd1;
      x = (x ^ (x >> 15)) * kOdd2;
      const Chances chance = chances_of(x);
      float lo, hi;
      split(m[2 * h + j / 2], lo, hi);
      const float mj = j % 2 ? hi : lo;
      split(v[2 * h + j / 2], lo, hi);
      const float vj = j % 2 ? hi : lo;
      cm[j] = encode_m(__fmul_rn(fabsf(mj), mo), chance.m) | (__float_as_uint(mj) & 0x80000000u);
      y[j] = __float_as_int(__fmul_rn(vj, vo));
      of_v[j] = chance.v;
      cv[j] = encode_v(y[j], chance.v);
    }
    // some below the lowest code: that one, but 0 for 0
    if (min(__vimin3_s32(y[0], y[1], y[2]), y[3]) < kLowestCode) {
#pragma unroll
      for (int j = 0; j < 4; ++j) cv[j] = y[j] ? encode_v(max(y[j], kLowestCode), of_v[j]) : 0;
    }
    mc[h] = bytes4(cm);
    vc[h] = bytes4(cv);
  }
  if (!usual) {
    const bool v_lost = v_top == 0x7f800000u, m_lost = m_top == 0x7f800000u || v_lost || isnan(old_ms);
    if (m_lost || m_top < kLow) {
      ms = m_lost ? NAN : 0.f;
      mc[0] = mc[1] = 0;
    }
    if (v_lost || v_top < kLow) {
      vs = v_lost ? NAN : 0.f;
      vc[0] = vc[1] = 0;
    }
  }
}

// bf16 parameters: as many registers as it likes (124, two CTAs an SM), for the instructions bound it: 72 M in 55
// tensors 139 us, 143 with the registers of two CTAs asked for, 150 of three.  fp32 parameters: three CTAs (100 M with
// copies 242 us, 247 with two).
template <typename P, typename G, bool kExact>
__global__ void __launch_bounds__(kThreads, sizeof(P) == 2 ? 1 : 3) adamw8_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  using Q = Place<P, G>;
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ float values[256];
  values[threadIdx.x] = decode_v(threadIdx.x);
  __syncthreads();
  const Step s = step_of(r);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  unsigned char* mine = ring + warp * (kPlaces * Q::kBytes);
  const uint32_t base = smem_u32(mine);
  Share share(a);
  int of;
  uint32_t block, count;
  while (share.next(a, &of, &block, &count)) {
    const Tensor& t = a.t[of];
    const int64_t n = t.n & INT64_MAX, i0 = (int64_t)block * kBlock;
    const uint32_t size = (uint32_t)min((int64_t)count * kBlock, n - i0);       // elements of the part
    const uint32_t whole = t.n >= 0 ? size / kBlock * kBlock : 0;               // of which copied in blocks
    const uint32_t key = mix(mix(s.key + a.ordinal[of]) + (uint32_t)(i0 >> 32));
    const Arrays<P, G> u(t, block);
    constexpr uint32_t kStep = kWarps * kBlock;
    uint32_t o = warp * kBlock;
#pragma unroll
    for (int q = 0; q < kPlaces; ++q) {
      if (o + q * kStep < whole) Q::fetch(base + q * Q::kBytes, u, o + q * kStep, lane);
      copies_close();
    }
    for (uint32_t place = 0; o < whole; o += kStep) {
      copies_wait<kPlaces - 1>();
      __syncwarp();
      const unsigned char* from = mine + place * Q::kBytes;
      Pair p[kPairs], g[kPairs];
      uint32_t mc[2], vc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        mc[h] = *reinterpret_cast<const uint32_t*>(from + 4 * lane + 128 * h);
        vc[h] = *reinterpret_cast<const uint32_t*>(from + kBlock + 4 * lane + 128 * h);
        const Four y = load4(reinterpret_cast<const G*>(from + Q::kG) + 4 * lane + 128 * h);
        const Four x = load4(reinterpret_cast<const P*>(from + Q::kP) + 4 * lane + 128 * h);
        g[2 * h] = y.a; g[2 * h + 1] = y.b;
        p[2 * h] = x.a; p[2 * h + 1] = x.b;
      }
      const float2 scales = *reinterpret_cast<const float2*>(from + Q::kScales);
      float ms = scales.x, vs = scales.y;
      __syncwarp();
      if (o + kPlaces * kStep < whole) Q::fetch(base + place * Q::kBytes, u, o + kPlaces * kStep, lane);
      copies_close();
      place = place + 1 < kPlaces ? place + 1 : 0;
      const uint32_t e = o + 4 * lane;
      step8<kExact>(p, g, mc, vc, ms, vs, s, r, (uint32_t)i0 + e, key, values);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        store4(u.p + e + 128 * h, p[2 * h], p[2 * h + 1]);
        if (u.copy) store4(u.copy + e + 128 * h, p[2 * h], p[2 * h + 1]);
        *reinterpret_cast<uint32_t*>(u.m + e + 128 * h) = mc[h];
        *reinterpret_cast<uint32_t*>(u.v + e + 128 * h) = vc[h];
      }
      if (lane == 0) {
        u.ms[o / kBlock] = ms;
        u.vs[o / kBlock] = vs;
      }
    }
    copies_wait<0>();
    // blocks that are not whole, or of arrays that start anywhere
    for (; o < size; o += kStep) {
      const int64_t left = size - o;
      Pair p[kPairs], g[kPairs];
      uint32_t mc[2], vc[2];
      float ms = u.ms[o / kBlock], vs = u.vs[o / kBlock];
      load_codes(u.m + o, lane, left, mc);
      load_codes(u.v + o, lane, left, vc);
      load8(u.g + o, lane, left, false, g);
      load8(u.p + o, lane, left, false, p);
      step8<kExact>(p, g, mc, vc, ms, vs, s, r, (uint32_t)i0 + o + 4 * lane, key, values);
      store8(u.p + o, lane, left, false, p);
      if (u.copy) store8(u.copy + o, lane, left, false, p);
      store_codes(u.m + o, lane, left, mc);
      store_codes(u.v + o, lane, left, vc);
      if (lane == 0) {
        u.ms[o / kBlock] = ms;
        u.vs[o / kBlock] = vs;
      }
    }
  }
}

// ---- host --------------------------------------------------------------------

// CTAs of a launch: as many as fit at once, or more of `per` blocks each, which the SMs take as they come: the memory does not serve
// all alike, and 8-bit moments with fp32 parameters are bound by it (100 M with copies: 243 us with 64 blocks each, 312 with
// equal shares for all that fit; 75 M: 184, 191 with 128).  bf16 parameters, bound by instructions, lose less to the CTAs'
// first loads with 128 (72 M in 55 tensors: 139 us, 143 with 96).  32-bit moments want their shares in a row
// (403 M fp32: 1662 us, 1672 by 64 blocks; 72 M bf16: 249, 255).
template <typename P>
unsigned blocks_of_cta(int bits) { return bits == 32 ? 0 : sizeof(P) == 2 ? 128 : 64; }
unsigned grid_of(unsigned blocks, int each, unsigned per) {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return std::max(std::min((blocks + kWarps - 1) / kWarps, (unsigned)(sms * each)), per ? blocks / per : 0);
}
int ctas_of_an_sm(const void* kernel, int smem) {
  int each = 1;
  cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kThreads, smem);
  return std::max(each, 1);
}
template <typename P, typename G, bool kExact>
cudaError_t launch(const Table& a, const Rates& r, int bits, cudaStream_t st) {
  const auto kernel = bits == 8 ? adamw8_kernel<P, G, kExact> : adamw_kernel<P, G, kExact>;
  const int smem = bits == 8 ? kWarps * kPlaces * Place<P, G>::kBytes : 0;
  if (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  static std::atomic<int> known[2];
  int each = known[bits == 8].load(std::memory_order_relaxed);
  if (!each) known[bits == 8].store(each = ctas_of_an_sm(reinterpret_cast<const void*>(kernel), smem), std::memory_order_relaxed);
  kernel<<<grid_of(a.first[a.count], each, blocks_of_cta<P>(bits)), kThreads, smem, st>>>(a, r);
  return cudaGetLastError();
}
// The fast root takes a v below the smallest normal float, whose root is 1.1e-19, for 0: no
// matter while that over sqrt(1 - beta2) is below 2^-24 of eps.
bool small_eps(const Rates& r) { return r.eps * std::sqrt(r.omb2) < 2e-12f; }
template <typename P, typename G>
cudaError_t launch(const Table& a, const Rates& r, int bits, cudaStream_t st) {
  return small_eps(r) ? launch<P, G, true>(a, r, bits, st) : launch<P, G, false>(a, r, bits, st);
}
cudaError_t launch(const Table& a, const Rates& r, const pgc_adamw& s, cudaStream_t st) {
  using H = __nv_bfloat16;
  if (s.param_dtype == PGC_BF16)
    return s.grad_dtype == PGC_BF16 ? launch<H, H>(a, r, s.bits, st) : launch<H, float>(a, r, s.bits, st);
  return s.grad_dtype == PGC_BF16 ? launch<float, H>(a, r, s.bits, st) : launch<float, float>(a, r, s.bits, st);
}

bool fraction(double b) { return b >= 0.0 && b < 1.0; }
bool dtype_ok(int32_t d) { return d == PGC_F32 || d == PGC_BF16; }
// Elements of a tensor at most: the blocks of all tensors of a launch are counted in 32 bits.
constexpr int64_t kMostElements = int64_t(1) << 38;

// Whether all of the addresses are multiples of `bytes`, a power of two.
template <typename... T>
bool multiples(uintptr_t bytes, const T*... p) { return ((reinterpret_cast<uintptr_t>(p) | ...) & (bytes - 1)) == 0; }

int check(const pgc_adamw& s, const pgc_adamw_tensor& t) {
  if (t.n < 0 || t.n > kMostElements) return PGC_EINVAL;
  if (!multiples(s.param_dtype == PGC_BF16 ? 2 : 4, t.param) || !multiples(s.grad_dtype == PGC_BF16 ? 2 : 4, t.grad) ||
      !multiples(2, t.copy) || !multiples(s.bits == 8 ? 1 : 4, t.m, t.v) || !multiples(4, t.m_scale, t.v_scale))
    return PGC_EINVAL;
  if (!t.n || !t.grad) return PGC_OK;
  return !t.param || !t.m || !t.v || (s.bits == 8 && (!t.m_scale || !t.v_scale)) ? PGC_EINVAL : PGC_OK;
}

// 16 bytes of every array at once: with 32-bit moments four elements, so that bf16 may start on 8.
bool at_once(const pgc_adamw& s, const pgc_adamw_tensor& t) {
  const uintptr_t half = s.bits == 32 ? 8 : 16;
  return multiples(s.param_dtype == PGC_BF16 ? half : 16, t.param) && multiples(s.grad_dtype == PGC_BF16 ? half : 16, t.grad) &&
         multiples(8, t.copy) && multiples(16, t.m, t.v);
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" int pgc_adamw_step(const pgc_adamw *s, const pgc_adamw_tensor *tensors, int64_t count, void *stream) {
  if (!s || count < 0 || count > INT32_MAX || (count && !tensors)) return PGC_EINVAL;
  if (!dtype_ok(s->param_dtype) || !dtype_ok(s->grad_dtype) || (s->bits != 8 && s->bits != 32)) return PGC_EINVAL;
  if (!std::isfinite(s->lr) || !std::isfinite(s->eps) || !std::isfinite(s->weight_decay) || s->eps < 0.0 || !fraction(s->beta1) ||
      !fraction(s->beta2))
    return PGC_EINVAL;
  if ((!s->step_at && s->step < 1) || (uintptr_t)s->step_at % 8 || (uintptr_t)s->lr_at % 4 || (uintptr_t)s->grad_scale % 4)
    return PGC_EINVAL;
  for (int64_t i = 0; i < count; ++i)
    if (const int rc = check(*s, tensors[i])) return rc;
  Rates r{};
  r.lr = (float)s->lr; r.decay = (float)s->weight_decay;
  r.lr_at = s->lr_at; r.step_at = s->step_at; r.scale_at = s->grad_scale;
  r.b1 = (float)s->beta1; r.b2 = (float)s->beta2;
  r.omb1 = (float)(1.0 - s->beta1); r.omb2 = (float)(1.0 - s->beta2);
  r.eps = (float)s->eps;
  r.one = 1.f;
  r.log_b1 = (float)std::log(s->beta1); r.log_b2 = (float)std::log(s->beta2);
  const double t = (double)s->step;
  r.size = (float)(s->lr / (1.0 - std::pow(s->beta1, t)));
  r.rc1 = (float)(1.0 / (1.0 - std::pow(s->beta1, t)));
  r.rc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(s->beta2, t)));
  r.keep = (float)(1.0 - s->lr * s->weight_decay);
  r.seed = s->seed; r.step_lo = (uint32_t)s->step;
  Table a;
  a.count = 0;
  a.first[0] = 0;
  for (int64_t i = 0; i <= count; ++i) {
    const bool end = i == count;
    const int64_t blocks = end || !tensors[i].grad ? 0 : (tensors[i].n + kBlock - 1) / kBlock;
    if (a.count && (end || a.count == kMost || a.first[a.count] + blocks > INT32_MAX)) {
      const cudaError_t e = launch(a, r, *s, (cudaStream_t)stream);
      if (e != cudaSuccess) return report_cuda(e);
      a.count = 0;
    }
    if (!blocks) continue;
    const pgc_adamw_tensor& q = tensors[i];
    a.t[a.count] = Tensor{q.param, q.grad, static_cast<__nv_bfloat16*>(q.copy), q.m, q.v, q.m_scale, q.v_scale, at_once(*s, q) ? q.n : q.n | INT64_MIN};
    a.ordinal[a.count] = (uint32_t)i;
    a.first[a.count + 1] = a.first[a.count] + (uint32_t)blocks;
    ++a.count;
  }
  return PGC_OK;
}
