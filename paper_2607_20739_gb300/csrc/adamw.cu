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
  uint32_t seed, step_lo;
};
constexpr int kMost = 240;            // tensors of a launch: what its arguments have room for
struct Table {
  Tensor t[kMost];
  uint32_t first[kMost + 1];          // units before each
  uint32_t ordinal[kMost];
  int count;
  int per;                            // blocks of a unit, which a CTA takes at once
};

// What every element of a step has in common.
struct Step {
  float size, rc2, keep, scale;
  uint32_t key;                       // of seed and step
};

// 32 bits scattered, one to one: products by odd numbers (digits of square roots) and shifts.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
  h = (h ^ (h >> 16)) * 0x6A09E667u;
  h = (h ^ (h >> 15)) * 0xBB67AE85u;
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

// Products and sums are rounded one by one, in this order, whatever kernel: the codes of a step are
// then the same wherever it is computed.
__device__ __forceinline__ float decay_to(float old, float keep, float now, float share) {
  return __fadd_rn(__fmul_rn(old, keep), __fmul_rn(now, share));
}
// kExact: with so small an eps a v below the smallest normal float still counts.
template <bool kExact>
__device__ __forceinline__ float param(float p, float m, float v, const Step& s, float eps) {
  if (kExact) return p * s.keep - s.size * m / (sqrtf(v) * s.rc2 + eps);
  float root, over;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(root) : "f"(v));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(over) : "f"(fmaf(root, s.rc2, eps)));
  return fmaf(-s.size * m, over, p * s.keep);
}

__device__ __forceinline__ int tensor_of(const Table& a, uint32_t unit) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.first[mid] <= unit) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Four elements at once; eight of a block are a lane's: 4 l .. 4 l + 3 and the same behind the first 128.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float4& v) {
  using H = Elem<__nv_bfloat16>;
  *reinterpret_cast<uint2*>(p) = make_uint2(H::two(pair(v.x, v.y)), H::two(pair(v.z, v.w)));
}
constexpr int kEach = kBlock / 32;
__device__ __forceinline__ int place_of(int lane, int j) { return 4 * lane + j % 4 + j / 4 * 128; }

// A lane's eight elements of the block at p; `all`: all there, and four at once allowed.
template <typename E>
__device__ __forceinline__ void load8(const E* p, int lane, int64_t left, bool all, float (&f)[kEach]) {
  if (all) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float4 v = load4(p + place_of(lane, 4 * h));
      f[4 * h] = v.x; f[4 * h + 1] = v.y; f[4 * h + 2] = v.z; f[4 * h + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < kEach; ++j) f[j] = place_of(lane, j) < left ? Elem<E>::get(p + place_of(lane, j)) : 0.f;
  }
}
template <typename E>
__device__ __forceinline__ void store8(E* p, int lane, int64_t left, bool all, const float (&f)[kEach]) {
  if (all) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      store4(p + place_of(lane, 4 * h), make_float4(f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]));
  } else {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (place_of(lane, j) < left) Elem<E>::put(p + place_of(lane, j), f[j]);
  }
}

template <typename P, typename G, bool kExact>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  const Step s = step_of(r);
  const int lane = threadIdx.x % 32;
  for (uint32_t unit = blockIdx.x; unit < a.first[a.count]; unit += gridDim.x) {
    const int at = tensor_of(a, unit);
    const Tensor& t = a.t[at];
    const int64_t n = t.n & INT64_MAX, blocks = (n + kBlock - 1) / kBlock;
    const int64_t b0 = (int64_t)(unit - a.first[at]) * a.per, b1 = min(b0 + a.per, blocks);
    for (int64_t b = b0 + threadIdx.x / 32; b < b1; b += kWarps) {
      const int64_t i = b * kBlock, left = n - i;
      const bool all = t.n >= 0 && left >= kBlock;
      float p[kEach], g[kEach], m[kEach], v[kEach];
      load8(static_cast<const G*>(t.g) + i, lane, left, all, g);
      load8(static_cast<const float*>(t.m) + i, lane, left, all, m);
      load8(static_cast<const float*>(t.v) + i, lane, left, all, v);
      load8(static_cast<const P*>(t.p) + i, lane, left, all, p);
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const float q = __fmul_rn(g[j], s.scale);
        m[j] = decay_to(m[j], r.b1, q, r.omb1);
        v[j] = decay_to(v[j], r.b2, __fmul_rn(q, q), r.omb2);
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

// The scale of a block whose largest magnitude has the bits `top`, and one over
// it: 2^(exponent - shift).  Below 2^-111 a block stands for zeros; with infinities or NaN it is NaN.
__device__ __forceinline__ float scale_of(uint32_t top, uint32_t shift, float* over) {
  const uint32_t e = top >> 23;
  *over = e >= 16 && e < 255 ? __uint_as_float((254 + shift - e) << 23) : 0.f;
  return e == 255 ? NAN : e >= 16 ? __uint_as_float((e - shift) << 23) : 0.f;
}
// Codes of four elements, and their values before the scale.
__device__ __forceinline__ void decode_m(uint32_t codes, float* f) {
  uint32_t lo, hi;
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(codes));
  const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&lo)), y = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  f[0] = x.x; f[1] = x.y; f[2] = y.x; f[3] = y.y;
}
__device__ __forceinline__ float decode_v(uint32_t c) {
  const uint32_t high = (c << 19) + (1857u << 19), low = (c << 20) + (865u << 20);
  return c ? __uint_as_float(c >= 127 ? high : low) : 0.f;
}
// y = |m| / scale, below 2^8; chance: 16 bits.  Twenty bits below the code's last place
// decide.  Below 2^-6, where codes are 2^-9 apart, y + 2^-6 has the same bits there.
__device__ __forceinline__ uint32_t encode_m(float y, uint32_t chance) {
  const bool normal = y >= 0x1p-6f;
  const uint32_t b = __float_as_uint(normal ? y : __fadd_rz(y, 0x1p-6f));
  return (b + (chance << 4) + (8u - (normal ? 120u << 23 : 121u << 23))) >> 20;
}
// Nineteen or twenty bits below the last place; at least 1, but 0 for 0.
__device__ __forceinline__ uint32_t encode_v(float y, uint32_t chance) {
  const uint32_t b = __float_as_uint(y), up = (chance << 4) + 8;
  const bool high = y >= 0x1p-3f;
  const int c = (int)((b + (high ? up >> 1 : up)) >> (high ? 19 : 20)) - (high ? 1857 : 865);
  return min((uint32_t)max(c, 1), b);
}
__device__ __forceinline__ uint32_t bytes4(const uint32_t* c) {
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
}
// A lane's eight codes of the block at p, four a word.
__device__ __forceinline__ void load_codes(const uint8_t* p, int lane, int64_t left, bool all, uint32_t (&c)[2]) {
  if (all) {
    c[0] = *reinterpret_cast<const uint32_t*>(p + place_of(lane, 0));
    c[1] = *reinterpret_cast<const uint32_t*>(p + place_of(lane, 4));
  } else {
    c[0] = c[1] = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (place_of(lane, j) < left) c[j / 4] |= (uint32_t)p[place_of(lane, j)] << (j % 4 * 8);
  }
}
__device__ __forceinline__ void store_codes(uint8_t* p, int lane, int64_t left, bool all, const uint32_t (&c)[2]) {
  if (all) {
    *reinterpret_cast<uint32_t*>(p + place_of(lane, 0)) = c[0];
    *reinterpret_cast<uint32_t*>(p + place_of(lane, 4)) = c[1];
  } else {
#pragma unroll
    for (int j = 0; j < kEach; ++j)
      if (place_of(lane, j) < left) p[place_of(lane, j)] = (uint8_t)(c[j / 4] >> (j % 4 * 8));
  }
}

// A warp per block: its largest magnitudes are two warp reductions.
template <typename P, typename G, bool kExact>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  const Step s = step_of(r);
  const int lane = threadIdx.x % 32;
  for (uint32_t unit = blockIdx.x; unit < a.first[a.count]; unit += gridDim.x) {
    const int at = tensor_of(a, unit);
    const Tensor& t = a.t[at];
    const int64_t n = t.n & INT64_MAX, blocks = (n + kBlock - 1) / kBlock;
    const int64_t b0 = (int64_t)(unit - a.first[at]) * a.per, b1 = min(b0 + a.per, blocks);
    const uint32_t of_tensor = mix(s.key + a.ordinal[at]);
    for (int64_t b = b0 + threadIdx.x / 32; b < b1; b += kWarps) {
      const int64_t i = b * kBlock, left = n - i;
      const bool all = t.n >= 0 && left >= kBlock;
      uint32_t mc[2], vc[2];
      float p[kEach], g[kEach], m[kEach], v[kEach];
      load_codes(static_cast<const uint8_t*>(t.m) + i, lane, left, all, mc);
      load_codes(static_cast<const uint8_t*>(t.v) + i, lane, left, all, vc);
      load8(static_cast<const G*>(t.g) + i, lane, left, all, g);
      load8(static_cast<const P*>(t.p) + i, lane, left, all, p);
      const float ms = t.ms[b], vs = t.vs[b];
      decode_m(mc[0], m);
      decode_m(mc[1], m + 4);
      uint32_t mt = 0, vt = 0;                               // as bits: NaN is above infinity
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        const float q = __fmul_rn(g[j], s.scale);
        m[j] = decay_to(__fmul_rn(m[j], ms), r.b1, q, r.omb1);
        v[j] = decay_to(__fmul_rn(decode_v(vc[j / 4] >> (j % 4 * 8) & 0xff), vs), r.b2, __fmul_rn(q, q), r.omb2);
        p[j] = param<kExact>(p[j], m[j], v[j], s, r.eps);
        mt = max(mt, __float_as_uint(fabsf(m[j])));
        vt = max(vt, __float_as_uint(v[j]));
      }
      store8(static_cast<P*>(t.p) + i, lane, left, all, p);
      if (t.copy) store8(t.copy + i, lane, left, all, p);
      float mo, vo;
      const float ms1 = scale_of(__reduce_max_sync(0xffffffffu, mt), 7, &mo);
      const float vs1 = scale_of(__reduce_max_sync(0xffffffffu, vt), 4, &vo);
      if (lane == 0) {
        t.ms[b] = ms1;
        t.vs[b] = vs1;
      }
      const uint32_t key = mix(of_tensor + (uint32_t)(i >> 32));
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        uint32_t cm[4], cv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float mj = m[4 * w + j];
          const uint32_t h = mix((uint32_t)(i + place_of(lane, 4 * w + j)) ^ key);
          cm[j] = encode_m(__fmul_rn(fabsf(mj), mo), h & 0xffff) | (mj < 0.f ? 0x80 : 0);
          cv[j] = encode_v(__fmul_rn(v[4 * w + j], vo), h >> 16);
        }
        mc[w] = mo > 0.f ? bytes4(cm) : 0;
        vc[w] = vo > 0.f ? bytes4(cv) : 0;
      }
      store_codes(static_cast<uint8_t*>(t.m) + i, lane, left, all, mc);
      store_codes(static_cast<uint8_t*>(t.v) + i, lane, left, all, vc);
    }
  }
}

// ---- host --------------------------------------------------------------------

// CTAs of a launch at most: as many as the SMs hold at once, so that what a CTA works out once serves many units.
int most_ctas(int each) {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms * each;
}
int ctas_of_an_sm(const void* kernel) {
  int each = 4;
  cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kThreads, 0);
  return std::max(each, 1);
}
template <typename P, typename G, bool kExact>
cudaError_t launch(const Table& a, const Rates& r, int bits, cudaStream_t st) {
  static const int each[2] = {ctas_of_an_sm(reinterpret_cast<const void*>(adamw_kernel<P, G, kExact>)),
                              ctas_of_an_sm(reinterpret_cast<const void*>(adamw8_kernel<P, G, kExact>))};
  const auto kernel = bits == 8 ? adamw8_kernel<P, G, kExact> : adamw_kernel<P, G, kExact>;
  const unsigned grid = std::min<unsigned>(a.first[a.count], (unsigned)most_ctas(each[bits == 8]));
  kernel<<<grid, kThreads, 0, st>>>(a, r);
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
// Elements of a tensor at most: units and blocks of all tensors of a launch are counted in 32 bits.
constexpr int64_t kMostElements = int64_t(1) << 38;

int check(const pgc_adamw& s, const pgc_adamw_tensor& t) {
  if (t.n < 0 || t.n > kMostElements) return PGC_EINVAL;
  const uintptr_t p = s.param_dtype == PGC_BF16 ? 2 : 4, g = s.grad_dtype == PGC_BF16 ? 2 : 4, st = s.bits == 8 ? 1 : 4;
  if ((uintptr_t)t.param % p || (uintptr_t)t.grad % g || (uintptr_t)t.copy % 2 || (uintptr_t)t.m % st || (uintptr_t)t.v % st ||
      (uintptr_t)t.m_scale % 4 || (uintptr_t)t.v_scale % 4)
    return PGC_EINVAL;
  if (!t.n || !t.grad) return PGC_OK;
  return !t.param || !t.m || !t.v || (s.bits == 8 && (!t.m_scale || !t.v_scale)) ? PGC_EINVAL : PGC_OK;
}

bool in_fours(const pgc_adamw& s, const pgc_adamw_tensor& t) {
  const uintptr_t p = s.param_dtype == PGC_BF16 ? 8 : 16, g = s.grad_dtype == PGC_BF16 ? 8 : 16, st = s.bits == 8 ? 4 : 16;
  return (uintptr_t)t.param % p == 0 && (uintptr_t)t.grad % g == 0 && (uintptr_t)t.copy % 8 == 0 && (uintptr_t)t.m % st == 0 &&
         (uintptr_t)t.v % st == 0;
}
constexpr int64_t kManyBlocks = 32768;

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
  // many blocks to a unit, so that its tensor is looked up once for them, but for few elements in all
  int64_t blocks = 0;
  for (int64_t i = 0; i < count; ++i) blocks += tensors[i].grad ? (tensors[i].n + kBlock - 1) / kBlock : 0;
  a.per = blocks >= kManyBlocks ? 4 * kWarps : kWarps;
  for (int64_t i = 0; i <= count; ++i) {
    const bool end = i == count;
    const int64_t units = end || !tensors[i].grad ? 0 : ((tensors[i].n + kBlock - 1) / kBlock + a.per - 1) / a.per;
    if (a.count && (end || a.count == kMost || a.first[a.count] + units > INT32_MAX)) {
      const cudaError_t e = launch(a, r, *s, (cudaStream_t)stream);
      if (e != cudaSuccess) return report_cuda(e);
      a.count = 0;
    }
    if (!units) continue;
    const pgc_adamw_tensor& q = tensors[i];
    a.t[a.count] = Tensor{q.param, q.grad, static_cast<__nv_bfloat16*>(q.copy), q.m, q.v, q.m_scale, q.v_scale, in_fours(*s, q) ? q.n : q.n | INT64_MIN};
    a.ordinal[a.count] = (uint32_t)i;
    a.first[a.count + 1] = a.first[a.count] + (uint32_t)units;
    ++a.count;
  }
  return PGC_OK;
}
