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

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kBlock = 256;           // elements with one scale
constexpr int kUnit = 2048;           // elements a CTA takes at once: a block per warp

struct Tensor {
  void* p;
  const void* g;
  __nv_bfloat16* copy;
  void *m, *v;
  float *ms, *vs;
  int64_t n;
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

template <typename E>
__device__ __forceinline__ float grad_at(const Tensor& t, int64_t i, const Step& s) {
  return __fmul_rn(Elem<E>::get(static_cast<const E*>(t.g) + i), s.scale);
}
// Products and sums are rounded one by one, in this order, whatever kernel: the codes of a step are
// then the same wherever it is computed.
__device__ __forceinline__ float decay_to(float old, float keep, float now, float share) {
  return __fadd_rn(__fmul_rn(old, keep), __fmul_rn(now, share));
}
__device__ __forceinline__ float param(float p, float m, float v, const Step& s, float eps) {
  return p * s.keep - s.size * m / (sqrtf(v) * s.rc2 + eps);
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

template <typename P, typename G>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  const Step s = step_of(r);
  const int at = tensor_of(a, blockIdx.x);
  const Tensor& t = a.t[at];
  const int64_t base = (int64_t)(blockIdx.x - a.first[at]) * kUnit;
  for (int64_t i = base + threadIdx.x; i < min(base + kUnit, t.n); i += kThreads) {
    const float g = grad_at<G>(t, i, s);
    float* m = static_cast<float*>(t.m) + i;
    float* v = static_cast<float*>(t.v) + i;
    *m = decay_to(*m, r.b1, g, r.omb1);
    *v = decay_to(*v, r.b2, __fmul_rn(g, g), r.omb2);
    P* p = static_cast<P*>(t.p) + i;
    const float q = param(Elem<P>::get(p), *m, *v, s, r.eps);
    Elem<P>::put(p, q);
    if (t.copy) Elem<__nv_bfloat16>::put(t.copy + i, q);
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
__device__ __forceinline__ float decode_m(uint32_t c, float scale) {
  // exponent and fraction in the place of a float's, whose exponents start 2^-120 lower
  const float f = __uint_as_float((c & 0x7f) << 20) * __uint_as_float(247u << 23);
  return __fmul_rn(c & 0x80 ? -f : f, scale);
}
__device__ __forceinline__ float decode_v(uint32_t c, float scale) {
  const float f = __uint_as_float(c >= 127 ? (c + 1857) << 19 : c ? (c + 865) << 20 : 0);
  return __fmul_rn(f, scale);
}
// y = |m| / scale, below 2^8; chance: 16 bits.  Twenty bits below the code's last place decide.
__device__ __forceinline__ uint32_t encode_m(float y, bool negative, uint32_t chance) {
  const uint32_t w = y >= 0x1p-6f ? __float_as_uint(y) - (120u << 23) : (uint32_t)(int)(y * 0x1p29f);
  return ((w + (chance << 4) + 8) >> 20) | (negative ? 0x80 : 0);
}
__device__ __forceinline__ uint32_t encode_v(float y, uint32_t chance) {
  const uint32_t b = __float_as_uint(y);
  if (y >= 0x1p-3f) return ((b + (chance << 3) + 4) >> 19) - 1857;
  const int low = (int)((b + (chance << 4) + 8) >> 20) - 865;
  return y > 0.f ? max(low, 1) : 0;
}

// A warp per block, elements 32 apart in its lanes.
template <typename P, typename G>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ Table a, const __grid_constant__ Rates r) {
  const Step s = step_of(r);
  const int at = tensor_of(a, blockIdx.x), lane = threadIdx.x % 32;
  const Tensor& t = a.t[at];
  const int64_t base = (int64_t)(blockIdx.x - a.first[at]) * kUnit + threadIdx.x / 32 * kBlock;
  if (base >= t.n) return;
  const int64_t block = base / kBlock;
  uint8_t* mc = static_cast<uint8_t*>(t.m);
  uint8_t* vc = static_cast<uint8_t*>(t.v);
  const float ms = t.ms[block], vs = t.vs[block];
  constexpr int R = kBlock / 32;
  float m[R], v[R];
  uint32_t mt = 0, vt = 0;
  for (int j = 0; j < R; ++j) {
    const int64_t i = base + lane + 32 * j;
    m[j] = v[j] = 0.f;
    if (i >= t.n) continue;
    const float g = grad_at<G>(t, i, s);
    m[j] = decay_to(decode_m(mc[i], ms), r.b1, g, r.omb1);
    v[j] = decay_to(decode_v(vc[i], vs), r.b2, __fmul_rn(g, g), r.omb2);
    P* p = static_cast<P*>(t.p) + i;
    const float q = param(Elem<P>::get(p), m[j], v[j], s, r.eps);
    Elem<P>::put(p, q);
    if (t.copy) Elem<__nv_bfloat16>::put(t.copy + i, q);
    mt = max(mt, __float_as_uint(fabsf(m[j])));
    vt = max(vt, __float_as_uint(fabsf(v[j])));
  }
  mt = __reduce_max_sync(0xffffffffu, mt);
  vt = __reduce_max_sync(0xffffffffu, vt);
  float mo, vo;
  const float ms1 = scale_of(mt, 7, &mo), vs1 = scale_of(vt, 4, &vo);
  if (lane == 0) {
    t.ms[block] = ms1;
    t.vs[block] = vs1;
  }
  const uint32_t key = mix(mix(s.key + a.ordinal[at]) + (uint32_t)(base >> 32));
  for (int j = 0; j < R; ++j) {
    const int64_t i = base + lane + 32 * j;
    if (i >= t.n) continue;
    const uint32_t h = mix((uint32_t)i ^ key);
    mc[i] = mo > 0.f ? encode_m(__fmul_rn(fabsf(m[j]), mo), m[j] < 0.f, h & 0xffff) : 0;
    vc[i] = vo > 0.f ? encode_v(__fmul_rn(v[j], vo), h >> 16) : 0;
  }
}

// ---- host --------------------------------------------------------------------

template <typename P, typename G>
cudaError_t launch(const Table& a, const Rates& r, int bits, cudaStream_t st) {
  const unsigned grid = a.first[a.count];
  if (bits == 8) adamw8_kernel<P, G><<<grid, kThreads, 0, st>>>(a, r);
  else adamw_kernel<P, G><<<grid, kThreads, 0, st>>>(a, r);
  return cudaGetLastError();
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
  for (int64_t i = 0; i <= count; ++i) {
    const bool end = i == count;
    const int64_t units = end || !tensors[i].grad ? 0 : (tensors[i].n + kUnit - 1) / kUnit;
    if (a.count && (end || a.count == kMost || a.first[a.count] + units > INT32_MAX)) {
      const cudaError_t e = launch(a, r, *s, (cudaStream_t)stream);
      if (e != cudaSuccess) return report_cuda(e);
      a.count = 0;
    }
    if (!units) continue;
    const pgc_adamw_tensor& q = tensors[i];
    a.t[a.count] = Tensor{q.param, q.grad, static_cast<__nv_bfloat16*>(q.copy), q.m, q.v, q.m_scale, q.v_scale, q.n};
    a.ordinal[a.count] = (uint32_t)i;
    a.first[a.count + 1] = a.first[a.count] + (uint32_t)units;
    ++a.count;
  }
  return PGC_OK;
}
