// Token scores (pgc_token_scores, pgc_token_scores_grad): the log probability of
// a row's target, the row's entropy and its k likeliest classes, and the
// gradient of the first two.
//
// With q_v = (x_v - m) / tau - L the log probability of class v (m the largest
// logit, L = log sum_v exp((x_v - m) / tau)) and p = exp q:
//   logp = q_y,   H = -sum_v p_v q_v = L - sum_v e_v z_v / sum_v e_v,  z = (x - m) / tau, e = exp z,
//   d logp / d x_v = ([v = y] - p_v) / tau,   d H / d x_v = -p_v (q_v + H) / tau.
// Every term of H is positive, so nothing cancels.
#include <algorithm>
#include <cmath>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256;
constexpr int kMostTop = 64;

struct Scores {
  const void* x;
  void* g;
  const int32_t* y;           // NULL: every row takes part, without a target
  int64_t T, ld, ldg;
  int32_t V, k;
  float inv_tau;
  float *logp, *entropy, *top_logp;
  int32_t* top;
  float2* stats;
};

__device__ float block_max(float v, float* red) {
  v = warp_max(v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = -INFINITY;
  for (int i = 0; i < kThreads / 32; ++i) v = fmaxf(v, red[i]);
  return v;
}
__device__ float block_add(float v, float* red) {
  v = warp_sum(v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
  for (int i = 0; i < kThreads / 32; ++i) v += red[i];
  return v;
}

// What is left of e z where e has run out: masked classes have z = -inf.
__device__ __forceinline__ float times_log(float e, float z) { return e * fmaxf(z, -1e4f); }

// One CTA per row: the maximum, the sums, then the k best one after another.
template <typename E>
__global__ void __launch_bounds__(kThreads) scores_kernel(Scores a) {
  __shared__ float red[kThreads / 32];
  __shared__ unsigned long long best;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x;
  const int32_t y = a.y ? a.y[t] : 0;
  int32_t* top = a.top + t * a.k;
  float* top_logp = a.top_logp + t * a.k;
  if (y < 0) {
    for (int j = tid; j < a.k; j += kThreads) {
      top[j] = -1;
      top_logp[j] = -INFINITY;
    }
    if (tid == 0) {
      if (a.logp) a.logp[t] = 0.f;
      a.entropy[t] = 0.f;
      a.stats[t] = make_float2(0.f, 0.f);
    }
    return;
  }
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  float m = -INFINITY, s = 0.f, w = 0.f;
  for (unsigned v = tid; v < (unsigned)a.V; v += kThreads) m = fmaxf(m, Elem<E>::get(x + v));
  m = block_max(m, red);
  for (unsigned v = tid; v < (unsigned)a.V; v += kThreads) {
    const float z = (Elem<E>::get(x + v) - m) * a.inv_tau, e = expf(z);
    s += e;
    w -= times_log(e, z);
  }
  s = block_add(s, red);
  w = block_add(w, red);
  const float L = logf(s);
  if (tid == 0) {
    if (a.logp) a.logp[t] = y < a.V ? (Elem<E>::get(x + y) - m) * a.inv_tau - L : NAN;
    a.entropy[t] = L + w / s;
    a.stats[t] = make_float2(m, L);
  }
  unsigned long long before = ~0ull;
  for (int j = 0; j < a.k; ++j) {
    if (tid == 0) best = 0;
    __syncthreads();
    unsigned long long mine = 0;
    for (unsigned v = tid; v < (unsigned)a.V; v += kThreads) {
      const float f = Elem<E>::get(x + v) + 0.f;
      const uint32_t b = __float_as_uint(f);
      const unsigned long long key =
          (unsigned long long)(b ^ ((int32_t)b < 0 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - v);
      if (f > -INFINITY && key < before && key > mine) mine = key;
    }
    atomicMax(&best, mine);
    __syncthreads();
    before = best;
    if (tid == 0) {
      const int32_t at = before ? (int32_t)(0xffffffffu - (uint32_t)before) : -1;
      top[j] = at;
      top_logp[j] = before ? (Elem<E>::get(x + at) - m) * a.inv_tau - L : -INFINITY;
    }
    __syncthreads();
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) scores_grad_kernel(Scores a, const float* dlogp, const float* dentropy) {
  const int64_t t = blockIdx.x;
  const int32_t y = a.y ? a.y[t] : 0;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const float da = dlogp && y >= 0 ? dlogp[t] : 0.f, db = dentropy && y >= 0 ? dentropy[t] : 0.f;
  const float2 st = a.stats[t];
  const float H = db != 0.f ? a.entropy[t] : 0.f;
  float fill = 0.f;
  if (da != 0.f || db != 0.f) fill = isnan(da) || isnan(db) || isnan(st.y) || isnan(H) || (da != 0.f && y >= a.V) ? NAN : 1.f;
  for (unsigned v = threadIdx.x; v < (unsigned)a.V; v += kThreads) {
    float d = fill;
    if (fill == 1.f) {
      const float q = (Elem<E>::get(x + v) - st.x) * a.inv_tau - st.y;
      d = -expf(q) * (da + db * fmaxf(q + H, -1e4f));
      d = (d + (da != 0.f && (int)v == y ? da : 0.f)) * a.inv_tau;
    }
    Elem<E>::put(g + v, d);
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
  return a;
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
  if (z->dtype == PGC_BF16) scores_kernel<__nv_bfloat16><<<(unsigned)z->rows, kThreads, 0, st>>>(a);
  else scores_kernel<float><<<(unsigned)z->rows, kThreads, 0, st>>>(a);
  return report_cuda(cudaGetLastError());
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
  if (z->dtype == PGC_BF16) scores_grad_kernel<__nv_bfloat16><<<(unsigned)z->rows, kThreads, 0, st>>>(a, dlogp, dentropy);
  else scores_grad_kernel<float><<<(unsigned)z->rows, kThreads, 0, st>>>(a, dlogp, dentropy);
  return report_cuda(cudaGetLastError());
}

}  // extern "C"
