// Losses on rows of logits with their gradients (pgc_token_logprob,
// pgc_token_logprob_grad, pgc_preference_loss, pgc_policy_loss).
//
// A row t holds V logits x; with the temperature tau, m = max x and
// L = log sum_v exp((x_v - m) / tau), the log probability of its target y is
// logp = (x_y - m) / tau - L, and d logp / d x_v = ([v = y] - p_v) / tau with
// p_v = exp((x_v - m) / tau - L).  Every loss here is a function of the rows'
// logp, so its gradient is coef_t ([v = y] - p_v) / tau with coef_t = dloss/dlogp_t.
#include <algorithm>
#include <cmath>

#include "dev_common.cuh"
#include "pgc.h"
#include "pgc_internal.h"

namespace pgc {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

struct Rows {
  const void* x;
  void* g;
  const int32_t* y;
  int64_t T, V, ld, ldg;
  float inv_tau;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ float block_max(float v, float* red) {
  v = warp_max(v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = red[0];
  for (int i = 1; i < kThreads / 32; ++i) v = fmaxf(v, red[i]);
  return v;
}
__device__ float block_sum(float v, float* red) {
  v = warp_sum(v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
  for (int i = 0; i < kThreads / 32; ++i) v += red[i];
  return v;
}
__device__ double block_sum_f64(double v, double* red) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.0;
  for (int i = 0; i < kThreads / 32; ++i) v += red[i];
  return v;
}

// What the calls of one loss hand from kernel to kernel (in the workspace).
struct Head {
  int32_t ticket;     // CTAs of the scalar kernel that have finished
  int32_t bad;        // offsets that fall, or leave [0, T]
};

// One CTA per row: largest logit, log of the sum, target's log probability.
template <typename E>
__global__ void __launch_bounds__(kThreads) row_stats_kernel(Rows a, float* logp, float2* stats, Head* head) {
  __shared__ float red[kThreads / 32];
  const int64_t t = blockIdx.x;
  if (head && t == 0 && threadIdx.x == 0) *head = Head{0, 0};
  const int32_t y = a.y[t];
  if (y < 0) {
    if (threadIdx.x == 0) {
      logp[t] = 0.f;
      stats[t] = make_float2(0.f, 0.f);
    }
    return;
  }
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  float m = -INFINITY;
  for (int64_t v = threadIdx.x; v < a.V; v += kThreads) m = fmaxf(m, to_float(x[v]));
  m = block_max(m, red);
  const float c = a.inv_tau * kLog2e;
  float s = 0.f;
  for (int64_t v = threadIdx.x; v < a.V; v += kThreads) s += exp2f((to_float(x[v]) - m) * c);
  s = block_sum(s, red);
  if (threadIdx.x == 0) {
    const float L = logf(s);
    logp[t] = y < a.V ? (to_float(x[y]) - m) * a.inv_tau - L : NAN;
    stats[t] = make_float2(m, L);
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) row_grad_kernel(Rows a, const float* coef, const float2* stats,
                                                            const Head* head) {
  const int64_t t = blockIdx.x;
  const int32_t y = a.y[t];
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const bool bad = head && head->bad;
  if (y < 0 && !bad) {
    for (int64_t v = threadIdx.x; v < a.V; v += kThreads) put(g + v, 0.f);
    return;
  }
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  const float k = (bad || y >= a.V ? NAN : coef[t]) * a.inv_tau;
  const float2 st = bad ? make_float2(0.f, 0.f) : stats[t];
  const float c = a.inv_tau * kLog2e, l2 = st.y * kLog2e;
  for (int64_t v = threadIdx.x; v < a.V; v += kThreads) {
    const float p = exp2f((to_float(x[v]) - st.x) * c - l2);
    put(g + v, k == 0.f ? 0.f : k * ((v == y ? 1.f : 0.f) - p));
  }
}

// ---- preference ------------------------------------------------------------

struct Pref {
  int kind, average;
  int64_t pairs, T;
  const int32_t* off;
  const int32_t* y;
  const float* ref;
  const float* logp;    // [T]
  float beta, margin, smoothing, scale;
  float* coef;          // [T]
  float* seq;           // [pairs][2] out
  double* pair_loss;    // [pairs]
  float* loss;
  Head* head;
};

// loss and its derivative of one pair's gap of log ratios
__device__ double pref_loss(const Pref& a, double gap, double* slope) {
  const double beta = a.beta, e = a.smoothing;
  gap -= (double)a.margin / beta;
  const double h = beta * gap;
  if (a.kind == PGC_PREF_SIGMOID) {
    const double soft = log1p(exp(-fabs(h)));
    *slope = beta * (1.0 / (1.0 + exp(-h)) - (1.0 - e));
    return (1.0 - e) * (soft + fmax(-h, 0.0)) + e * (soft + fmax(h, 0.0));
  }
  if (a.kind == PGC_PREF_HINGE) {
    *slope = beta * ((h > -1.0 ? e : 0.0) - (h < 1.0 ? 1.0 - e : 0.0));
    return (1.0 - e) * fmax(1.0 - h, 0.0) + e * fmax(1.0 + h, 0.0);
  }
  const double up = gap - 0.5 / beta, down = gap + 0.5 / beta;
  *slope = 2.0 * ((1.0 - e) * up + e * down);
  return (1.0 - e) * up * up + e * down * down;
}

__global__ void __launch_bounds__(kThreads) pair_kernel(Pref a) {
  __shared__ double red[kThreads / 32];
  __shared__ int last;
  const int64_t i = blockIdx.x;
  if (i < a.pairs) {
    int64_t at[3];
    bool bad = false;
    for (int j = 0; j < 3; ++j) {
      at[j] = a.off[2 * i + j];
      bad |= at[j] < 0 || at[j] > a.T || (j && at[j] < at[j - 1]);
    }
    double score[2] = {0.0, 0.0}, n[2] = {0.0, 0.0};
    if (!bad)
      for (int j = 0; j < 2; ++j) {
        double s = 0.0, m = 0.0;
        for (int64_t t = at[j] + threadIdx.x; t < at[j + 1]; t += kThreads)
          if (a.y[t] >= 0) {
            s += a.logp[t];
            m += 1.0;
          }
        n[j] = fmax(block_sum_f64(m, red), 1.0);
        score[j] = block_sum_f64(s, red) / (a.average ? n[j] : 1.0);
      }
    double gap = score[0] - score[1];
    if (a.ref) gap -= (double)a.ref[2 * i] - (double)a.ref[2 * i + 1];
    double slope;
    const double loss = pref_loss(a, gap, &slope);
    slope *= (double)a.scale / (double)a.pairs;
    if (!bad)
      for (int j = 0; j < 2; ++j) {
        const float c = (float)((j ? -slope : slope) / (a.average ? n[j] : 1.0));
        for (int64_t t = at[j] + threadIdx.x; t < at[j + 1]; t += kThreads) a.coef[t] = c;
      }
    if (threadIdx.x == 0) {
      a.seq[2 * i] = bad ? NAN : (float)score[0];
      a.seq[2 * i + 1] = bad ? NAN : (float)score[1];
      a.pair_loss[i] = loss;
      if (bad) atomicOr(&a.head->bad, 1);
    }
  }
  // rows outside every sequence
  if (i == 0) {
    const int64_t end = a.pairs ? min((int64_t)max(a.off[0], 0), a.T) : a.T;
    for (int64_t t = threadIdx.x; t < end; t += kThreads) a.coef[t] = 0.f;
  }
  if (a.pairs && i == a.pairs - 1)
    for (int64_t t = max(a.off[2 * a.pairs], 0) + (int64_t)threadIdx.x; t < a.T; t += kThreads) a.coef[t] = 0.f;
  __syncthreads();
  if (threadIdx.x == 0) last = atomic_add_acq_rel(&a.head->ticket, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (!last) return;
  double s = 0.0;
  for (int64_t j = threadIdx.x; j < a.pairs; j += kThreads) s += __ldcg(a.pair_loss + j);
  s = block_sum_f64(s, red);
  if (threadIdx.x == 0) {
    const bool bad = *(volatile int32_t*)&a.head->bad != 0;
    *a.loss = bad ? NAN : a.pairs ? (float)(s * a.scale / (double)a.pairs) : 0.f;
  }
}

// ---- policy ------------------------------------------------------------------

struct Policy {
  int reduction;
  int64_t T, S;
  const int32_t* off;
  const int32_t* y;
  const float *old_logp, *ref_logp, *advantage;
  const float* logp;
  float low, high, kl, scale;
  float* coef;          // [T]
  int32_t* count;       // [grid of the count kernel]: rows with a target, or sequences that have one
  int counts;
  float* share;         // [T]: 1 / rows with a target in the row's sequence
  double* part;         // [grid][3]
  float *loss, *terms;
  Head* head;
};

// Rows with a target (tokens), or sequences with one and 1 / their rows (sequences).
__global__ void __launch_bounds__(kThreads) count_kernel(Policy a) {
  __shared__ double red[kThreads / 32];
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.head = Head{0, 0};
  double total = 0.0;
  if (a.reduction == PGC_MEAN_SEQUENCES) {
    for (int64_t s = blockIdx.x; s < a.S; s += gridDim.x) {
      const int64_t lo = a.off[s], hi = a.off[s + 1];
      const bool bad = lo < 0 || hi < lo || hi > a.T;
      double n = 0.0;
      if (!bad)
        for (int64_t t = lo + threadIdx.x; t < hi; t += kThreads) n += a.y[t] >= 0;
      n = block_sum_f64(n, red);
      if (n > 0.0) total += 1.0;
      if (!bad)
        for (int64_t t = lo + threadIdx.x; t < hi; t += kThreads) a.share[t] = (float)(1.0 / fmax(n, 1.0));
      if (bad) total = NAN;
    }
    if (blockIdx.x == 0) {
      const int64_t end = a.S ? min((int64_t)max(a.off[0], 0), a.T) : a.T;
      for (int64_t t = threadIdx.x; t < end; t += kThreads) a.share[t] = 0.f;
      if (a.S)
        for (int64_t t = max(a.off[a.S], 0) + (int64_t)threadIdx.x; t < a.T; t += kThreads) a.share[t] = 0.f;
    }
  } else {
    for (int64_t t = blockIdx.x * (int64_t)kThreads + threadIdx.x; t < a.T; t += gridDim.x * (int64_t)kThreads)
      total += a.y[t] >= 0;
    total = block_sum_f64(total, red);
  }
  if (threadIdx.x == 0) a.count[blockIdx.x] = total >= 0.0 ? (int32_t)total : -1;
}

__global__ void __launch_bounds__(kThreads) policy_kernel(Policy a) {
  __shared__ double red[kThreads / 32];
  __shared__ int last;
  double n = 0.0;
  bool bad = false;
  for (int i = 0; i < a.counts; ++i) {
    bad |= a.count[i] < 0;
    n += a.count[i];
  }
  const float w0 = a.reduction == PGC_SUM ? 1.f : (float)(1.0 / fmax(n, 1.0));
  double term = 0.0, klsum = 0.0, clipped = 0.0;
  for (int64_t t = blockIdx.x * (int64_t)kThreads + threadIdx.x; t < a.T; t += gridDim.x * (int64_t)kThreads) {
    if (a.y[t] < 0 || bad) {
      a.coef[t] = bad ? NAN : 0.f;
      continue;
    }
    const float w = a.reduction == PGC_MEAN_SEQUENCES ? w0 * a.share[t] : w0;
    if (w == 0.f) {
      a.coef[t] = 0.f;
      continue;
    }
    const float lp = a.logp[t], A = a.advantage[t];
    const float r = expf(lp - a.old_logp[t]);
    const float rc = fminf(fmaxf(r, 1.f - a.low), 1.f + a.high);
    // the smaller product; an advantage of zero takes nothing of a ratio that overflowed
    const bool free = !(r * A > rc * A);
    const float f = A == 0.f && !isnan(r) ? 0.f : free ? -r * A : -rc * A;
    float slope = free ? f : 0.f;
    term += (double)w * f;
    clipped += free ? 0.0 : (double)w;
    if (a.ref_logp) {
      const float away = a.ref_logp[t] - lp, ex = expf(away);
      klsum += (double)w * (isinf(ex) ? ex : ex - away - 1.f);
      if (a.kl != 0.f) slope += a.kl * (1.f - ex);
    }
    a.coef[t] = a.scale * w * slope;
  }
  term = block_sum_f64(term, red);
  klsum = block_sum_f64(klsum, red);
  clipped = block_sum_f64(clipped, red);
  if (threadIdx.x == 0) {
    a.part[3 * blockIdx.x] = term;
    a.part[3 * blockIdx.x + 1] = klsum;
    a.part[3 * blockIdx.x + 2] = clipped;
    if (bad) atomicOr(&a.head->bad, 1);
    last = atomic_add_acq_rel(&a.head->ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last || threadIdx.x) return;
  double s[3] = {0.0, 0.0, 0.0};
  for (int i = 0; i < (int)gridDim.x; ++i)
    for (int j = 0; j < 3; ++j) s[j] += __ldcg(a.part + 3 * i + j);
  for (int j = 0; j < 3; ++j) a.terms[j] = bad ? NAN : (float)s[j];
  *a.loss = bad ? NAN : (float)((double)a.scale * (s[0] + (a.kl != 0.f ? (double)a.kl * s[1] : 0.0)));
}

// ---- host --------------------------------------------------------------------

// 0, or why the rows cannot be taken
int check_rows(const pgc_logits* z, bool grad_required) {
  if (!z) return PGC_EINVAL;
  if (z->dtype != PGC_F32 && z->dtype != PGC_BF16) return PGC_EINVAL;
  if (z->rows < 0 || z->rows > INT32_MAX || z->classes < 1 || z->classes > INT32_MAX) return PGC_EINVAL;
  if (!(z->temperature > 0.f) || !std::isfinite(z->temperature) || !std::isfinite(1.f / z->temperature)) return PGC_EINVAL;
  const uintptr_t size = z->dtype == PGC_BF16 ? 2 : 4;
  const int64_t far = int64_t(1) << 31;
  if (z->ld < z->classes || z->ld > far) return PGC_EINVAL;
  if (z->grad && (z->grad_ld < z->classes || z->grad_ld > far)) return PGC_EINVAL;
  if (z->grad == z->x && z->grad && z->grad_ld != z->ld) return PGC_EINVAL;
  if (z->rows > 0 && (!z->x || !z->target || (grad_required && !z->grad))) return PGC_EINVAL;
  if ((uintptr_t)z->x % size || (uintptr_t)z->grad % size || (uintptr_t)z->target % 4) return PGC_EINVAL;
  return PGC_OK;
}

Rows rows_of(const pgc_logits* z) {
  return Rows{z->x, z->grad, z->target, z->rows, z->classes, z->ld, z->grad_ld, 1.f / z->temperature};
}

cudaError_t launch_stats(const pgc_logits* z, float* logp, float2* stats, Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  const Rows a = rows_of(z);
  if (z->dtype == PGC_BF16)
    row_stats_kernel<__nv_bfloat16><<<(unsigned)z->rows, kThreads, 0, st>>>(a, logp, stats, head);
  else
    row_stats_kernel<float><<<(unsigned)z->rows, kThreads, 0, st>>>(a, logp, stats, head);
  return cudaGetLastError();
}

cudaError_t launch_grad(const pgc_logits* z, const float* coef, const float2* stats, const Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  const Rows a = rows_of(z);
  if (z->dtype == PGC_BF16)
    row_grad_kernel<__nv_bfloat16><<<(unsigned)z->rows, kThreads, 0, st>>>(a, coef, stats, head);
  else
    row_grad_kernel<float><<<(unsigned)z->rows, kThreads, 0, st>>>(a, coef, stats, head);
  return cudaGetLastError();
}

constexpr int kMaxParts = 1024;       // CTAs of the kernels that leave partial sums

// Layout of the workspace (bytes): head, counts [kMaxParts], partial sums
// [max(3 kMaxParts, sequences)] of 8 bytes, stats [rows], logp [rows], coef [rows], share [rows].
struct Work {
  Head* head;
  int32_t* count;
  double* part;
  float2* stats;
  float *logp, *coef, *share;
};
constexpr int64_t kHeadBytes = 256, kCountBytes = kMaxParts * 4;
int64_t part_bytes(int64_t sequences) { return 8 * std::max<int64_t>(3 * kMaxParts, sequences); }
int64_t work_bytes(int64_t rows, int64_t sequences) {
  return kHeadBytes + kCountBytes + part_bytes(sequences) + rows * 20;
}
Work work_at(void* ws, int64_t rows, int64_t sequences) {
  char* p = static_cast<char*>(ws);
  Work w;
  w.head = reinterpret_cast<Head*>(p);
  p += kHeadBytes;
  w.count = reinterpret_cast<int32_t*>(p);
  p += kCountBytes;
  w.part = reinterpret_cast<double*>(p);
  p += part_bytes(sequences);
  w.stats = reinterpret_cast<float2*>(p);
  w.logp = reinterpret_cast<float*>(p + 8 * rows);
  w.coef = w.logp + rows;
  w.share = w.coef + rows;
  return w;
}
int check_work(const void* ws, int64_t bytes, int64_t rows, int64_t sequences) {
  if (!ws || (uintptr_t)ws % 16) return PGC_EINVAL;
  return bytes < work_bytes(rows, sequences) ? PGC_ESCRATCH : PGC_OK;
}
bool finite_all(std::initializer_list<float> v) {
  return std::all_of(v.begin(), v.end(), [](float f) { return std::isfinite(f); });
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_loss_workspace(int64_t rows, int64_t sequences, int64_t *bytes) {
  if (!bytes || rows < 0 || rows > INT32_MAX || sequences < 0 || sequences > INT32_MAX) return PGC_EINVAL;
  *bytes = work_bytes(rows, sequences);
  return PGC_OK;
}

int pgc_token_logprob(const pgc_logits *z, float *logp, float *stats, void *stream) {
  int rc = check_rows(z, false);
  if (rc) return rc;
  if (z->rows && (!logp || !stats)) return PGC_EINVAL;
  if ((uintptr_t)logp % 4 || (uintptr_t)stats % 8) return PGC_EINVAL;
  return report_cuda(launch_stats(z, logp, reinterpret_cast<float2*>(stats), nullptr, (cudaStream_t)stream));
}

int pgc_token_logprob_grad(const pgc_logits *z, const float *stats, const float *dlogp, void *stream) {
  int rc = check_rows(z, true);
  if (rc) return rc;
  if (z->rows && (!dlogp || !stats)) return PGC_EINVAL;
  if ((uintptr_t)dlogp % 4 || (uintptr_t)stats % 8) return PGC_EINVAL;
  return report_cuda(launch_grad(z, dlogp, reinterpret_cast<const float2*>(stats), nullptr, (cudaStream_t)stream));
}

int pgc_preference_loss(const pgc_logits *z, int32_t kind, int64_t pairs, const int32_t *offsets, const float *ref_logp,
                        float beta, float margin, float smoothing, int32_t average, float scale, float *loss,
                        float *logp, void *workspace, int64_t workspace_bytes, void *stream) {
  int rc = check_rows(z, false);
  if (rc) return rc;
  if (kind != PGC_PREF_SIGMOID && kind != PGC_PREF_HINGE && kind != PGC_PREF_SQUARED) return PGC_EINVAL;
  if (pairs < 0 || pairs > INT32_MAX / 2 || !offsets || !loss || (pairs && !logp)) return PGC_EINVAL;
  if (!finite_all({beta, margin, smoothing, scale}) || !(beta > 0.f) || smoothing < 0.f || smoothing > 1.f) return PGC_EINVAL;
  if ((uintptr_t)offsets % 4 || (uintptr_t)ref_logp % 4 || (uintptr_t)loss % 4 || (uintptr_t)logp % 4) return PGC_EINVAL;
  rc = check_work(workspace, workspace_bytes, z->rows, 2 * pairs);
  if (rc) return rc;
  const Work w = work_at(workspace, z->rows, 2 * pairs);
  const cudaStream_t st = (cudaStream_t)stream;
  cudaError_t e = z->rows ? launch_stats(z, w.logp, w.stats, w.head, st)
                          : cudaMemsetAsync(w.head, 0, sizeof(Head), st);
  if (e != cudaSuccess) return report_cuda(e);
  Pref a{kind, average, pairs, z->rows, offsets, z->target, ref_logp, w.logp, beta, margin, smoothing, scale,
         w.coef, logp, w.part, loss, w.head};
  pair_kernel<<<(unsigned)std::max<int64_t>(pairs, 1), kThreads, 0, st>>>(a);
  e = cudaGetLastError();
  if (e == cudaSuccess && z->grad) e = launch_grad(z, w.coef, w.stats, w.head, st);
  return report_cuda(e);
}

int pgc_policy_loss(const pgc_logits *z, int32_t reduction, int64_t sequences, const int32_t *offsets,
                    const float *old_logp, const float *advantage, const float *ref_logp, float clip_low,
                    float clip_high, float kl, float scale, float *loss, float *terms, float *logp, void *workspace,
                    int64_t workspace_bytes, void *stream) {
  int rc = check_rows(z, false);
  if (rc) return rc;
  if (reduction != PGC_MEAN_TOKENS && reduction != PGC_MEAN_SEQUENCES && reduction != PGC_SUM) return PGC_EINVAL;
  if (reduction != PGC_MEAN_SEQUENCES) sequences = 0;
  if (sequences < 0 || sequences > INT32_MAX || (reduction == PGC_MEAN_SEQUENCES && !offsets)) return PGC_EINVAL;
  if (!finite_all({clip_low, clip_high, kl, scale}) || clip_low < 0.f || clip_low > 1.f || clip_high < 0.f) return PGC_EINVAL;
  if (!loss || !terms || (kl != 0.f && z->rows && !ref_logp)) return PGC_EINVAL;
  if (z->rows && (!old_logp || !advantage || !logp)) return PGC_EINVAL;
  for (const void* p : {(const void*)offsets, (const void*)old_logp, (const void*)advantage, (const void*)ref_logp,
                        (const void*)loss, (const void*)terms, (const void*)logp})
    if ((uintptr_t)p % 4) return PGC_EINVAL;
  rc = check_work(workspace, workspace_bytes, z->rows, sequences);
  if (rc) return rc;
  const Work w = work_at(workspace, z->rows, sequences);
  const cudaStream_t st = (cudaStream_t)stream;
  Policy a{reduction, z->rows, sequences, offsets, z->target, old_logp, ref_logp, advantage, logp, clip_low, clip_high,
           kl, scale, w.coef, w.count, 0, w.share, w.part, loss, terms, w.head};
  const int64_t units = reduction == PGC_MEAN_SEQUENCES ? sequences : (z->rows + kThreads - 1) / kThreads;
  a.counts = (int)std::min<int64_t>(std::max<int64_t>(units, 1), 64);
  count_kernel<<<a.counts, kThreads, 0, st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) e = launch_stats(z, logp, w.stats, nullptr, st);
  if (e != cudaSuccess) return report_cuda(e);
  const int grid = (int)std::min<int64_t>(std::max<int64_t>((z->rows + kThreads - 1) / kThreads, 1), kMaxParts);
  policy_kernel<<<grid, kThreads, 0, st>>>(a);
  e = cudaGetLastError();
  if (e == cudaSuccess && z->grad) e = launch_grad(z, w.coef, w.stats, w.head, st);
  return report_cuda(e);
}

}  // extern "C"
