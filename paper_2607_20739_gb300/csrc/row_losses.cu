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

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 4;            // 16-byte pieces a thread has in flight
constexpr int kMaxCluster = 8;

struct Rows {
  const void* x;
  void* g;
  const int32_t* y;
  int64_t T, V, ld, ldg;
  float inv_tau, c;                   // 1 / tau, log2(e) / tau
};

__device__ double block_sum_f64(double v, double* red) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.0;
  for (int i = 0; i < kWarps; ++i) v += red[i];
  return v;
}

// What the calls of one loss hand from kernel to kernel (in the workspace).
struct Head {
  int32_t ticket;     // CTAs of the scalar kernel that have finished
  int32_t bad;        // offsets that fall, or leave [0, T]
};

__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

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

// A row belongs to a warp (G = 32), or to the CTA, or the cluster of CTAs, of
// the group's threads.  Exchanges alternate between two buffers, so that one
// barrier each is enough.
struct Shared {
  float2 part[2][kWarps];
  float2 cta[2][kMaxCluster];
};
template <int G>
__device__ __forceinline__ Online merge(Online o, float c, Shared& sh, int& turn, int rank, int ranks) {
  o = warp_merge(o, c);
  if (G == 32) return o;
  const int lane = threadIdx.x % 32, b = turn++ & 1;
  if (lane == 0) sh.part[b][threadIdx.x / 32] = make_float2(o.m, o.s);
  __syncthreads();
  Online q;
  if (lane < kWarps) {
    q.m = sh.part[b][lane].x;
    q.s = sh.part[b][lane].y;
    q.M = ref_of(q.m, c);
  }
  o = warp_merge(q, c);
  if (ranks == 1) return o;
  if (threadIdx.x < ranks) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&sh.cta[b][rank])), "r"((uint32_t)threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(o.m), "f"(o.s) : "memory");
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  q = Online();
  if (lane < ranks) {
    q.m = sh.cta[b][lane].x;
    q.s = sh.cta[b][lane].y;
    q.M = ref_of(q.m, c);
  }
  return warp_merge(q, c);
}

// The row's largest logit and log sum, for all threads of the group.
template <typename E, int G>
__device__ __forceinline__ float2 row_stats(const E* x, const Slice& s, int tid, float c, Shared& sh, int& turn,
                                            int rank, int ranks) {
  Online o = merge<G>(slice_stats<E, G, kUnroll>(x, s, tid, c), c, sh, turn, rank, ranks);
  if (!is_extreme(o.m, c)) return make_float2(o.m, logf(o.s) - kLn2 * fmaf(o.m, c, -o.M));
  Online q;
  q.M = 0.f;
  for (int v = s.first + tid; v < s.last; v += G) q.s += exp2f((Elem<E>::get(x + v) - o.m) * c);
  q.m = 0.f;
  return make_float2(o.m, logf(merge<G>(q, c, sh, turn, rank, ranks).s));
}

__device__ __forceinline__ float target_logp(float xy, float2 st, const Rows& a) {
  return (xy - st.x) * a.inv_tau - st.y;
}

// One row per group: largest logit, log of the sum, target's log probability.
template <typename E, int G>
__global__ void __launch_bounds__(kThreads) row_stats_kernel(Rows a, float* logp, float2* stats, Head* head) {
  __shared__ Shared sh;
  const int rank = G == 32 ? 0 : cluster_rank(), ranks = G == 32 ? 1 : cluster_ranks();
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x / ranks;
  let_next_start();
  if (head && blockIdx.x == 0 && threadIdx.x == 0) *head = Head{0, 0};
  if (t >= a.T) return;
  const int32_t y = a.y[t];
  if (y < 0) {
    if (tid == 0 && rank == 0) {
      logp[t] = 0.f;
      stats[t] = make_float2(0.f, 0.f);
    }
    return;
  }
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  const float xy = y < a.V ? Elem<E>::get(x + y) : NAN;
  int turn = 0;
  const float2 st = row_stats<E, G>(x, slice_of(x, (int)a.V, rank, ranks), tid, a.c, sh, turn, rank, ranks);
  if (tid == 0 && rank == 0) {
    logp[t] = target_logp(xy, st, a);
    stats[t] = st;
  }
}

template <typename E, int G>
__global__ void __launch_bounds__(kThreads) row_grad_kernel(Rows a, const float* coef, const float2* stats,
                                                            const Head* head) {
  const int rank = G == 32 ? 0 : cluster_rank(), ranks = G == 32 ? 1 : cluster_ranks();
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x / ranks;
  if (t >= a.T) return;
  const int32_t y = a.y[t];
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  const Slice s = slice_of(x, (int)a.V, rank, ranks);
  if (head) wait_for_previous();
  const bool bad = head && head->bad;
  const float k = bad || y >= a.V ? NAN : y < 0 ? 0.f : coef[t];
  if (k == 0.f || isnan(k)) {
    slice_fill<E, G>(g, s.first, s.last, tid, k);
    return;
  }
  const float2 st = stats[t];
  slice_grad<E, G, kUnroll>(x, g, s, tid, row_grad(st.x, st.y, k, a.inv_tau, a.c, y));
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
  __shared__ double red[kWarps];
  __shared__ int last;
  const int64_t i = blockIdx.x;
  let_next_start();
  wait_for_previous();
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
  __shared__ double red[kWarps];
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
  __shared__ double red[kWarps];
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
  const float inv_tau = 1.f / z->temperature;
  return Rows{z->x, z->grad, z->target, z->rows, z->classes, z->ld, z->grad_ld, inv_tau, inv_tau * kLog2e};
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 148;
  return n;
}

// How a call's rows lie on the grid: a warp each (short rows), a CTA each, or
// a cluster each (few long rows).
constexpr int64_t kWarpRowBytes = 4096;
struct Shape {
  bool warp;
  int ranks;
  unsigned grid;
};
Shape shape_of(const pgc_logits* z) {
  const int64_t bytes = z->classes * (z->dtype == PGC_BF16 ? 2 : 4);
  Shape s{bytes <= kWarpRowBytes, 1, 0};
  if (s.warp) {
    s.grid = (unsigned)((z->rows + kWarps - 1) / kWarps);
    return s;
  }
  const int64_t sms = sm_count();
  while (s.ranks < kMaxCluster && z->rows * s.ranks * 2 <= 2 * sms && bytes / (s.ranks * 2) >= kWarpRowBytes) s.ranks *= 2;
  s.grid = (unsigned)(z->rows * s.ranks);
  return s;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), unsigned grid, int ranks, bool pdl, cudaStream_t st, A... args) {
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cfg.attrs = attr;
  if (ranks > 1) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
    attr[cfg.numAttrs].val.clusterDim.x = (unsigned)ranks;
    attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
    ++cfg.numAttrs;
  }
  if (pdl) {
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs].val.programmaticStreamSerializationAllowed = 1;
    ++cfg.numAttrs;
  }
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

cudaError_t launch_stats(const pgc_logits* z, float* logp, float2* stats, Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  const Shape s = shape_of(z);
  const bool half = z->dtype == PGC_BF16;
  return launch(half ? s.warp ? row_stats_kernel<__nv_bfloat16, 32> : row_stats_kernel<__nv_bfloat16, kThreads>
                     : s.warp ? row_stats_kernel<float, 32> : row_stats_kernel<float, kThreads>,
                s.grid, s.ranks, false, st, rows_of(z), logp, stats, head);
}

cudaError_t launch_grad(const pgc_logits* z, const float* coef, const float2* stats, const Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  const Shape s = shape_of(z);
  const bool half = z->dtype == PGC_BF16;
  return launch(half ? s.warp ? row_grad_kernel<__nv_bfloat16, 32> : row_grad_kernel<__nv_bfloat16, kThreads>
                     : s.warp ? row_grad_kernel<float, 32> : row_grad_kernel<float, kThreads>,
                s.grid, s.ranks, head != nullptr, st, rows_of(z), coef, stats, head);
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
  e = launch(pair_kernel, (unsigned)std::max<int64_t>(pairs, 1), 1, true, st, a);
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
