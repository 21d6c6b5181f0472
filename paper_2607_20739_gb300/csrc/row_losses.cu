// Losses on rows of logits with their gradients (pgc_token_logprob,
// pgc_token_logprob_grad, pgc_preference_loss, pgc_policy_loss).
//
// A row t holds V logits x; with the temperature tau, m = max x and
// L = log sum_v exp((x_v - m) / tau), the log probability of its target y is
// logp = (x_y - m) / tau - L, and d logp / d x_v = ([v = y] - p_v) / tau with
// p_v = exp((x_v - m) / tau - L).  Every loss here is a function of the rows'
// logp, so its gradient is coef_t ([v = y] - p_v) / tau with coef_t = dloss/dlogp_t.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <initializer_list>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxWarps = 32;
constexpr int kUnroll = 4;            // 16-byte pieces a thread has in flight
constexpr int kMaxCluster = 8;

struct Rows {
  const void* x;
  void* g;
  const int32_t* y;
  int64_t T, ld, ldg;
  int32_t V;
  float inv_tau, c;                   // 1 / tau, log2(e) / tau
};

// The block's sum, in all threads.
__device__ int block_sum(int v, int* red) {
  v = __reduce_add_sync(0xffffffffu, v);
  __syncthreads();
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < (int)blockDim.x / 32; ++i) v += red[i];
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
// A CTA's shared memory may be written by another one of its cluster only once
// it runs: every CTA says so (arrive), and knows it of all of them (wait) before its first store
// to a neighbour.  All threads of the cluster call both, or neither.
__device__ __forceinline__ void cluster_say_started(int ranks) {
  if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait_started(int ranks) {
  if (ranks <= 1) return;
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// A row belongs to a warp (G = 32), or to the CTA, or the cluster of CTAs, of
// the group's threads.  Exchanges alternate between two buffers, so that one
// barrier each is enough.
struct Shared {
  float2 part[2][kMaxWarps];
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
  if (lane < G / 32) {
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
  __syncwarp();
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

// Logarithm of a row's sum at its maximum.
__device__ __forceinline__ float log_sum(const Online& o, float c) { return logf(o.s) - kLn2 * fmaf(o.m, c, -o.M); }

// The row's largest logit and log sum, for all threads of the group, or of the
// cluster, which takes one row only.
template <typename E, int G>
__device__ __forceinline__ float2 row_stats(const E* x, const Slice& s, int tid, float c, Shared& sh, int& turn,
                                            int rank, int ranks) {
  cluster_say_started(ranks);
  Online o = slice_stats<E, G, kUnroll>(x, s, tid, c);
  cluster_wait_started(ranks);
  o = merge<G>(o, c, sh, turn, rank, ranks);
  if (!is_extreme(o.m, c)) return make_float2(o.m, log_sum(o, c));
  Online q;
  q.M = 0.f;
  for (unsigned v = s.first + tid; v < (unsigned)s.last; v += G) q.s += exp2f((Elem<E>::get(x + v) - o.m) * c);
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
  const float2 st = row_stats<E, G>(x, slice_of(x, a.V, rank, ranks), tid, a.c, sh, turn, rank, ranks);
  if (tid == 0 && rank == 0) {
    logp[t] = target_logp(xy, st, a);
    stats[t] = st;
  }
}

// A row's coefficient: 0 where nothing is asked of it, whatever its target, and
// NaN where that is no class.
__device__ __forceinline__ float row_coef(bool bad, int32_t y, int32_t V, const float* coef) {
  if (bad) return NAN;
  const float k = y < 0 ? 0.f : *coef;
  return y >= V && k != 0.f ? NAN : k;
}

// A row, or one of its `parts`, per group: nothing is exchanged between them.
template <typename E, int G>
__global__ void __launch_bounds__(kThreads) row_grad_kernel(Rows a, int parts, const float* coef, const float2* stats,
                                                            const Head* head) {
  const int rank = G == 32 ? 0 : blockIdx.x % parts, ranks = G == 32 ? 1 : parts;
  const int tid = threadIdx.x % G;
  const int64_t t = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x / parts;
  if (t >= a.T) return;
  const int32_t y = a.y[t];
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  const Slice s = slice_of(x, a.V, rank, ranks);
  if (head) wait_for_previous();
  const bool bad = head && head->bad;
  const float k = row_coef(bad, y, a.V, coef + t);
  if (k == 0.f || isnan(k)) {
    slice_fill<E, G>(g, s.first, s.last, tid, k);
    return;
  }
  const float2 st = stats[t];
  slice_grad<E, G, kUnroll>(x, g, s, tid, Elem<E>::get(x + y), row_grad(st.x, st.y, k, a.inv_tau, a.c, y));
}

// ---- short rows ----------------------------------------------------------------
// Rows of up to L R classes in the registers of L lanes, single elements, so
// that a warp has 32 / L rows at once: what a row costs there is its own
// instructions, not its bytes.  (x - m) c serves rows of any range.
template <int L>
__device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
template <int L>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Which element a lane's j-th is: single ones, or (P = 2: bf16 rows of even
// length and pitch that start on 4 bytes) two neighbours, read at once.
template <int L, int P>
__device__ __forceinline__ int short_at(int l, int j) { return P * (l + j / P * L) + j % P; }
// A row's elements of lane l and -inf behind them (throughout, if not taken).
template <typename E, int L, int P, int R>
__device__ __forceinline__ void short_load(const E* x, int l, int V, bool taken, float (&v)[R]) {
#pragma unroll
  for (int j = 0; j < R; j += P) {
    const int e = short_at<L, P>(l, j);
    if (P == 2) {
      uint32_t w = Elem<E>::kLowest;
      if (taken && e < V) w = *reinterpret_cast<const uint32_t*>(x + e);
      v[j] = __uint_as_float(w << 16);
      v[j + P - 1] = __uint_as_float(w & 0xffff0000u);
    } else {
      v[j] = taken && e < V ? Elem<E>::get(x + e) : -INFINITY;
    }
  }
}
// (m, sum) of a row, v becoming 2^((x - m) c).  All lanes of the warp take part.
template <int L, int R>
__device__ __forceinline__ float2 short_exps(float (&v)[R], bool taken, float c) {
  float m = v[0], s = 0.f;
#pragma unroll
  for (int j = 1; j < R; ++j) m = fmaxf(m, v[j]);
  m = group_max<L>(m);
  if (!taken) m = 0.f;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    v[j] = ex2((v[j] - m) * c);
    s += v[j];
  }
  return make_float2(m, group_sum<L>(s));
}
// k ([v = y] - p) / tau of the row, where v times scale is p; 0 or NaN throughout with such a k.
template <typename E, int L, int P, int R>
__device__ __forceinline__ void short_store(E* g, int l, int V, const float (&v)[R], float scale, float k, float inv_tau, int y) {
  const bool fill = k == 0.f || isnan(k), at_once = reinterpret_cast<uintptr_t>(g) % 4 == 0;
  const float at = k * inv_tau;
  auto value = [&](int j, int e) { return fill ? k : fmaf(v[j] * scale, -at, e == y ? at : 0.f); };
#pragma unroll
  for (int j = 0; j < R; j += P) {
    const int e = short_at<L, P>(l, j);
    if (e >= V) continue;
    if constexpr (P == 2) {
      const uint32_t w = Elem<E>::two(pair(value(j, e), value(j + 1, e + 1)));
      if (at_once) {
        *reinterpret_cast<uint32_t*>(g + e) = w;
      } else {
        reinterpret_cast<uint16_t*>(g)[e] = (uint16_t)w;
        reinterpret_cast<uint16_t*>(g)[e + 1] = (uint16_t)(w >> 16);
      }
    } else {
      Elem<E>::put(g + e, value(j, e));
    }
  }
}

template <typename E, int L, int R, int P>
__global__ void __launch_bounds__(kThreads) short_stats_kernel(Rows a, float* logp, float2* stats, Head* head) {
  const int lane = threadIdx.x % 32, l = lane % L;
  const int64_t t = (blockIdx.x * (int64_t)kWarps + threadIdx.x / 32) * (32 / L) + lane / L;
  let_next_start();
  if (head && blockIdx.x == 0 && threadIdx.x == 0) *head = Head{0, 0};
  const int32_t y = t < a.T ? a.y[t] : -1;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  float v[R];
  short_load<E, L, P>(x, l, a.V, y >= 0, v);
  const float xy = y >= 0 ? y < a.V ? Elem<E>::get(x + y) : NAN : 0.f;
  const float2 ms = short_exps<L>(v, y >= 0, a.c);
  if (l || t >= a.T) return;
  const float2 st = y >= 0 ? make_float2(ms.x, logf(ms.y)) : make_float2(0.f, 0.f);
  logp[t] = y >= 0 ? target_logp(xy, st, a) : 0.f;
  stats[t] = st;
}

template <typename E, int L, int R, int P>
__global__ void __launch_bounds__(kThreads) short_grad_kernel(Rows a, const float* coef, const float2* stats, const Head* head) {
  const int lane = threadIdx.x % 32, l = lane % L;
  const int64_t t = (blockIdx.x * (int64_t)kWarps + threadIdx.x / 32) * (32 / L) + lane / L;
  if (t >= a.T) return;
  const int32_t y = a.y[t];
  float v[R];
  short_load<E, L, P>(static_cast<const E*>(a.x) + t * a.ld, l, a.V, y >= 0, v);
  if (head) wait_for_previous();
  const bool bad = head && head->bad;
  const float k = row_coef(bad, y, a.V, coef + t);
  const float2 st = y >= 0 ? stats[t] : make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < R; ++j) v[j] = ex2((v[j] - st.x) * a.c - st.y * kLog2e);
  short_store<E, L, P>(static_cast<E*>(a.g) + t * a.ldg, l, a.V, v, 1.f, k, a.inv_tau, y);
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
  float* pair_loss;     // [pairs]
  float* loss;
  Head* head;
};

// Loss of one pair's gap of log ratios, and its derivative (squared: of the gap
// less margin / beta, which for a small beta only this kind has to hold).  A branch of
// weight 0 takes no part, so that an infinite gap (an answer that the model
// cannot give) has the loss and slope of its limit.
__device__ float pref_loss(const Pref& a, float gap, float* slope) {
  const float beta = a.beta, e = a.smoothing;
  const float h = fmaf(beta, gap, -a.margin);
  auto both = [e](float chosen, float rejected) {      // (1 - e) chosen + e rejected
    return (e < 1.f ? (1.f - e) * chosen : 0.f) + (e > 0.f ? e * rejected : 0.f);
  };
  if (isnan(h)) {
    *slope = h;
    return h;
  }
  if (a.kind == PGC_PREF_SIGMOID) {
    // e sig(h) - (1 - e) sig(-h): both from exp(-|h|), so that the one near 0 keeps its
    // digits (sig(h) - (1 - e) has none left at h = 17, where a pair still moves a little)
    const float t = expf(-fabsf(h)), soft = log1pf(t);
    const float near = 1.f / (1.f + t), far = t / (1.f + t);
    *slope = beta * (e * (h < 0.f ? far : near) - (1.f - e) * (h < 0.f ? near : far));
    return both(soft + fmaxf(-h, 0.f), soft + fmaxf(h, 0.f));
  }
  if (a.kind == PGC_PREF_HINGE) {
    *slope = beta * ((h > -1.f ? e : 0.f) - (h < 1.f ? 1.f - e : 0.f));
    return both(fmaxf(1.f - h, 0.f), fmaxf(1.f + h, 0.f));
  }
  const float up = gap - 0.5f / beta, down = gap + 0.5f / beta;
  *slope = 2.f * both(up, down);
  return both(up * up, down * down);
}

// A pair's scores, loss and coefficients from its rows' log probabilities, by
// a warp (G = 32) or the CTA; the results are in lane 0 of its first warp.  No
// doubles: a few of them take longer than the rest.
struct PairWork {
  Sum red[2][kWarps];
  int count[2][kWarps];
};
template <int G>
__device__ __forceinline__ float2 finish_pair(const Pref& a, int64_t i, const int32_t (&at)[3], PairWork& sh) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  Sum score[2];
  int n[2] = {0, 0};
  for (int64_t t = at[0] + (int64_t)(threadIdx.x % G); t < at[2]; t += G) {
    const int j = t >= at[1];
    const float lp = __ldcg(a.logp + t);
    if (a.y[t] < 0) continue;
    score[0].add(j ? 0.f : lp);
    score[1].add(j ? lp : 0.f);
    n[0] += !j;
    n[1] += j;
  }
  for (int j = 0; j < 2; ++j) {
    for (int o = 16; o > 0; o >>= 1) score[j].add(shuffle_down(score[j], o));
    n[j] = __reduce_add_sync(0xffffffffu, n[j]);
    if (G > 32 && lane == 0) {
      sh.red[j][warp] = score[j];
      sh.count[j][warp] = n[j];
    }
  }
  if (G > 32) {
    __syncthreads();
    if (warp) return make_float2(0.f, 0.f);
    for (int j = 0; j < 2; ++j) {
      score[j] = lane < kWarps ? sh.red[j][lane] : Sum();
      n[j] = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.count[j][lane] : 0);
      for (int o = kWarps / 2; o > 0; o >>= 1) score[j].add(shuffle_down(score[j], o));
    }
  }
  float share[2];
  Sum gap;
  for (int j = 0; j < 2; ++j) {
    share[j] = a.average ? 1.f / (float)max(n[j], 1) : 1.f;
    if (a.average) {
      score[j].s = score[j].value() / (float)max(n[j], 1);
      score[j].e = 0.f;
    }
    if (lane == 0) a.seq[2 * i + j] = score[j].value();
    gap.add(j ? -score[j].s : score[j].s);
    gap.e += j ? -score[j].e : score[j].e;
  }
  if (a.ref) {
    gap.add(-a.ref[2 * i]);
    gap.add(a.ref[2 * i + 1]);
  }
  if (a.kind == PGC_PREF_SQUARED) gap.add(-a.margin / a.beta);
  float slope;
  const float loss = pref_loss(a, gap.value(), &slope);
  if (lane == 0) a.pair_loss[i] = loss;
  slope = slope * a.scale / (float)a.pairs;
  return make_float2(slope * share[0], -slope * share[1]);
}
// The mean of the pairs' losses.
__device__ void finish_loss(const Pref& a, bool bad, PairWork& sh) {
  Sum s;
  for (int64_t j = threadIdx.x; j < a.pairs; j += kThreads) s.add(__ldcg(a.pair_loss + j));
  s = block_sum(s, sh.red[0]);
  if (threadIdx.x == 0) *a.loss = bad ? NAN : a.pairs ? s.value() * a.scale / (float)a.pairs : 0.f;
}

template <int G>
__global__ void __launch_bounds__(kThreads) pair_kernel(Pref a) {
  __shared__ PairWork sh;
  __shared__ float2 shared_coef;
  __shared__ int last;
  const int64_t i = G == 32 ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x;
  const int tid = threadIdx.x % G;
  let_next_start();
  wait_for_previous();
  if (i < a.pairs) {
    const int32_t at[3] = {a.off[2 * i], a.off[2 * i + 1], a.off[2 * i + 2]};
    const bool bad = at[0] < 0 || at[1] < at[0] || at[2] < at[1] || at[2] > a.T;
    if (bad) {
      if (tid == 0) {
        a.seq[2 * i] = a.seq[2 * i + 1] = NAN;
        atomicOr(&a.head->bad, 1);
      }
    } else {
      float2 coef = finish_pair<G>(a, i, at, sh);
      if (G == 32) {
        coef.x = __shfl_sync(0xffffffffu, coef.x, 0);
        coef.y = __shfl_sync(0xffffffffu, coef.y, 0);
      } else {
        if (tid == 0) shared_coef = coef;
        __syncthreads();
        coef = shared_coef;
      }
      for (int64_t t = at[0] + (int64_t)tid; t < at[2]; t += G) a.coef[t] = t < at[1] ? coef.x : coef.y;
    }
  }
  // rows outside every sequence
  if (blockIdx.x == 0) {
    const int64_t end = a.pairs ? min((int64_t)max(a.off[0], 0), a.T) : a.T;
    for (int64_t t = threadIdx.x; t < end; t += kThreads) a.coef[t] = 0.f;
  }
  if (a.pairs && blockIdx.x == gridDim.x - 1)
    for (int64_t t = max(a.off[2 * a.pairs], 0) + (int64_t)threadIdx.x; t < a.T; t += kThreads) a.coef[t] = 0.f;
  __syncthreads();
  if (threadIdx.x == 0) last = atomic_add_acq_rel(&a.head->ticket, 1) == (int)gridDim.x - 1;
  __syncthreads();
  if (last) finish_loss(a, *(volatile int32_t*)&a.head->bad != 0, sh);
}

// ---- policy ------------------------------------------------------------------

struct Policy {
  int reduction;
  int64_t T, S;
  const int32_t* off;
  const int32_t* y;
  const float *old_logp, *ref_logp, *advantage;
  float* logp;
  float low, high, kl, scale;
  int32_t* count;       // [grid of the count kernel]: rows with a target, or sequences that have one
  int counts;
  float* share;         // [T]: 1 / rows with a target in the row's sequence
  float2* part;         // [grid][3]
  float *loss, *terms;
  Head* head;
};

// Rows with a target (tokens), or sequences with one and 1 / their rows (sequences).
__global__ void __launch_bounds__(kThreads) count_kernel(Policy a) {
  __shared__ int red[kWarps];
  let_next_start();
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.head = Head{0, 0};
  int total = 0;
  bool bad = false;
  if (a.reduction == PGC_MEAN_SEQUENCES) {
    // a CTA per sequence, or a warp each where there are more of them than CTAs
    const bool warp = a.S > gridDim.x;
    const int tid = warp ? threadIdx.x % 32 : threadIdx.x, step = warp ? 32 : kThreads;
    const int64_t first = warp ? blockIdx.x * (int64_t)kWarps + threadIdx.x / 32 : blockIdx.x;
    for (int64_t s = first; s < a.S; s += warp ? gridDim.x * (int64_t)kWarps : gridDim.x) {
      const int64_t lo = a.off[s], hi = a.off[s + 1];
      if (lo < 0 || hi < lo || hi > a.T) {
        bad = true;
        continue;
      }
      int n = 0;
      for (int64_t t = lo + tid; t < hi; t += step) n += a.y[t] >= 0;
      n = warp ? __reduce_add_sync(0xffffffffu, n) : block_sum(n, red);
      total += n > 0;
      for (int64_t t = lo + tid; t < hi; t += step) a.share[t] = 1.f / (float)max(n, 1);
    }
    if (warp) {
      total = block_sum(tid == 0 ? total : 0, red);
      bad = __syncthreads_or(bad);
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
    total = block_sum(total, red);
  }
  if (threadIdx.x == 0) a.count[blockIdx.x] = bad ? -1 : total;
}

// A row's inputs besides its logits, read a row ahead (its target two rows).
struct RowIn {
  int32_t y;
  float xy, advantage, old, ref, share;
};
template <typename E>
__device__ __forceinline__ RowIn row_in(const Rows& a, const Policy& p, int64_t t, int32_t y) {
  RowIn r{y, 0.f, 0.f, 0.f, 0.f, 1.f};
  if (y < 0) return r;
  r.xy = y < a.V ? Elem<E>::get(static_cast<const E*>(a.x) + t * a.ld + y) : NAN;
  r.advantage = p.advantage[t];
  r.old = p.old_logp[t];
  if (p.ref_logp) r.ref = p.ref_logp[t];
  if (p.reduction == PGC_MEAN_SEQUENCES) r.share = p.share[t];
  return r;
}

// exp(u) - u - 1 with em = exp(u) - 1.  Near the reference policy, where training
// starts, it is about u^2 / 2 and em - u has few digits left (none below u = 3e-4): there the Taylor series
// u^2 (1/2! + u/3! + ... + u^6/8!), whose rest is below 2^-24 of it up to |u| = 1/2.
__device__ __forceinline__ float kl_of(float u, float em) {
  if (isinf(em)) return em;
  if (!(fabsf(u) < 0.5f)) return em - u;
  float s = 1.f / 40320.f;
  s = fmaf(s, u, 1.f / 5040.f);
  s = fmaf(s, u, 1.f / 720.f);
  s = fmaf(s, u, 1.f / 120.f);
  s = fmaf(s, u, 1.f / 24.f);
  s = fmaf(s, u, 1.f / 6.f);
  s = fmaf(s, u, 0.5f);
  return s * u * u;
}

// The scalars of the policy loss: the rows' weights, of the counts that the
// kernel before has taken, a row's part of the sums and its coefficient.
struct PolicyState {
  Sum sum[3];        // term, KL, clipped
  bool bad = false;
  float w0 = 1.f;

  // by the CTA's first warp, for all: the counts are a few lines that every CTA reads
  __device__ void weigh(const Policy& p, int2& all) {
    wait_for_previous();
    if (threadIdx.x < 32) {
      int n = 0;
      for (int i = threadIdx.x; i < p.counts; i += 32) {
        const int q = p.count[i];
        bad |= q < 0;
        n += q;
      }
      bad = __any_sync(0xffffffffu, bad);
      n = __reduce_add_sync(0xffffffffu, n);
      if (threadIdx.x == 0) all = make_int2(n, bad);
    }
    __syncthreads();
    bad = all.y != 0;
    if (p.reduction != PGC_SUM) w0 = 1.f / (float)max(all.x, 1);
  }
  // first: the thread that keeps the sums
  __device__ float coefficient(const Rows& a, const Policy& p, const RowIn& in, float lp, bool first) {
    const float w = w0 * in.share;
    if (bad) return NAN;
    if (w == 0.f) return 0.f;
    const float A = in.advantage, r = expf(lp - in.old);
    const float rc = fminf(fmaxf(r, 1.f - p.low), 1.f + p.high);
    // the smaller product; an advantage of zero takes nothing of a ratio that overflowed
    const bool free = !(r * A > rc * A);
    const float f = A == 0.f && !isnan(r) ? 0.f : free ? -r * A : -rc * A;
    float slope = free ? f : 0.f, kl = 0.f;
    if (p.ref_logp) {
      const float away = in.ref - lp, em = expm1f(away);
      kl = kl_of(away, em);
      if (p.kl != 0.f) slope -= p.kl * em;
    }
    if (first) {
      sum[0].add(w * f);
      sum[1].add(w * kl);
      sum[2].add(free ? 0.f : w);
    }
    return in.y < a.V ? p.scale * w * slope : NAN;
  }
  // the sums of a CTA's groups and of all CTAs, in order, by the CTA that comes last
  __device__ void finish(const Policy& p, Sum (*red)[3], int* last, bool keeps) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (lane == 0)
      for (int j = 0; j < 3; ++j) red[warp][j] = keeps ? sum[j] : Sum();
    __syncthreads();
    if (warp) return;
    if (lane < 3) {
      Sum s;
      for (int i = 0; i < (int)blockDim.x / 32; ++i) s.add(red[i][lane]);
      p.part[3 * blockIdx.x + lane] = make_float2(s.s, s.e);
    }
    __syncwarp();
    if (lane == 0) *last = atomic_add_acq_rel(&p.head->ticket, 1) == (int)gridDim.x - 1;
    __syncwarp();
    if (!*last) return;
    Sum s[3];
    for (int i = lane; i < (int)gridDim.x; i += 32)
      for (int j = 0; j < 3; ++j) {
        const float2 v = __ldcg(p.part + 3 * i + j);
        Sum q;
        q.s = v.x;
        q.e = v.y;
        s[j].add(q);
      }
    for (int j = 0; j < 3; ++j)
      for (int o = 16; o > 0; o >>= 1) s[j].add(shuffle_down(s[j], o));
    if (lane) return;
    for (int j = 0; j < 3; ++j) p.terms[j] = bad ? NAN : s[j].value();
    if (p.kl != 0.f) {
      s[0].add(p.kl * s[1].s);
      s[0].e += p.kl * s[1].e;
    }
    *p.loss = bad ? NAN : p.scale * s[0].value();
  }
};

// What all threads of a row need for its gradient, from the warp that works
// it out.
enum { kFast = 0, kFill = 1, kExtremeSum = 2, kExtreme = 3 };   // kFill: the row is k throughout (0 or NaN)
struct __align__(16) Published {
  float M, scale, at_y, xy;
  float m, l2, k;
  int kind;
};
// of a row with maximum m and log sum L; `first` writes its log probability and keeps its part of the sums
__device__ __forceinline__ Published work_out(const Rows& a, const Policy& p, PolicyState& state, const RowIn& in, float m,
                                              float L, int kind, int64_t t, bool first) {
  const float lp = target_logp(in.xy, make_float2(m, L), a);
  const float coef = state.coefficient(a, p, in, lp, first);
  const RowGrad r = row_grad(m, L, coef, a.inv_tau, a.c, in.y);
  if (first) p.logp[t] = lp;
  const bool fill = coef == 0.f || isnan(coef);
  return Published{r.M, r.scale, r.at_y, in.xy, r.m, r.l2, fill ? coef : r.k, fill ? kFill : kind};
}
// Maximum and sum of a row: for the warps that work out its scalars (the row's own, or the CTA's first).
template <int G>
__device__ __forceinline__ Online gather(Online o, float c, Shared& sh, int& turn, int rank, int ranks) {
  o = warp_merge(o, c);
  if (G == 32) return o;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  if (lane == 0) sh.part[0][warp] = make_float2(o.m, o.s);
  __syncthreads();
  auto among = [&](const float2* from, int n) {
    Online q;
    if (lane < n) {
      q.m = from[lane].x;
      q.s = from[lane].y;
      q.M = ref_of(q.m, c);
    }
    return warp_merge(q, c);
  };
  if (warp == 0) o = among(sh.part[0], G / 32);
  if (ranks == 1) return o;
  const int b = turn++ & 1;
  if (threadIdx.x < ranks) {
    uint32_t at;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&sh.cta[b][rank])), "r"((uint32_t)threadIdx.x));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(o.m), "f"(o.s) : "memory");
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp == 0) o = among(sh.cta[b], ranks);
  return o;
}

// Every row once, held in shared memory from the pass that sums its
// exponentials to the pass that writes its gradient, which also starts the
// next row's copies piece by piece: the logits are read once, and reads and
// writes of memory overlap.  The grid stays; a group takes every groups-th row.
// The scalars of a row are the first warp's: eight warps working them out cost
// a tenth of the kernel's time in issue slots.
template <typename E, int G, int NT>
__global__ void __launch_bounds__(NT, 768 / NT) policy_held_kernel(Rows a, Policy p, int most) {
  extern __shared__ __align__(16) unsigned char rows_smem[];
  __shared__ Shared sh;
  __shared__ Published pub;
  __shared__ Sum red[(NT / 32)][3];
  __shared__ int2 counted;
  __shared__ int last;
  constexpr bool kWarpRow = G == 32;
  const int rank = kWarpRow ? 0 : cluster_rank(), ranks = kWarpRow ? 1 : cluster_ranks();
  const int tid = threadIdx.x % G;
  const bool scalars = kWarpRow || threadIdx.x < 32;      // this warp works out the row's scalars
  const bool first = tid == 0 && rank == 0;
  const int64_t groups = kWarpRow ? gridDim.x * (int64_t)(NT / 32) : gridDim.x / ranks;
  int64_t t = kWarpRow ? blockIdx.x * (int64_t)(NT / 32) + threadIdx.x / 32 : blockIdx.x / ranks;
  const uint32_t at = smem_u32(rows_smem) + (kWarpRow ? (threadIdx.x / 32) * most * G * 16 : 0);
  int turn = 0;
  cluster_say_started(ranks);
  PolicyState state;
  const E* x = static_cast<const E*>(a.x) + t * a.ld;
  E* g = static_cast<E*>(a.g) + t * a.ldg;
  const int64_t x_step = groups * a.ld, g_step = groups * a.ldg;
  auto target_of = [&](int64_t row) { return row < a.T ? a.y[row] : -1; };
  int32_t y = target_of(t), y1 = target_of(t + groups);
  Held<E> row{nullptr, Slice{0, 0, 0, 0}, 0.f, -1};
  if (y >= 0) {
    row = hold(x, slice_of(x, a.V, rank, ranks), tid);
    copy_row<E, G>(row, at, tid, most);
  }
  state.weigh(p, counted);
  cluster_wait_started(ranks);
  RowIn in{-1, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (scalars) in = row_in<E>(a, p, t, y);
  for (; t < a.T; t += groups, x += x_step, g += g_step) {
    const int32_t y2 = target_of(t + 2 * groups);
    const bool copy = y1 >= 0;
    RowIn in1 = in;
    Held<E> next = row;
    if (copy) {
      if (scalars) in1 = row_in<E>(a, p, t + groups, y1);
      next = hold(x + x_step, slice_of(x + x_step, a.V, rank, ranks), tid);
    }
    Published q;
    q.kind = kFill;
    q.k = state.bad ? NAN : 0.f;
    if (y >= 0) {
      Online o = gather<G>(held_stats<E, G>(row, at, tid, a.c, most), a.c, sh, turn, rank, ranks);
      auto publish = [&] {
        if (kWarpRow) return;
        if (threadIdx.x == 0) pub = q;
        __syncthreads();
        q = pub;
      };
      if (scalars) {
        if (is_extreme(o.m, a.c)) q.m = o.m, q.kind = kExtremeSum;
        else q = work_out(a, p, state, in, o.m, log_sum(o, a.c), kFast, t, first);
      }
      publish();
      if (q.kind == kExtremeSum) {
        const float m = q.m;
        Online e;
        e.m = e.M = 0.f;
        e.s = held_sum_extreme<E, G>(row, at, tid, m, a.c);
        e = gather<G>(e, a.c, sh, turn, rank, ranks);
        if (scalars) q = work_out(a, p, state, in, o.m, logf(e.s), kExtreme, t, first);
        publish();
      }
    } else if (first) {
      p.logp[t] = 0.f;
    }
    const RowGrad r{q.m, q.M, a.c, q.scale, q.at_y, y, q.kind == kExtreme, q.l2, q.k};
    if (a.g && q.kind == kFast) {
      held_grad<E, G>(row, g, at, tid, q.xy, r, most, copy, next);
    } else {
      if (a.g && q.kind == kExtreme) held_grad_extreme<E, G>(row, g, at, tid, r);
      if (a.g && q.kind == kFill) {
        const Slice s = slice_of(x, a.V, rank, ranks);
        slice_fill<E, G>(g, s.first, s.last, tid, q.k);
      }
      if (copy) copy_row<E, G>(next, at, tid, most);
    }
    row = next;
    in = in1;
    y = y1;
    y1 = y2;
  }
  state.finish(p, red, &last, first);
}

// Short rows: from and to memory through registers.
template <typename E, int L, int R, int P>
__global__ void __launch_bounds__(kThreads, 4) policy_short_kernel(Rows a, Policy p) {
  __shared__ Sum red[kWarps][3];
  __shared__ int2 counted;
  __shared__ int last;
  constexpr int kRows = 32 / L;
  const int lane = threadIdx.x % 32, l = lane % L;
  PolicyState state;
  state.weigh(p, counted);
  for (int64_t t0 = (blockIdx.x * (int64_t)kWarps + threadIdx.x / 32) * kRows; t0 < a.T;
       t0 += gridDim.x * (int64_t)kWarps * kRows) {
    const int64_t t = t0 + lane / L;
    const int32_t y = t < a.T ? a.y[t] : -1;
    const RowIn in = row_in<E>(a, p, t, y);
    float v[R];
    short_load<E, L, P>(static_cast<const E*>(a.x) + t * a.ld, l, a.V, y >= 0, v);
    const float2 ms = short_exps<L>(v, y >= 0, a.c);
    if (t >= a.T) continue;
    float coef = state.bad ? NAN : 0.f, lp = 0.f;
    if (y >= 0) {
      lp = target_logp(in.xy, make_float2(ms.x, logf(ms.y)), a);
      coef = state.coefficient(a, p, in, lp, l == 0);
    }
    if (l == 0) p.logp[t] = lp;
    if (a.g) short_store<E, L, P>(static_cast<E*>(a.g) + t * a.ldg, l, a.V, v, 1.f / ms.y, coef, a.inv_tau, y);
  }
  __syncwarp();
  for (int j = 0; j < 3; ++j)
    for (int o = 16; o >= L; o >>= 1) state.sum[j].add(shuffle_down(state.sum[j], o));
  state.finish(p, red, &last, lane == 0);
}

// The same with the second reading from memory (the L2 cache, mostly).
constexpr int kLongThreads = 1024;
template <typename E>
__global__ void __launch_bounds__(kLongThreads, 1) policy_long_kernel(Rows a, Policy p) {
  constexpr int G = kLongThreads;
  __shared__ Shared sh;
  __shared__ Published pub;
  __shared__ Sum red[G / 32][3];
  __shared__ int2 counted;
  __shared__ int last;
  const int rank = cluster_rank(), ranks = cluster_ranks();
  const int tid = threadIdx.x;
  const bool scalars = tid < 32, first = tid == 0 && rank == 0;
  int turn = 0;
  cluster_say_started(ranks);
  PolicyState state;
  state.weigh(p, counted);
  cluster_wait_started(ranks);
  const int64_t groups = gridDim.x / ranks;
  for (int64_t t = blockIdx.x / ranks; t < a.T; t += groups) {
    const int32_t y = a.y[t];
    const E* x = static_cast<const E*>(a.x) + t * a.ld;
    E* g = static_cast<E*>(a.g) + t * a.ldg;
    const Slice s = slice_of(x, a.V, rank, ranks);
    Published q;
    q.kind = kFill;
    q.k = state.bad ? NAN : 0.f;
    if (y >= 0) {
      RowIn in{-1, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (scalars) in = row_in<E>(a, p, t, y);
      Online o = gather<G>(slice_stats<E, G, kUnroll>(x, s, tid, a.c), a.c, sh, turn, rank, ranks);
      auto publish = [&] {
        if (threadIdx.x == 0) pub = q;
        __syncthreads();
        q = pub;
      };
      if (scalars) {
        if (is_extreme(o.m, a.c)) q.m = o.m, q.kind = kExtremeSum;
        else q = work_out(a, p, state, in, o.m, log_sum(o, a.c), kFast, t, first);
      }
      publish();
      if (q.kind == kExtremeSum) {
        Online e;
        e.m = e.M = 0.f;
        for (unsigned v = s.first + tid; v < (unsigned)s.last; v += G) e.s += exp2f((Elem<E>::get(x + v) - q.m) * a.c);
        e = gather<G>(e, a.c, sh, turn, rank, ranks);
        if (scalars) q = work_out(a, p, state, in, o.m, logf(e.s), kExtreme, t, first);
        publish();
      }
    } else if (first) {
      p.logp[t] = 0.f;
    }
    if (!a.g) continue;
    const RowGrad r{q.m, q.M, a.c, q.scale, q.at_y, y, q.kind == kExtreme, q.l2, q.k};
    if (q.kind == kFill) slice_fill<E, G>(g, s.first, s.last, tid, q.k);
    else slice_grad<E, G, kUnroll>(x, g, s, tid, q.xy, r);
  }
  state.finish(p, red, &last, first);
}

// ---- host --------------------------------------------------------------------

// 0, or why the rows cannot be taken
int check_rows(const pgc_logits* z, bool grad_required) {
  if (!z) return PGC_EINVAL;
  if (z->dtype != PGC_F32 && z->dtype != PGC_BF16) return PGC_EINVAL;
  if (z->rows < 0 || z->rows > INT32_MAX || z->classes < 1 || z->classes > INT32_MAX) return PGC_EINVAL;
  if (!(z->temperature > 0.f) || !std::isfinite(z->temperature)) return PGC_EINVAL;
  if (!std::isfinite(1.f / z->temperature * kLog2e)) return PGC_EINVAL;
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
  return Rows{z->x, z->grad, z->target, z->rows, z->ld, z->grad_ld, (int32_t)z->classes, inv_tau, inv_tau * kLog2e};
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 148;
  return n;
}

// How the rows of a streaming pass lie on the grid: a warp each, a CTA each, or
// a cluster each.  A warp takes a row up to 24 KB where there are rows for all
// warps (bf16, 8192 classes, forward and gradient: 115 and 181 us for 800 and
// 1200 MB, at the copy rate; 168 and 192 with CTAs; at 32 KB the gradient turns: 193
// and 175, the forward pass 124 and 130), else one up to 4 KB.  Few long rows are split over a cluster while
// the SMs hold more CTAs and a part stays above 4 KB.
constexpr int64_t kWarpRowBytes = 4 * 1024, kWarpManyRowsBytes = 24 * 1024;
struct Shape {
  bool warp;
  int ranks;
  unsigned grid;
};
Shape shape_of(const pgc_logits* z) {
  const int64_t bytes = z->classes * (z->dtype == PGC_BF16 ? 2 : 4), sms = sm_count();
  Shape s{bytes <= kWarpRowBytes || (bytes <= kWarpManyRowsBytes && z->rows >= 32 * sms), 1, 0};
  if (s.warp) {
    s.grid = (unsigned)((z->rows + kWarps - 1) / kWarps);
    return s;
  }
  while (s.ranks < kMaxCluster && z->rows * s.ranks * 2 <= 2 * sms && bytes / (s.ranks * 2) >= kWarpRowBytes) s.ranks *= 2;
  s.grid = (unsigned)(z->rows * s.ranks);
  return s;
}

template <typename... P, typename... A>
cudaError_t launch(void (*kernel)(P...), unsigned grid, int threads, int ranks, bool pdl, size_t smem, cudaStream_t st, A... args) {
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
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

// Rows of bf16 whose elements can be taken in pairs (whatever the gradient's
// pitch: it does not change the results).
bool in_pairs(const pgc_logits* z) { return z->classes % 2 == 0 && z->ld % 2 == 0 && (uintptr_t)z->x % 4 == 0; }
// Short rows: up to 128 classes by 8 lanes, 256 by 16, 512 by 32 (fp32, and bf16 in
// pairs); rows above are read in 16-byte pieces by a warp.  131072 rows of 10, 100 and 256 bf16
// classes: forward 14, 12 and 20 us a call (36, 46 and 50 in pieces), gradient 12, 15
// and 27 (33, 58 and 62), policy (130624 rows) 28, 33 and 55 (85, 89 and 89); gradient of 65536 x 511 fp32 44 (54) and x 512
// bf16 27 (39).  Up to 1024 classes this way the policy loss turns: 84 us for 65337 x 1000 bf16, 64 in pieces.
bool short_rows(const pgc_logits* z) { return z->classes <= (z->dtype == PGC_F32 || in_pairs(z) ? 512 : 256); }
unsigned short_grid(const pgc_logits* z) {
  const int64_t rows = kWarps * (z->classes <= 128 ? 4 : z->classes <= 256 ? 2 : 1);
  return (unsigned)((z->rows + rows - 1) / rows);
}
// f.template operator()<E, L, R, P>()
template <typename F>
auto by_width(const pgc_logits* z, F f) {
  const int64_t V = z->classes;
  if (z->dtype == PGC_F32) {
    if (V <= 16) return f.template operator()<float, 8, 2, 1>();
    if (V <= 64) return f.template operator()<float, 8, 8, 1>();
    if (V <= 128) return f.template operator()<float, 8, 16, 1>();
    if (V <= 256) return f.template operator()<float, 16, 16, 1>();
    return f.template operator()<float, 32, 16, 1>();
  }
  using H = __nv_bfloat16;
  if (V <= 16) return f.template operator()<H, 8, 2, 1>();
  const bool two = in_pairs(z);
  if (V <= 64) return two ? f.template operator()<H, 8, 8, 2>() : f.template operator()<H, 8, 8, 1>();
  if (V <= 128) return two ? f.template operator()<H, 8, 16, 2>() : f.template operator()<H, 8, 16, 1>();
  if (V <= 256) return two ? f.template operator()<H, 16, 16, 2>() : f.template operator()<H, 16, 16, 1>();
  return f.template operator()<H, 32, 16, 2>();
}
struct ShortStats { template <typename E, int L, int R, int P> auto operator()() { return short_stats_kernel<E, L, R, P>; } };
struct ShortGrad { template <typename E, int L, int R, int P> auto operator()() { return short_grad_kernel<E, L, R, P>; } };
struct ShortPolicy { template <typename E, int L, int R, int P> auto operator()() { return policy_short_kernel<E, L, R, P>; } };

cudaError_t launch_stats(const pgc_logits* z, float* logp, float2* stats, Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  if (short_rows(z))
    return launch(by_width(z, ShortStats()), short_grid(z), kThreads, 1, false, 0, st, rows_of(z), logp, stats, head);
  const Shape s = shape_of(z);
  const bool half = z->dtype == PGC_BF16;
  return launch(half ? s.warp ? row_stats_kernel<__nv_bfloat16, 32> : row_stats_kernel<__nv_bfloat16, kThreads>
                     : s.warp ? row_stats_kernel<float, 32> : row_stats_kernel<float, kThreads>,
                s.grid, kThreads, s.ranks, false, 0, st, rows_of(z), logp, stats, head);
}

// The gradient pass takes a row that a CTA or a cluster has in parts of 32 to 64 KB (whole up to 64 KB; few
// rows in as many parts as the cluster has CTAs, of 4 KB at least): smaller grains
// level the last wave (2000 x 50001 fp32: 114 us, 125 with whole rows; parts of 16 KB 127).
constexpr int64_t kGradPartBytes = 32 * 1024;
cudaError_t launch_grad(const pgc_logits* z, const float* coef, const float2* stats, const Head* head, cudaStream_t st) {
  if (z->rows == 0) return cudaSuccess;
  if (short_rows(z))
    return launch(by_width(z, ShortGrad()), short_grid(z), kThreads, 1, head != nullptr, 0, st, rows_of(z), coef, stats, head);
  const Shape s = shape_of(z);
  const bool half = z->dtype == PGC_BF16;
  const int64_t bytes = z->classes * (half ? 2 : 4), most = INT32_MAX / z->rows;
  const int parts = s.warp ? 1 : (int)std::min(std::max<int64_t>(s.ranks, bytes / kGradPartBytes), most);
  return launch(half ? s.warp ? row_grad_kernel<__nv_bfloat16, 32> : row_grad_kernel<__nv_bfloat16, kThreads>
                     : s.warp ? row_grad_kernel<float, 32> : row_grad_kernel<float, kThreads>,
                s.warp ? s.grid : (unsigned)(z->rows * parts), kThreads, 1, head != nullptr, 0, st, rows_of(z), parts,
                coef, stats, head);
}

constexpr int kMaxParts = 1024;       // CTAs of the kernels that leave partial sums

// Policy loss.  Rows up to 12 KB are a warp's (bf16, 24041 x 4096: 83 us with
// warps, 104 with CTAs; 16816 x 8192, 16 KB a row: 116 against 109), longer ones a CTA's: of 128
// threads up to 36 KB, of 256 up to 110, of 512 above (a thread then has about
// 16 places, and the SM as many warps as its shared memory allows rows for:
// 12195 x 16384: 142 us with 128 threads, 157 with 256).  A row between 110 and 148 KB
// leaves room for no second one on the SM, so two CTAs of a cluster share it
// (4506 x 65536: 226 us, 254 by one CTA); beyond that sharing costs more than
// it brings, as each CTA waits for the other (4472 x 100000: 342 us by one CTA, 351 by two),
// but where rows are too few for the SMs more CTAs shorten a row's
// time.  A thread's places are even, so 512 threads hold rows in steps of 16 KB, the longest
// 208 KB; above that a row is read twice by 1024 threads (4472 x 131072:
// 446 us, 534 in two halves held by two SMs; 4472 x 100000 read twice: 382).
constexpr int64_t kHeldWarpBytes = 12 * 1024, kHeld128Bytes = 36 * 1024, kHeld256Bytes = 110 * 1024,
                  kHeldPairBytes = 148 * 1024, kHeldSmem = 216 * 1024;
// Shared memory above 48 KB is asked for once per device and kernel.
cudaError_t allow_smem(const void* kernel, int which) {
  static std::atomic<uint32_t> allowed[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  std::atomic<uint32_t>* seen = dev >= 0 && dev < 64 ? &allowed[dev] : nullptr;
  if (seen && seen->load(std::memory_order_acquire) >> which & 1u) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kHeldSmem);
  if (e == cudaSuccess && seen) seen->fetch_or(1u << which, std::memory_order_release);
  return e;
}

template <typename E>
cudaError_t launch_policy(const pgc_logits* z, const Policy& p, cudaStream_t st) {
  const int64_t sms = sm_count(), pieces = z->classes / Elem<E>::N, bytes = pieces * 16;
  if (short_rows(z)) {
    const int64_t most = std::min<int64_t>(sms * 4, kMaxParts);
    return launch(by_width(z, ShortPolicy()), (unsigned)std::max<int64_t>(std::min<int64_t>(short_grid(z), most), 1), kThreads, 1,
                  true, 0, st, rows_of(z), p);
  }
  const bool warp = bytes <= kHeldWarpBytes;
  int ranks = 1;
  if (!warp) {
    if (bytes > kHeld256Bytes && bytes <= kHeldPairBytes) ranks = 2;
    while (ranks < kMaxCluster && z->rows * ranks * 2 <= sms && bytes / ranks > 16384) ranks *= 2;
  }
  const int64_t slice = (pieces + ranks - 1) / ranks;
  const int threads = warp ? 256 : slice * 16 <= kHeld128Bytes ? 128 : slice * 16 <= kHeld256Bytes ? 256 : 512;
  const int group = warp ? 32 : threads;
  const int most = (int)std::max<int64_t>(((slice + group - 1) / group + 1) / 2 * 2, 2);
  const int64_t smem = (int64_t)most * 16 * threads;
  const int64_t units = warp ? (z->rows + threads / 32 - 1) / (threads / 32) : z->rows * ranks;
  if (smem > kHeldSmem) {
    const unsigned grid = (unsigned)std::max<int64_t>(std::min<int64_t>(units, sms / ranks * ranks), ranks);
    return launch(policy_long_kernel<E>, grid, kLongThreads, ranks, true, 0, st, rows_of(z), p);
  }
  const auto kernel = warp ? policy_held_kernel<E, 32, 256>
                      : threads == 128 ? policy_held_kernel<E, 128, 128>
                      : threads == 256 ? policy_held_kernel<E, 256, 256> : policy_held_kernel<E, 512, 512>;
  const cudaError_t e = allow_smem(reinterpret_cast<const void*>(kernel),
                                   (warp ? 0 : threads == 128 ? 1 : threads == 256 ? 2 : 3) + (Elem<E>::N == 8 ? 4 : 0));
  if (e != cudaSuccess) return e;
  int64_t most_ctas = sms * std::max<int64_t>(1, std::min<int64_t>(768 / threads, (226 * 1024) / (smem + 2048)));
  most_ctas = std::min<int64_t>(most_ctas, kMaxParts) / ranks * ranks;
  return launch(kernel, (unsigned)std::max<int64_t>(std::min(units, most_ctas), ranks), threads, ranks, true, (size_t)smem, st,
                rows_of(z), p, most);
}

// Layout of the workspace (bytes): head, counts [kMaxParts], partial sums
// [kMaxParts][3] of 8, the pairs' losses [sequences], stats [rows], logp [rows],
// coef or share [rows].
struct Work {
  Head* head;
  int32_t* count;
  float2* sums;
  float2* stats;
  float *pair_loss, *logp, *coef, *share;
};
constexpr int64_t kHeadBytes = 256, kCountBytes = kMaxParts * 4, kSumBytes = kMaxParts * 24;
int64_t work_bytes(int64_t rows, int64_t sequences) {
  return kHeadBytes + kCountBytes + kSumBytes + rows * 16 + sequences * 4;
}
Work work_at(void* ws, int64_t rows) {
  char* p = static_cast<char*>(ws);
  Work w;
  w.head = reinterpret_cast<Head*>(p);
  p += kHeadBytes;
  w.count = reinterpret_cast<int32_t*>(p);
  p += kCountBytes;
  w.sums = reinterpret_cast<float2*>(p);
  p += kSumBytes;
  w.stats = reinterpret_cast<float2*>(p);
  w.logp = reinterpret_cast<float*>(p + 8 * rows);
  w.coef = w.share = w.logp + rows;
  w.pair_loss = w.coef + rows;
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
  if (!z) return PGC_EINVAL;
  pgc_logits forward = *z;              // z->grad and its pitch are not used
  forward.grad = nullptr;
  int rc = check_rows(&forward, false);
  if (rc) return rc;
  if (z->rows && (!logp || !stats)) return PGC_EINVAL;
  if ((uintptr_t)logp % 4 || (uintptr_t)stats % 8) return PGC_EINVAL;
  return report_cuda(launch_stats(&forward, logp, reinterpret_cast<float2*>(stats), nullptr, (cudaStream_t)stream));
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
  const Work w = work_at(workspace, z->rows);
  const cudaStream_t st = (cudaStream_t)stream;
  Pref a{kind, average, pairs, z->rows, offsets, z->target, ref_logp, w.logp, beta, margin, smoothing, scale,
         w.coef, logp, w.pair_loss, loss, w.head};
  cudaError_t e = z->rows ? launch_stats(z, w.logp, w.stats, w.head, st)
                          : cudaMemsetAsync(w.head, 0, sizeof(Head), st);
  if (e != cudaSuccess) return report_cuda(e);
  // a warp per pair while pairs are short (64 rows a sequence): tens of thousands of them are a few waves
  const bool warp = z->rows <= 128 * pairs;
  e = launch(warp ? pair_kernel<32> : pair_kernel<kThreads>,
             (unsigned)std::max<int64_t>(warp ? (pairs + kWarps - 1) / kWarps : pairs, 1), kThreads, 1, true, 0, st, a);
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
  const Work w = work_at(workspace, z->rows);
  const cudaStream_t st = (cudaStream_t)stream;
  Policy a{reduction, z->rows, sequences, offsets, z->target, old_logp, ref_logp, advantage, logp, clip_low, clip_high,
           kl, scale, w.count, 0, w.share, w.sums, loss, terms, w.head};
  const int64_t units = reduction == PGC_MEAN_SEQUENCES ? sequences : (z->rows + kThreads - 1) / kThreads;
  a.counts = (int)std::min<int64_t>(std::max<int64_t>(units, 1), 128);
  count_kernel<<<a.counts, kThreads, 0, st>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return report_cuda(e);
  return report_cuda(z->dtype == PGC_BF16 ? launch_policy<__nv_bfloat16>(z, a, st) : launch_policy<float>(z, a, st));
}

}  // extern "C"
