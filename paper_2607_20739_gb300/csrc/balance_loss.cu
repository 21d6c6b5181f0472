// Router choice, per-expert counts and balance loss with its gradient
// (pgc_balance_loss).
//
// n tokens take part; token t chooses the k experts of its largest logits,
// c_e tokens chose expert e, p_t = softmax(x_t).  With f_e = c_e / (k n) and
// P_e = (1/n) sum_t p_te the loss is L = alpha E sum_e f_e P_e.  The counts are
// constants to the gradient: with w_e = alpha E c_e / (k n^2),
//   L = sum_t sum_e w_e p_te,   dL/dx_te = p_te (w_e - sum_j w_j p_tj),
// so a token's part of the loss is the inner product that its gradient needs,
// and no mean of probabilities over the tokens has to be formed.
#include <algorithm>
#include <cmath>

#include "dev_common.cuh"
#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxExperts = 1024, kMaxChoices = 64;
constexpr int kMaxGrid = 1024;

struct Head {
  int32_t tokens;                 // n
  int32_t ticket;
  int32_t counts[kMaxExperts];
};

struct Balance {
  const void* x;
  void* g;
  const uint8_t* mask;
  int32_t* choice;
  int32_t* counts;
  float* loss;
  Sum* part;                      // [grid]
  Head* head;
  int64_t T, ld, ldg;
  int E, k, given;
  int wide_x, wide_g;             // rows of logits / gradients in whole 16-byte pieces
  float alpha;
};

// What bounds it, at 65536 tokens x 256 experts, k = 8, fp32 (64 us, of which the
// choice 37 and the gradient 27; reading and writing the logits would take 20): the choice the ALU
// (63 % busy with 417 instructions a token, comparisons mostly) and the latencies between
// them; the gradient the memory's latency (205 instructions a token are 40 % of the issue slots; 134 MB in 27 us are
// 4.8 TB/s).  More or fewer than 4 CTAs of 256 threads per SM are slower (60000 x 256: 60 us; 66
// with 3, 72 with 6, 68 with 8).  16384 x 128 bf16: 18 us on the GPU.
//
// A token belongs to L lanes, lane l of them has experts l R .. l R + R - 1 in
// registers (-inf behind the last expert): as many tokens per warp as fit.
template <typename X, int R>
__device__ __forceinline__ void load_experts(const X* x, int l, int E, bool wide, float (&v)[R]) {
  const int e0 = l * R;
  if (wide) {
    constexpr int N = Elem<X>::N;
#pragma unroll
    for (int q = 0; q < R / N; ++q) {
      uint4 piece = no_piece(Elem<X>::kLowest);
      if (e0 + q * N < E) piece = load16(reinterpret_cast<const uint4*>(x + e0) + q);
      Pair f[N / 2];
      Elem<X>::widen(piece, f);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) split(f[i], v[q * N + 2 * i], v[q * N + 2 * i + 1]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = e0 + j < E ? Elem<X>::get(x + e0 + j) : -INFINITY;
  }
}
template <typename X, int R>
__device__ __forceinline__ void store_experts(X* g, int l, int E, bool wide, const float (&v)[R]) {
  const int e0 = l * R;
  if (wide) {
    constexpr int N = Elem<X>::N;
#pragma unroll
    for (int q = 0; q < R / N; ++q) {
      Pair f[N / 2];
#pragma unroll
      for (int i = 0; i < N / 2; ++i) f[i] = pair(v[q * N + 2 * i], v[q * N + 2 * i + 1]);
      if (e0 + q * N < E) store16(reinterpret_cast<uint4*>(g + e0) + q, Elem<X>::narrow(f));
    }
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (e0 + j < E) Elem<X>::put(g + e0 + j, v[j]);
  }
}

template <int L>
__device__ __forceinline__ unsigned group_max(unsigned v) {
  if (L == 32) return __reduce_max_sync(0xffffffffu, v);
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
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

// Order of floats as unsigned numbers; below kChosen what is never chosen (-inf,
// and NaN as -inf).
constexpr unsigned kChosen = 0x00800000u;
__device__ __forceinline__ unsigned order_of(float f) {
  const unsigned u = __float_as_uint(fmaxf(f, -INFINITY) + 0.f);      // -0 as 0
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}

// The choice by definition: the largest logit behind the last one chosen, in the
// order (value, expert), k times.  Choice i is lane i % L's, which writes and
// counts it if out is given; returns the lane's last one.
template <int L, int R>
__device__ __noinline__ int choose_exact(const float (&v)[R], int l, int k, int32_t* out, int* count) {
  unsigned last = 0xffffffffu;
  int last_e = -1, held = -1;
  for (int i = 0; i < k; ++i) {
    unsigned best = kChosen - 1;
    int best_e = kMaxExperts;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const unsigned o = order_of(v[j]);
      const int e = l * R + j;
      if ((o < last || (o == last && e > last_e)) && o > best) {
        best = o;
        best_e = e;
      }
    }
    for (int s = L / 2; s > 0; s >>= 1) {
      const unsigned o = __shfl_xor_sync(0xffffffffu, best, s);
      const int e = __shfl_xor_sync(0xffffffffu, best_e, s);
      if (o > best || (o == best && e < best_e)) {
        best = o;
        best_e = e;
      }
    }
    if (l == (i & (L - 1))) {
      held = best >= kChosen ? best_e : -1;
      if (out) {
        out[i] = held;
        if (held >= 0) atomicAdd(count + held, 1);
      }
    }
    last = best;
    last_e = best_e;
  }
  return held;
}

// The same from keys of 32 bits, for k <= L: each lane sorts its own and the
// group takes the largest head k times; returns lane i's choice i.  A bf16
// logit and its expert fit one key (16 bits each, the lower expert the larger
// key).  A float keeps the upper bits of its order and its place in the lane;
// where two of the chosen, or the last of them and the next, agree in these upper
// bits, the definition decides.
template <typename X, int L, int R>
__device__ __forceinline__ int choose_keys(const float (&v)[R], int l, int k) {
  constexpr bool kWhole = sizeof(X) == 2;
  constexpr int kBits = R == 8 ? 3 : 4;
  constexpr unsigned kPlace = (1u << kBits) - 1;
  static_assert(R == 8 || R == 16, "places of a lane");
  unsigned key[R];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const unsigned o = order_of(v[j]);
    key[j] = kWhole ? (o & 0xffff0000u) | (0xffffu - (unsigned)(l * R + j)) : (o & ~kPlace) | (kPlace - (unsigned)j);
  }
  // Batcher's odd-even merge sort, largest first
#pragma unroll
  for (int p = 1; p < R; p *= 2)
#pragma unroll
    for (int q = p; q >= 1; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < R; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < R && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const unsigned hi = max(key[i + j], key[i + j + q]);
            key[i + j + q] = min(key[i + j], key[i + j + q]);
            key[i + j] = hi;
          }
  unsigned last = 0;
  int held = -1;
  bool unsure = false;
  // choice i; `left` of the lane's keys can still matter behind it
  auto take = [&](int i, int left) {
    const unsigned best = group_max<L>(key[0]);
    const bool mine = key[0] == best;
    int e;
    if (kWhole) {
      e = 0xffff - (int)(best & 0xffffu);
    } else {
      unsigned who = __ballot_sync(0xffffffffu, mine);
      if (L < 32) who = who >> (threadIdx.x % 32 / L * L) & ((1u << (L % 32)) - 1u);
      unsure |= best >= kChosen && ((who & (who - 1)) || best >> kBits == last >> kBits);
      e = (__ffs(who) - 1) * R + (int)(kPlace - (best & kPlace));
    }
    last = best;
    if (l == i) held = best >= kChosen ? e : -1;
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (j < left) key[j] = mine ? (j + 1 < R ? key[j + 1] : 0u) : key[j];
  };
  if (R == 8 && k <= 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < k) take(i, 8 - i);
  } else {
    for (int i = 0; i < k; ++i) take(i, R);
  }
  if (!kWhole) {
    const unsigned next = group_max<L>(key[0]);
    unsure |= next >= kChosen && next >> kBits == last >> kBits;
    if (__any_sync(0xffffffffu, unsure)) {
      const int exact = choose_exact<L, R>(v, l, k, nullptr, nullptr);
      if (unsure) held = exact;
    }
  }
  return held;
}

// For a whole warp per token and k <= kFew: the k-th largest of the lanes'
// maxima is no more than the k-th largest logit, and few logits reach it.  They are gathered, one
// per lane, and the largest of them (ties: the lowest expert) is taken k times,
// in fewer instructions than sorted lanes (60000 x 256 fp32, k = 8: 60 us for the call, 67
// with sorted keys; 30000 x 384 bf16: 56, 60).  bf16 up to 256 experts stays with keys that
// hold logit and expert at once (60000 x 256: 50, 56 this way).  -2: more than 32 reach it.
constexpr int kFew = 8;
template <int R>
__device__ __forceinline__ int choose_few(const float (&v)[R], int lane, int k, uint2* slot) {
  unsigned key[R], top = 0;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    key[j] = order_of(v[j]);
    top = max(top, key[j]);
  }
  unsigned least = 0;
  for (int i = 0; i < k; ++i) {
    least = __reduce_max_sync(0xffffffffu, top);
    top = top == least ? 0u : top;
  }
  least = max(least, kChosen);
  const unsigned below = (1u << lane) - 1u;
  int n = 0;
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const bool reaches = key[j] >= least;
    const unsigned all = __ballot_sync(0xffffffffu, reaches);
    const int at = n + __popc(all & below);
    if (reaches && at < 32) slot[at] = make_uint2(key[j], (unsigned)(lane * R + j));
    n += __popc(all);
  }
  __syncwarp();
  uint2 mine = lane < n ? slot[lane] : make_uint2(0u, 0xffffffffu);
  __syncwarp();
  if (n > 32) return -2;
  int held = -1;
  for (int i = 0; i < k; ++i) {
    const unsigned best = __reduce_max_sync(0xffffffffu, mine.x);
    const unsigned e = __reduce_min_sync(0xffffffffu, mine.x == best ? mine.y : 0xffffffffu);
    if (lane == i && best) held = (int)e;
    if (mine.y == e) mine.x = 0u;
  }
  return held;
}

// Choices and counts of the rows that this CTA takes (every `step`-th block of
// rows from block `first`); counts, tokens and slots (32 per warp) are in shared memory.
template <typename X, int L, int R>
__device__ __forceinline__ void choose_rows(const Balance& a, int64_t first, int64_t step, int* count, int* tokens, uint2* slots) {
  constexpr int kRows = 32 / L;                     // tokens per warp
  const int lane = threadIdx.x % 32, l = lane % L;
  int n = 0;
  for (int64_t t0 = (first * (blockDim.x / 32) + threadIdx.x / 32) * kRows; t0 < a.T; t0 += step * (blockDim.x / 32) * kRows) {
    const int64_t t = t0 + lane / L;
    const bool on = t < a.T && (!a.mask || a.mask[t]);
    int32_t* out = a.choice + t * a.k;
    n += on && l == 0;
    if (a.given) {
      if (on)
        for (int j = l; j < a.k; j += L)
          if (out[j] >= 0 && out[j] < a.E) atomicAdd(count + out[j], 1);
      continue;
    }
    float v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = -INFINITY;
    if (on) load_experts<X, R>(static_cast<const X*>(a.x) + t * a.ld, l, a.E, a.wide_x, v);
    if constexpr (R <= 16) {
      int e = -2;
      if constexpr (L == 32 && (sizeof(X) == 4 || R > 8)) {
        if (a.k <= kFew) e = choose_few<R>(v, l, a.k, slots + (threadIdx.x / 32) * 32);
        if (__any_sync(0xffffffffu, e == -2)) e = choose_keys<X, L, R>(v, l, a.k);
      } else {
        e = choose_keys<X, L, R>(v, l, a.k);
      }
      if (t < a.T && l < a.k) {
        out[l] = e;
        if (e >= 0) atomicAdd(count + e, 1);
      }
    } else {
      choose_exact<L, R>(v, l, a.k, t < a.T ? out : nullptr, count);
    }
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if (lane == 0 && n) atomicAdd(tokens, n);
}

// Gradients of the same rows and the CTA's part of the loss (in thread 0);
// counts in shared memory.
template <typename X, int L, int R>
__device__ __forceinline__ Sum grad_rows(const Balance& a, int64_t first, int64_t step, const int* counts, float base, Sum* red) {
  constexpr int kRows = 32 / L;
  const int lane = threadIdx.x % 32, l = lane % L;
  float w[R];                                       // base times the counts of this lane's experts
#pragma unroll
  for (int j = 0; j < R; ++j) w[j] = l * R + j < a.E ? base * (float)counts[l * R + j] : 0.f;
  Sum sum;
  for (int64_t t0 = (first * (blockDim.x / 32) + threadIdx.x / 32) * kRows; t0 < a.T; t0 += step * (blockDim.x / 32) * kRows) {
    const int64_t t = t0 + lane / L;
    const bool on = t < a.T && (!a.mask || a.mask[t]);
    float v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = -INFINITY;
    if (on) load_experts<X, R>(static_cast<const X*>(a.x) + t * a.ld, l, a.E, a.wide_x, v);
    float m = v[0];
#pragma unroll
    for (int j = 1; j < R; ++j) m = fmaxf(m, v[j]);
    m = group_max<L>(m);
    if (m == -INFINITY) m = 0.f;     // no part taken, or no expert left: all zeros (a NaN stays)
    float s = 0.f, dot = 0.f;
#pragma unroll
    for (int j = 0; j < R; ++j) {
      v[j] = ex2((v[j] - m) * kLog2e);
      s += v[j];
      dot = fmaf(v[j], w[j], dot);
    }
    s = group_sum<L>(s);
    dot = group_sum<L>(dot);
    const float r = s == 0.f ? 0.f : 1.f / s;
    dot *= r;
    if (l == 0 && on) sum.add(dot);
    if (a.g && t < a.T) {
#pragma unroll
      for (int j = 0; j < R; ++j) v[j] = v[j] * r * (w[j] - dot);
      store_experts<X, R>(static_cast<X*>(a.g) + t * a.ldg, l, a.E, a.wide_g, v);
    }
  }
  return block_sum(sum, red);
}

// alpha E / (k n^2)
__device__ __forceinline__ float weight_of(const Balance& a, int tokens) {
  const float n = (float)max(tokens, 1);
  return a.alpha * (float)a.E / (float)a.k / n / n;
}

template <typename X, int L, int R>
__global__ void __launch_bounds__(kThreads) choose_kernel(Balance a) {
  __shared__ int count[kMaxExperts];
  __shared__ uint2 slots[L == 32 ? kThreads : 1];
  __shared__ int tokens;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  for (int e = threadIdx.x; e < a.E; e += kThreads) count[e] = 0;
  if (threadIdx.x == 0) tokens = 0;
  __syncthreads();
  choose_rows<X, L, R>(a, blockIdx.x, gridDim.x, count, &tokens, slots);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kThreads)
    if (count[e]) atomicAdd(a.head->counts + e, count[e]);
  if (threadIdx.x == 0 && tokens) atomicAdd(&a.head->tokens, tokens);
}

template <typename X, int L, int R>
__global__ void __launch_bounds__(kThreads) balance_grad_kernel(Balance a) {
  __shared__ int count[kMaxExperts];               // every CTA reads the counts once: they are a few lines of the L2 cache
  __shared__ Sum red[32];
  __shared__ int last;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    count[e] = __ldcg(a.head->counts + e);
    if (blockIdx.x == 0) a.counts[e] = count[e];
  }
  const float base = weight_of(a, __ldcg(&a.head->tokens));
  __syncthreads();
  const Sum sum = grad_rows<X, L, R>(a, blockIdx.x, gridDim.x, count, base, red);
  if (threadIdx.x == 0) {
    a.part[blockIdx.x] = sum;
    last = atomic_add_acq_rel(&a.head->ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  Sum all;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) {
    const float2 v = __ldcg(reinterpret_cast<const float2*>(a.part) + i);
    Sum q;
    q.s = v.x;
    q.e = v.y;
    all.add(q);
  }
  all = block_sum(all, red);
  if (threadIdx.x == 0) *a.loss = all.value();
}

// One CTA for few tokens: no counts to clear in memory, and one launch.
constexpr int kSmallThreads = 1024;
template <typename X, int L, int R>
__global__ void __launch_bounds__(kSmallThreads) balance_small_kernel(Balance a) {
  __shared__ int count[kMaxExperts];
  __shared__ uint2 slots[L == 32 ? kSmallThreads : 1];
  __shared__ Sum red[32];
  __shared__ int tokens;
  for (int e = threadIdx.x; e < a.E; e += kSmallThreads) count[e] = 0;
  if (threadIdx.x == 0) tokens = 0;
  __syncthreads();
  choose_rows<X, L, R>(a, 0, 1, count, &tokens, slots);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kSmallThreads) a.counts[e] = count[e];
  const Sum sum = grad_rows<X, L, R>(a, 0, 1, count, weight_of(a, tokens), red);
  if (threadIdx.x == 0) *a.loss = sum.value();
}

constexpr int64_t kWorkBytes = (sizeof(Head) + 255) / 256 * 256 + kMaxGrid * sizeof(Sum);

// Tokens times lanes of one: one CTA takes up to two passes of its 1024 threads
// (512 x 8, two passes: 20 us a call; 26.5 with the two kernels and the clearing before
// them; one token of 64 experts: 20 and 25).
constexpr int64_t kSmallLanes = 2 * kSmallThreads;
template <typename X, int L, int R>
cudaError_t launch_balance(Balance a, cudaStream_t st) {
  if (a.T * L <= kSmallLanes) {
    balance_small_kernel<X, L, R><<<1, kSmallThreads, 0, st>>>(a);
    return cudaGetLastError();
  }
  cudaError_t e = cudaMemsetAsync(a.head, 0, offsetof(Head, counts) + a.E * sizeof(int32_t), st);
  if (e != cudaSuccess) return e;
  constexpr int kRows = kWarps * 32 / L;
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    sms = 148;
  const unsigned grid = (unsigned)std::min<int64_t>(std::min<int64_t>((a.T + kRows - 1) / kRows, (int64_t)sms * 4), kMaxGrid);
  choose_kernel<X, L, R><<<grid, kThreads, 0, st>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, balance_grad_kernel<X, L, R>, a);
}
// The fewest lanes that hold a token's experts, 8 each, and its choices, one each.
template <typename X>
cudaError_t launch_balance(const Balance& a, cudaStream_t st) {
  if (a.E <= 32 && a.k <= 4) return launch_balance<X, 4, 8>(a, st);
  if (a.E <= 64 && a.k <= 8) return launch_balance<X, 8, 8>(a, st);
  if (a.E <= 128 && a.k <= 16) return launch_balance<X, 16, 8>(a, st);
  if (a.E <= 256 && a.k <= 32) return launch_balance<X, 32, 8>(a, st);
  if (a.E <= 512 && a.k <= 32) return launch_balance<X, 32, 16>(a, st);
  return launch_balance<X, 32, 32>(a, st);
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_balance_workspace(int64_t rows, int64_t experts, int64_t *bytes) {
  if (!bytes || rows < 0 || rows > INT32_MAX || experts < 1 || experts > kMaxExperts) return PGC_EINVAL;
  *bytes = kWorkBytes;
  return PGC_OK;
}

int pgc_balance_loss(int32_t dtype, int64_t rows, int64_t experts, const void *logits, int64_t ld, const uint8_t *mask,
                     int32_t k, int32_t given, int32_t *choice, float alpha, float *loss, int32_t *counts, void *grad,
                     int64_t grad_ld, void *workspace, int64_t workspace_bytes, void *stream) {
  if (dtype != PGC_F32 && dtype != PGC_BF16) return PGC_EINVAL;
  if (rows < 0 || rows > INT32_MAX || experts < 1 || k < 1 || k > experts || !std::isfinite(alpha)) return PGC_EINVAL;
  const int64_t far = int64_t(1) << 31;
  if (ld < experts || ld > far || (grad && (grad_ld < experts || grad_ld > far))) return PGC_EINVAL;
  if (grad && grad == logits && grad_ld != ld) return PGC_EINVAL;
  if (!loss || !counts || (rows && (!logits || !choice))) return PGC_EINVAL;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if ((uintptr_t)logits % size || (uintptr_t)grad % size || (uintptr_t)loss % 4 || (uintptr_t)counts % 4 ||
      (uintptr_t)choice % 4 || !workspace || (uintptr_t)workspace % 16)
    return PGC_EINVAL;
  if (experts > kMaxExperts || k > kMaxChoices) return PGC_ENOTSUP;
  if (workspace_bytes < kWorkBytes) return PGC_ESCRATCH;
  Balance a;
  a.x = logits; a.g = grad; a.mask = mask; a.choice = choice; a.counts = counts; a.loss = loss;
  a.head = static_cast<Head*>(workspace);
  a.part = reinterpret_cast<Sum*>(static_cast<char*>(workspace) + kWorkBytes - kMaxGrid * sizeof(Sum));
  a.T = rows; a.ld = ld; a.ldg = grad_ld; a.E = (int)experts; a.k = k; a.given = given; a.alpha = alpha;
  const int64_t n = 16 / (int64_t)size;
  a.wide_x = (uintptr_t)logits % 16 == 0 && ld % n == 0 && experts % n == 0;
  a.wide_g = (uintptr_t)grad % 16 == 0 && grad_ld % n == 0 && experts % n == 0;
  const cudaStream_t st = (cudaStream_t)stream;
  return report_cuda(dtype == PGC_BF16 ? launch_balance<__nv_bfloat16>(a, st) : launch_balance<float>(a, st));
}

}  // extern "C"
