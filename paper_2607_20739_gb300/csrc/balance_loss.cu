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

namespace pgc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kMaxExperts = 1024, kMaxChoices = 64;

struct Head {
  int32_t tokens;   // n
  int32_t ticket;
};

struct Balance {
  const void* x;
  void* g;
  const uint8_t* mask;
  int32_t* choice;
  int32_t* counts;
  float* loss;
  double* part;
  Head* head;
  int64_t T, ld, ldg;
  int E, k, given;
  float alpha;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A warp per token.  Largest first, ties to the lowest expert; an expert of
// logit -inf (or NaN) is never chosen, its place in the choice is -1.
template <typename X>
__global__ void __launch_bounds__(kThreads) choose_kernel(Balance a) {
  __shared__ int count[kMaxExperts];
  __shared__ int tokens;
  for (int e = threadIdx.x; e < a.E; e += kThreads) count[e] = 0;
  if (threadIdx.x == 0) tokens = 0;
  __syncthreads();
  const int lane = threadIdx.x % 32;
  for (int64_t t = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32; t < a.T; t += gridDim.x * (int64_t)kWarps) {
    const bool on = !a.mask || a.mask[t];
    int32_t* out = a.choice + t * a.k;
    if (on && lane == 0) atomicAdd(&tokens, 1);
    if (a.given) {
      if (on)
        for (int j = lane; j < a.k; j += 32)
          if (out[j] >= 0 && out[j] < a.E) atomicAdd(&count[out[j]], 1);
      continue;
    }
    if (!on) {
      for (int j = lane; j < a.k; j += 32) out[j] = -1;
      continue;
    }
    const X* x = static_cast<const X*>(a.x) + t * a.ld;
    float last = INFINITY;
    int last_e = -1;
    for (int j = 0; j < a.k; ++j) {
      // the largest behind (last, last_e) in the order of the choice
      float best = -INFINITY;
      int best_e = a.E;
      for (int e = lane; e < a.E; e += 32) {
        const float v = to_float(x[e]);
        if ((v < last || (v == last && e > last_e)) && v > best) {
          best = v;
          best_e = e;
        }
      }
      for (int o = 16; o > 0; o >>= 1) {
        const float v = __shfl_xor_sync(0xffffffffu, best, o);
        const int e = __shfl_xor_sync(0xffffffffu, best_e, o);
        if (v > best || (v == best && e < best_e)) {
          best = v;
          best_e = e;
        }
      }
      const bool found = best_e < a.E;
      if (lane == 0) {
        out[j] = found ? best_e : -1;
        if (found) atomicAdd(&count[best_e], 1);
      }
      last = best;
      last_e = best_e;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += kThreads)
    if (count[e]) atomicAdd(a.counts + e, count[e]);
  if (threadIdx.x == 0 && tokens) atomicAdd(&a.head->tokens, tokens);
}

template <typename X>
__global__ void __launch_bounds__(kThreads) balance_grad_kernel(Balance a) {
  __shared__ float w[kMaxExperts];
  __shared__ double red[kWarps];
  __shared__ int last;
  const double n = max(a.head->tokens, 1);
  for (int e = threadIdx.x; e < a.E; e += kThreads)
    w[e] = (float)((double)a.alpha * a.E * a.counts[e] / (a.k * n * n));
  __syncthreads();
  const int lane = threadIdx.x % 32;
  double sum = 0.0;
  for (int64_t t = blockIdx.x * (int64_t)kWarps + threadIdx.x / 32; t < a.T; t += gridDim.x * (int64_t)kWarps) {
    X* g = static_cast<X*>(a.g) + t * a.ldg;
    if (a.mask && !a.mask[t]) {
      if (a.g)
        for (int e = lane; e < a.E; e += 32) put(g + e, 0.f);
      continue;
    }
    const X* x = static_cast<const X*>(a.x) + t * a.ld;
    float m = -INFINITY;
    for (int e = lane; e < a.E; e += 32) m = fmaxf(m, to_float(x[e]));
    m = warp_max(m);
    if (m == -INFINITY) {
      bool nan = false;
      for (int e = lane; e < a.E; e += 32) nan |= isnan(to_float(x[e]));
      if (!__any_sync(0xffffffffu, nan)) {   // no expert left
        if (a.g)
          for (int e = lane; e < a.E; e += 32) put(g + e, 0.f);
        continue;
      }
    }
    float s = 0.f, dot = 0.f;
    for (int e = lane; e < a.E; e += 32) {
      const float p = expf(to_float(x[e]) - m);
      s += p;
      dot += p * w[e];
    }
    s = warp_sum(s);
    dot = warp_sum(dot) / s;
    sum += dot;
    if (a.g)
      for (int e = lane; e < a.E; e += 32) {
        const float p = expf(to_float(x[e]) - m) / s;
        put(g + e, p * (w[e] - dot));
      }
  }
  if (lane == 0) red[threadIdx.x / 32] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    sum = 0.0;
    for (int i = 0; i < kWarps; ++i) sum += red[i];
    a.part[blockIdx.x] = sum;
    last = atomic_add_acq_rel(&a.head->ticket, 1) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!last || threadIdx.x) return;
  sum = 0.0;
  for (int i = 0; i < (int)gridDim.x; ++i) sum += __ldcg(a.part + i);
  *a.loss = (float)sum;
}

constexpr int kMaxGrid = 1024;
constexpr int64_t kWorkBytes = 256 + kMaxGrid * 8;

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
  const cudaStream_t st = (cudaStream_t)stream;
  Balance a;
  a.x = logits; a.g = grad; a.mask = mask; a.choice = choice; a.counts = counts; a.loss = loss;
  a.head = static_cast<Head*>(workspace);
  a.part = reinterpret_cast<double*>(static_cast<char*>(workspace) + 256);
  a.T = rows; a.ld = ld; a.ldg = grad_ld; a.E = (int)experts; a.k = k; a.given = given; a.alpha = alpha;
  cudaError_t e = cudaMemsetAsync(a.head, 0, sizeof(Head), st);
  if (e == cudaSuccess) e = cudaMemsetAsync(counts, 0, (size_t)experts * 4, st);
  if (e != cudaSuccess) return report_cuda(e);
  const unsigned grid = (unsigned)std::min<int64_t>(std::max<int64_t>((rows + kWarps - 1) / kWarps, 1), kMaxGrid);
  if (dtype == PGC_BF16) choose_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(a);
  else choose_kernel<float><<<grid, kThreads, 0, st>>>(a);
  e = cudaGetLastError();
  if (e != cudaSuccess) return report_cuda(e);
  if (dtype == PGC_BF16) balance_grad_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(a);
  else balance_grad_kernel<float><<<grid, kThreads, 0, st>>>(a);
  return report_cuda(cudaGetLastError());
}

}  // extern "C"
