// Tokens to their experts and back (pgc_route, pgc_spread, pgc_join, pgc_join_grad).
//
// A router chose k experts for each of T tokens: slot s = t k + j holds an
// expert or nothing.  Slots sorted by expert, in their order within one, give
//   place[s] = offsets[e] + number of slots before s that hold e,
// and, with rows[place[t, j]] the row that expert made of token t,
//   spread     rows[place[t, j]] = x[t]
//   join       y[t] = sum_j w[t, j] rows[place[t, j]]       (weights 1: the gradient of spread)
//   join_grad  drows[place[t, j]] = w[t, j] dy[t],  dw[t, j] = <dy[t], rows[place[t, j]]>.
// All three go through the rows token by token, so that a token's own row is
// read or written once.
#include <algorithm>
#include <cmath>

#include "pgc.h"
#include "pgc_internal.h"
#include "row_slice.cuh"

namespace pgc {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxExperts = 1024, kMaxChoices = 64;

// ---- sorting -------------------------------------------------------------------

struct Route {
  const int32_t* choice;
  int32_t *place, *slot, *offsets;
  int n, E;                     // slots, experts
};
__device__ __forceinline__ int expert_of(const Route& a, int s) {
  const int e = a.choice[s];
  return e >= 0 && e < a.E ? e : -1;
}

// One CTA: counts, their running sum, then 32 slots after another by one warp.
constexpr int kRouteThreads = 1024;
__global__ void __launch_bounds__(kRouteThreads) route_kernel(Route a) {
  __shared__ int next[kMaxExperts];
  __shared__ int total;
  const int tid = threadIdx.x;
  for (int e = tid; e < a.E; e += kRouteThreads) next[e] = 0;
  __syncthreads();
  for (int64_t s = tid; s < a.n; s += kRouteThreads) {
    const int e = expert_of(a, (int)s);
    if (e >= 0) atomicAdd(&next[e], 1);
  }
  __syncthreads();
  if (tid == 0) {
    int sum = 0;
    for (int e = 0; e < a.E; ++e) {
      const int c = next[e];
      a.offsets[e] = next[e] = sum;
      sum += c;
    }
    a.offsets[a.E] = total = sum;
  }
  __syncthreads();
  for (int64_t i = total + (int64_t)tid; i < a.n; i += kRouteThreads) a.slot[i] = -1;
  if (tid >= 32) return;
  for (int64_t s0 = 0; s0 < a.n; s0 += 32) {
    const int64_t s = s0 + tid;
    const int e = s < a.n ? expert_of(a, (int)s) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, e);
    int at = -1;
    if (e >= 0) at = next[e] + __popc(same & ((1u << tid) - 1));
    __syncwarp();
    if (e >= 0) {
      if (tid == __ffs(same) - 1) next[e] += __popc(same);
      a.slot[at] = (int)s;
    }
    if (s < a.n) a.place[s] = at;
    __syncwarp();
  }
}

// ---- rows ----------------------------------------------------------------------

struct Move {
  const void* x;                // spread: tokens; join, join_grad: the experts' rows
  const void* dy;               // join_grad
  void* out;                    // spread: the experts' rows; join: tokens; join_grad: gradient of the experts' rows
  const int32_t* place;
  const float* weight;
  float* dweight;
  int64_t T, rows, ldx, ldy, ldo;
  int k, d;
};
__device__ __forceinline__ int64_t row_of(const Move& a, int64_t slot) {
  const int at = a.place[slot];
  return at >= 0 && at < a.rows ? at : -1;
}

template <typename E>
__global__ void __launch_bounds__(kThreads) spread_kernel(Move a) {
  const int64_t t = blockIdx.x;
  const E* x = static_cast<const E*>(a.x) + t * a.ldx;
  for (int j = 0; j < a.k; ++j) {
    const int64_t r = row_of(a, t * a.k + j);
    if (r < 0) continue;
    E* out = static_cast<E*>(a.out) + r * a.ldo;
    for (unsigned c = threadIdx.x; c < (unsigned)a.d; c += kThreads) out[c] = x[c];
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) join_kernel(Move a) {
  const int64_t t = blockIdx.x;
  E* out = static_cast<E*>(a.out) + t * a.ldo;
  for (unsigned c = threadIdx.x; c < (unsigned)a.d; c += kThreads) {
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const int64_t r = row_of(a, t * a.k + j);
      if (r < 0) continue;
      const float f = Elem<E>::get(static_cast<const E*>(a.x) + r * a.ldx + c);
      sum = a.weight ? fmaf(a.weight[t * a.k + j], f, sum) : sum + f;
    }
    Elem<E>::put(out + c, sum);
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) join_grad_kernel(Move a) {
  __shared__ float red[kThreads / 32];
  const int64_t t = blockIdx.x;
  const E* dy = static_cast<const E*>(a.dy) + t * a.ldy;
  for (int j = 0; j < a.k; ++j) {
    const int64_t r = row_of(a, t * a.k + j);
    float sum = 0.f;
    if (r >= 0) {
      const float w = a.weight[t * a.k + j];
      const E* x = static_cast<const E*>(a.x) + r * a.ldx;
      E* out = static_cast<E*>(a.out) + r * a.ldo;
      for (unsigned c = threadIdx.x; c < (unsigned)a.d; c += kThreads) {
        const float f = Elem<E>::get(dy + c);
        sum = fmaf(f, Elem<E>::get(x + c), sum);
        Elem<E>::put(out + c, w * f);
      }
    }
    sum = warp_sum(sum);
    __syncthreads();
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      sum = 0.f;
      for (int i = 0; i < kThreads / 32; ++i) sum += red[i];
      a.dweight[t * a.k + j] = sum;
    }
  }
}

// ---- host --------------------------------------------------------------------

constexpr int64_t kFar = int64_t(1) << 31;

int check_sizes(int64_t tokens, int32_t k) {
  if (tokens < 0 || k < 1 || tokens > INT32_MAX / k) return PGC_EINVAL;
  return k > kMaxChoices ? PGC_ENOTSUP : PGC_OK;
}
// Rows of d elements: `count` of them at p, each `ld` behind the last.
bool bad_rows(const void* p, int64_t count, int64_t d, int64_t ld, uintptr_t size) {
  return ld < d || ld > kFar || (count && !p) || (uintptr_t)p % size;
}
int check_move(int32_t dtype, int64_t tokens, int32_t k, int64_t d, int64_t rows, const int32_t* place) {
  if (dtype != PGC_F32 && dtype != PGC_BF16) return PGC_EINVAL;
  if (tokens < 0 || k < 1 || tokens > INT32_MAX / k || d < 1 || d > INT32_MAX || rows < 0 || rows > INT32_MAX) return PGC_EINVAL;
  return (tokens && !place) || (uintptr_t)place % 4 ? PGC_EINVAL : PGC_OK;
}

}  // namespace
}  // namespace pgc

using namespace pgc;

extern "C" {

int pgc_route_workspace(int64_t tokens, int32_t k, int32_t experts, int64_t *bytes) {
  if (!bytes || tokens < 0 || k < 1 || tokens > INT32_MAX / k || experts < 1) return PGC_EINVAL;
  if (experts > kMaxExperts || k > kMaxChoices) return PGC_ENOTSUP;
  *bytes = 16;
  return PGC_OK;
}

int pgc_route(int64_t tokens, int32_t k, int32_t experts, const int32_t *choice, int32_t *place, int32_t *slot,
              int32_t *offsets, void *workspace, int64_t workspace_bytes, void *stream) {
  int64_t need = 0;
  const int rc = pgc_route_workspace(tokens, k, experts, &need);
  if (rc) return rc;
  if (!offsets || (tokens && (!choice || !place || !slot)) || !workspace) return PGC_EINVAL;
  if ((uintptr_t)choice % 4 || (uintptr_t)place % 4 || (uintptr_t)slot % 4 || (uintptr_t)offsets % 4 || (uintptr_t)workspace % 16)
    return PGC_EINVAL;
  if (workspace_bytes < need) return PGC_ESCRATCH;
  route_kernel<<<1, kRouteThreads, 0, (cudaStream_t)stream>>>(Route{choice, place, slot, offsets, (int)(tokens * k), experts});
  return report_cuda(cudaGetLastError());
}

int pgc_spread(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *x, int64_t ld, const int32_t *place,
               int64_t rows, void *out, int64_t out_ld, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(x, tokens, d, ld, size) || bad_rows(out, rows, d, out_ld, size)) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens || !rows) return rc;
  Move a{};
  a.x = x; a.out = out; a.place = place; a.T = tokens; a.rows = rows; a.ldx = ld; a.ldo = out_ld; a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PGC_BF16) spread_kernel<__nv_bfloat16><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  else spread_kernel<float><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  return report_cuda(cudaGetLastError());
}

int pgc_join(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *rows_in, int64_t ld, int64_t rows,
             const int32_t *place, const float *weight, void *out, int64_t out_ld, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(rows_in, rows, d, ld, size) || bad_rows(out, tokens, d, out_ld, size) || (uintptr_t)weight % 4) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens) return rc;
  Move a{};
  a.x = rows_in; a.out = out; a.place = place; a.weight = weight; a.T = tokens; a.rows = rows; a.ldx = ld; a.ldo = out_ld;
  a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PGC_BF16) join_kernel<__nv_bfloat16><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  else join_kernel<float><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  return report_cuda(cudaGetLastError());
}

int pgc_join_grad(int32_t dtype, int64_t tokens, int32_t k, int64_t d, const void *dy, int64_t dy_ld, const void *rows_in,
                  int64_t ld, int64_t rows, const int32_t *place, const float *weight, void *drows, int64_t drows_ld,
                  float *dweight, void *stream) {
  int rc = check_move(dtype, tokens, k, d, rows, place);
  if (rc) return rc;
  const uintptr_t size = dtype == PGC_BF16 ? 2 : 4;
  if (bad_rows(dy, tokens, d, dy_ld, size) || bad_rows(rows_in, rows, d, ld, size) || bad_rows(drows, rows, d, drows_ld, size))
    return PGC_EINVAL;
  if ((tokens && (!weight || !dweight)) || (uintptr_t)weight % 4 || (uintptr_t)dweight % 4) return PGC_EINVAL;
  if (drows && drows == rows_in && drows_ld != ld) return PGC_EINVAL;
  rc = check_sizes(tokens, k);
  if (rc || !tokens) return rc;
  Move a{};
  a.x = rows_in; a.dy = dy; a.out = drows; a.place = place; a.weight = weight; a.dweight = dweight;
  a.T = tokens; a.rows = rows; a.ldx = ld; a.ldy = dy_ld; a.ldo = drows_ld; a.k = k; a.d = (int)d;
  const cudaStream_t st = (cudaStream_t)stream;
  if (dtype == PGC_BF16) join_grad_kernel<__nv_bfloat16><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  else join_grad_kernel<float><<<(unsigned)tokens, kThreads, 0, st>>>(a);
  return report_cuda(cudaGetLastError());
}

}  // extern "C"
