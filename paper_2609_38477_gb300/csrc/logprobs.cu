// Log probability, rank, entropy and top alternatives of a token under a row of
// logits (seedq_token_logprobs).
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <cmath>

#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = 32;

struct ScoreArgs {
  const void *x;
  int dtype;
  int64_t stride;
  int32_t vocab;
  float scale;
  const int64_t *targets;
  float *logprob, *entropy;
  int32_t *rank;
  int top_k;
  float *top_logprob;
  int32_t *top_index;
};

// A logit's place in the order as a whole number: larger logits first, NaN
// before all, -0 equal to +0, the lower index first among equals.  Never 0.
__device__ __forceinline__ uint64_t order_key(float x, int i) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t u = isnan(x) ? 0xffffffffu : (b >> 31) ? ~b : (b | 0x80000000u);
  return ((uint64_t)u << 32) | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return u == 0xffffffffu ? CUDART_NAN_F : __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u);
}

__device__ float cta_sum(float v, float *sm) {
  sm[threadIdx.x] = v;
  __syncthreads();
  for (int s = kThreads / 2; s; s >>= 1) {
    if (threadIdx.x < s) sm[threadIdx.x] += sm[threadIdx.x + s];
    __syncthreads();
  }
  v = sm[0];
  __syncthreads();
  return v;
}
__device__ uint64_t cta_max(uint64_t v, uint64_t *sm) {
  sm[threadIdx.x] = v;
  __syncthreads();
  for (int s = kThreads / 2; s; s >>= 1) {
    if (threadIdx.x < s) sm[threadIdx.x] = max(sm[threadIdx.x], sm[threadIdx.x + s]);
    __syncthreads();
  }
  v = sm[0];
  __syncthreads();
  return v;
}

// One CTA per row, one pass for the maximum, one for the sums, one per
// alternative.
__global__ void __launch_bounds__(kThreads) k_score(ScoreArgs a) {
  __shared__ float smf[kThreads];
  __shared__ uint64_t smk[kThreads];
  __shared__ int s_rank;
  const int64_t row = blockIdx.x, base = row * a.stride;
  uint64_t best = 0;
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) best = max(best, order_key(load_elem(a.x, a.dtype, base + i), i));
  best = cta_max(best, smk);
  const float m = key_value(best) * a.scale;
  const bool empty = m == -CUDART_INF_F, bad = isnan(m) || m == CUDART_INF_F;
  const int64_t t = a.targets ? a.targets[row] : -1;
  const bool has = t >= 0 && t < a.vocab;
  const float xt = has ? load_elem(a.x, a.dtype, base + t) : 0.f;
  const uint64_t kt = has ? order_key(xt, (int)t) : ~0ull;
  float s1 = 0.f, s2 = 0.f;
  int before = 0;
  for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
    const float x = load_elem(a.x, a.dtype, base + i), d = x * a.scale - m;
    before += order_key(x, i) > kt;
    const float e = expf(d);
    if (e > 0.f) s1 += e, s2 += e * d;
  }
  s1 = cta_sum(s1, smf);
  s2 = cta_sum(s2, smf);
  if (threadIdx.x == 0) s_rank = 0;
  __syncthreads();
  atomicAdd(&s_rank, before);
  __syncthreads();
  const int rank = s_rank;
  const float ln = logf(s1);
  if (threadIdx.x == 0) {
    if (a.entropy) a.entropy[row] = bad ? CUDART_NAN_F : empty ? 0.f : ln - s2 / s1;
    if (a.targets) {
      a.logprob[row] = t == -1 ? 0.f : !has || bad ? CUDART_NAN_F : empty ? -CUDART_INF_F : xt * a.scale - m - ln;
      a.rank[row] = has && !isnan(m) ? rank : -1;
    }
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top_k; ++k) {
    uint64_t b = 0;
    for (int i = threadIdx.x; i < a.vocab; i += kThreads) {
      const uint64_t key = order_key(load_elem(a.x, a.dtype, base + i), i);
      if (key < last) b = max(b, key);
    }
    last = cta_max(b, smk);
    if (threadIdx.x == 0) {
      a.top_index[row * a.top_k + k] = last ? (int)~(uint32_t)last : -1;
      a.top_logprob[row * a.top_k + k] = !last || empty ? -CUDART_INF_F : bad ? CUDART_NAN_F
                                                        : key_value(last) * a.scale - m - ln;
    }
  }
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_token_logprobs_workspace_bytes(int64_t n_rows, int64_t vocab) {
  (void)vocab;
  return n_rows < 0 ? 0 : 16;
}

seedq_status seedq_token_logprobs(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                                  float scale, const int64_t *targets, float *logprob, float *entropy, int32_t *rank,
                                  int32_t top_k, float *top_logprob, int32_t *top_index, void *workspace,
                                  uint64_t workspace_bytes, void *cuda_stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || n_rows > INT32_MAX || vocab < 1 || vocab > (1 << 30) || row_stride < vocab ||
      !std::isfinite(scale) || scale <= 0.f || top_k < 0 || top_k > kMaxTop)
    return SEEDQ_ERR_INVALID_ARG;
  if (n_rows == 0) return SEEDQ_OK;
  if (!logits || (targets && (!logprob || !rank)) || (top_k && (!top_logprob || !top_index)) || !workspace ||
      (uintptr_t)workspace % 16 || workspace_bytes < seedq_token_logprobs_workspace_bytes(n_rows, vocab))
    return SEEDQ_ERR_INVALID_ARG;
  const ScoreArgs a{logits, dtype, row_stride, (int32_t)vocab, scale, targets, logprob, entropy, rank, top_k, top_logprob,
                    top_index};
  k_score<<<(unsigned)n_rows, kThreads, 0, (cudaStream_t)cuda_stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
