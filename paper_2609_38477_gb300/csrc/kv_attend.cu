// Attention of the newest tokens over the 8-bit paged cache (seedq_kv_attend).
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kWarps = 4;
constexpr int kMaxDim = 256;

// One CTA per (query token, query head): a warp per key, a running maximum and
// sum per warp, joined at the end.
template <int KIND>
__global__ void __launch_bounds__(kWarps * 32) k_attend(seedq_kv_cache c, seedq_attend_args a) {
  const int64_t row = blockIdx.x;
  const int hq = blockIdx.y, h = hq / (a.n_heads / c.n_kv_heads);
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int D = c.head_dim, P = c.page_size;
  if (row < a.starts[0] || row >= a.starts[a.n_requests]) return;
  int lo = 0, hi = a.n_requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.starts[mid] <= row) lo = mid;
    else hi = mid;
  }
  const int first = a.starts[lo], fresh = a.starts[lo + 1] - first;
  const int64_t pos = (int64_t)a.seq_lens[lo] - fresh + (row - first);
  const int64_t end = min(pos + 1, (int64_t)a.table_width * P);
  int64_t j0 = a.window > 0 ? pos - a.window + 1 : 0;
  if (j0 < 0) j0 = 0;
  __shared__ float sm[kWarps], sl[kWarps], so[kWarps][kMaxDim];
  float q[kMaxDim / 32], o[kMaxDim / 32];
  for (int i = 0; i < kMaxDim / 32; ++i) {
    const int d = i * 32 + lane;
    o[i] = 0.f;
    q[i] = d < D ? load_elem(a.q, a.q_dtype, row * a.q_token_stride + hq * a.q_head_stride + d) : 0.f;
  }
  float m = -CUDART_INF_F, l = 0.f;
  for (int64_t j = j0 + w; j < end; j += kWarps) {
    const int64_t page = a.block_table[lo * a.table_stride + j / P];
    if (page < 0 || page >= c.n_pages) continue;
    const int64_t at = page * c.page_stride + h * c.head_stride + (j % P) * c.token_stride;
    const float ks = c.k_scale[page * c.n_kv_heads + h], vs = c.v_scale[page * c.n_kv_heads + h];
    float s = 0.f;
    for (int i = 0; i < kMaxDim / 32; ++i)
      if (i * 32 + lane < D) s += q[i] * code_value<KIND>(((const uint8_t *)c.k)[at + i * 32 + lane]);
    for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(~0u, s, x);
    s *= ks * a.scale;
    const float mn = fmaxf(m, s), corr = expf(m - mn), p = isnan(s) ? s : expf(s - mn);
    m = mn;
    l = l * corr + p;
    for (int i = 0; i < kMaxDim / 32; ++i)
      if (i * 32 + lane < D) o[i] = o[i] * corr + p * vs * code_value<KIND>(((const uint8_t *)c.v)[at + i * 32 + lane]);
  }
  if (lane == 0) sm[w] = m, sl[w] = l;
  for (int i = 0; i < kMaxDim / 32; ++i) so[w][i * 32 + lane] = o[i];
  __syncthreads();
  float M = -CUDART_INF_F, L = 0.f;
  for (int i = 0; i < kWarps; ++i) M = fmaxf(M, sm[i]);
  for (int i = 0; i < kWarps; ++i) L += sl[i] == 0.f ? 0.f : sl[i] * expf(sm[i] - M);
  for (int d = threadIdx.x; d < D; d += blockDim.x) {
    float x = 0.f;
    for (int i = 0; i < kWarps; ++i) x += sl[i] == 0.f ? 0.f : so[i][d] * expf(sm[i] - M);
    store_elem(a.out, a.out_dtype, row * a.out_token_stride + hq * a.out_head_stride + d, L == 0.f ? 0.f : x / L);
  }
  if (threadIdx.x == 0 && a.lse) a.lse[row * a.n_heads + hq] = L == 0.f ? -CUDART_INF_F : M + logf(L);
}

seedq_status check(const seedq_kv_cache *c, int32_t n_heads, int32_t max_new) {
  const seedq_status st = kv_check(c);
  if (st != SEEDQ_OK) return st;
  if (n_heads < 1 || max_new < 1) return SEEDQ_ERR_INVALID_ARG;
  return n_heads % c->n_kv_heads ? SEEDQ_ERR_UNSUPPORTED : SEEDQ_OK;
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_kv_attend_workspace_bytes(const seedq_kv_cache *cache, int32_t n_heads, int32_t max_new) {
  return check(cache, n_heads, max_new) == SEEDQ_OK ? 16 : 0;
}

seedq_status seedq_kv_attend(const seedq_kv_cache *cache, const seedq_attend_args *args, void *cuda_stream) {
  if (!args) return SEEDQ_ERR_INVALID_ARG;
  const seedq_attend_args &a = *args;
  const seedq_status st = check(cache, a.n_heads, a.max_new);
  if (st != SEEDQ_OK) return st;
  if (a.n_requests < 1 || a.n_requests > SEEDQ_MAX_REQUESTS || a.n_tokens < 0 || a.n_tokens > INT32_MAX ||
      !dtype_ok(a.q_dtype) || !dtype_ok(a.out_dtype) || a.table_width < 1 || a.table_width > (1 << 20) ||
      a.table_width > a.table_stride || a.window < 0 || !isfinite(a.scale))
    return SEEDQ_ERR_INVALID_ARG;
  if (a.n_tokens == 0) return SEEDQ_OK;
  if (!a.q || !a.out || !a.seq_lens || !a.starts || !a.block_table || !a.workspace || (uintptr_t)a.workspace % 16 ||
      a.workspace_bytes < seedq_kv_attend_workspace_bytes(cache, a.n_heads, a.max_new))
    return SEEDQ_ERR_INVALID_ARG;
  const dim3 grid((unsigned)a.n_tokens, a.n_heads);
  if (cache->kind == SEEDQ_KV_INT8) k_attend<SEEDQ_KV_INT8><<<grid, kWarps * 32, 0, (cudaStream_t)cuda_stream>>>(*cache, a);
  else k_attend<SEEDQ_KV_E4M3><<<grid, kWarps * 32, 0, (cudaStream_t)cuda_stream>>>(*cache, a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
