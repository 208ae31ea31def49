// The 8-bit paged key/value cache: append (seedq_kv_append) and its inverse
// (seedq_kv_gather).
#include <cuda_runtime.h>
#include <stdint.h>

#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kAppendThreads = 128;

struct AppendArgs {
  seedq_kv_cache c;
  const void *x[2];
  int64_t ts, hs, n;
  const int64_t *slots;
  int dtype;
};

// One CTA per (token, head, tensor); it works if its token is the first of a
// stretch of tokens on one page, and then for the whole stretch, run of
// consecutive slots by run.
template <int KIND>
__global__ void __launch_bounds__(kAppendThreads) k_kv_append(AppendArgs a) {
  int64_t t0 = blockIdx.x;
  const int h = blockIdx.y, which = blockIdx.z;
  const int P = a.c.page_size, D = a.c.head_dim;
  int64_t slot = a.slots[t0];
  const int64_t page = slot >= 0 ? slot / P : -1;
  if (page < 0 || page >= a.c.n_pages) return;
  if (t0 > 0) {
    const int64_t prev = a.slots[t0 - 1];
    if (prev >= 0 && prev / P == page) return;
  }
  const void *x = a.x[which];
  float *scale = (which ? a.c.v_scale : a.c.k_scale) + page * a.c.n_kv_heads + h;
  uint8_t *code = (uint8_t *)(which ? a.c.v : a.c.k) + page * a.c.page_stride + h * a.c.head_stride;
  float old = *scale;
  __shared__ int s_count;
  __shared__ uint32_t s_amax;
  while (true) {
    const int off = (int)(slot - page * P);
    if (threadIdx.x == 0) {
      int m = 1;
      while (off + m < P && t0 + m < a.n && a.slots[t0 + m] == slot + m) ++m;
      s_count = m;
      s_amax = 0;
    }
    __syncthreads();
    const int m = s_count;
    uint32_t amax = 0;
    for (int i = threadIdx.x; i < m * D; i += kAppendThreads) {
      const int t = i / D, d = i - t * D;
      amax = max(amax, __float_as_uint(load_elem(x, a.dtype, (t0 + t) * a.ts + h * a.hs + d)) & 0x7fffffffu);
    }
    atomicMax(&s_amax, amax);
    __syncthreads();
    const float want = block_scale<KIND>(s_amax);
    float now = want;
    if (off > 0 && !(want > old) && !isnan(want)) now = old;  // a NaN scale stays
    if (off > 0 && now > old) {
      const float r = __fdiv_rn(old, now);
      for (int i = threadIdx.x; i < off * D; i += kAppendThreads) {
        const int t = i / D, d = i - t * D;
        uint8_t *p = code + t * a.c.token_stride + d;
        *p = (uint8_t)value_code<KIND>(code_value<KIND>(*p) * r);
      }
    }
    for (int i = threadIdx.x; i < m * D; i += kAppendThreads) {
      const int t = i / D, d = i - t * D;
      const float v = load_elem(x, a.dtype, (t0 + t) * a.ts + h * a.hs + d);
      code[(off + t) * a.c.token_stride + d] = now > 0.f ? (uint8_t)value_code<KIND>(__fdiv_rn(v, now)) : 0;
    }
    old = now;
    t0 += m;
    if (t0 >= a.n) break;
    slot = a.slots[t0];
    if (slot < 0 || slot / P != page) break;
    __syncthreads();
  }
  if (threadIdx.x == 0) *scale = old;
}

template <int KIND>
__global__ void k_kv_gather(AppendArgs a, void *k, void *v) {
  const int64_t t = blockIdx.x;
  const int P = a.c.page_size, D = a.c.head_dim;
  const int64_t slot = a.slots[t];
  const int64_t page = slot >= 0 ? slot / P : -1;
  const bool in = page >= 0 && page < a.c.n_pages;
  for (int i = threadIdx.x; i < a.c.n_kv_heads * D; i += blockDim.x) {
    const int h = i / D, d = i - h * D;
    float x = 0.f, y = 0.f;
    if (in) {
      const int64_t at = page * a.c.page_stride + h * a.c.head_stride + (slot - page * P) * a.c.token_stride + d;
      const int64_t s = page * a.c.n_kv_heads + h;
      x = code_value<KIND>(((const uint8_t *)a.c.k)[at]) * a.c.k_scale[s];
      y = code_value<KIND>(((const uint8_t *)a.c.v)[at]) * a.c.v_scale[s];
    }
    const int64_t o = t * a.ts + h * a.hs + d;
    store_elem(k, a.dtype, o, x);
    store_elem(v, a.dtype, o, y);
  }
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

seedq_status seedq_kv_append(const seedq_kv_cache *cache, const void *k, const void *v, int32_t dtype,
                             int64_t token_stride, int64_t head_stride, const int64_t *slots, int64_t n_tokens,
                             void *cuda_stream) {
  const seedq_status st = kv_check(cache);
  if (st != SEEDQ_OK) return st;
  if (!dtype_ok(dtype) || n_tokens < 0 || n_tokens > INT32_MAX) return SEEDQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return SEEDQ_OK;
  if (!k || !v || !slots) return SEEDQ_ERR_INVALID_ARG;
  const AppendArgs a{*cache, {k, v}, token_stride, head_stride, n_tokens, slots, dtype};
  const dim3 grid((unsigned)n_tokens, cache->n_kv_heads, 2);
  if (cache->kind == SEEDQ_KV_INT8) k_kv_append<SEEDQ_KV_INT8><<<grid, kAppendThreads, 0, (cudaStream_t)cuda_stream>>>(a);
  else k_kv_append<SEEDQ_KV_E4M3><<<grid, kAppendThreads, 0, (cudaStream_t)cuda_stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

seedq_status seedq_kv_gather(const seedq_kv_cache *cache, const int64_t *slots, int64_t n_tokens, void *k, void *v,
                             int32_t dtype, int64_t token_stride, int64_t head_stride, void *cuda_stream) {
  const seedq_status st = kv_check(cache);
  if (st != SEEDQ_OK) return st;
  if (!dtype_ok(dtype) || n_tokens < 0 || n_tokens > INT32_MAX) return SEEDQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return SEEDQ_OK;
  if (!k || !v || !slots) return SEEDQ_ERR_INVALID_ARG;
  const AppendArgs a{*cache, {nullptr, nullptr}, token_stride, head_stride, n_tokens, slots, dtype};
  if (cache->kind == SEEDQ_KV_INT8) k_kv_gather<SEEDQ_KV_INT8><<<(unsigned)n_tokens, 256, 0, (cudaStream_t)cuda_stream>>>(a, k, v);
  else k_kv_gather<SEEDQ_KV_E4M3><<<(unsigned)n_tokens, 256, 0, (cudaStream_t)cuda_stream>>>(a, k, v);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
