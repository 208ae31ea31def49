// Device helpers shared by the serving kernels (cache, attention, log
// probabilities): element types and the 8-bit codes.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/seedq.h"

namespace seedq {

seedq_status cuda_fail(cudaError_t e);  // records the message, returns SEEDQ_ERR_CUDA

inline bool dtype_ok(int32_t d) { return d >= SEEDQ_F32 && d <= SEEDQ_F16; }
__host__ __device__ inline int dtype_bytes(int32_t d) { return d == SEEDQ_F32 ? 4 : 2; }

// Element i of an array of type dt, and its rounding store.
__device__ __forceinline__ float load_elem(const void *p, int dt, int64_t i) {
  if (dt == SEEDQ_F32) return ((const float *)p)[i];
  if (dt == SEEDQ_BF16) return __bfloat162float(((const __nv_bfloat16 *)p)[i]);
  return __half2float(((const __half *)p)[i]);
}
__device__ __forceinline__ void store_elem(void *p, int dt, int64_t i, float x) {
  if (dt == SEEDQ_F32) ((float *)p)[i] = x;
  else if (dt == SEEDQ_BF16) ((__nv_bfloat16 *)p)[i] = __float2bfloat16_rn(x);
  else ((__half *)p)[i] = __float2half_rn(x);
}

// Two E4M3 codes as binary16 numbers (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
  return h;
}
// The number an 8-bit code stands for.
template <int KIND>
__device__ __forceinline__ float code_value(uint32_t b) {
  if (KIND == SEEDQ_KV_INT8) return (float)(int8_t)b;
  return __half2float(__ushort_as_half((unsigned short)e4m3x2_to_half2(b & 0xffu)));
}
// The code of x / s, |x / s| at most 127 or 448 by the choice of s; nearest even.
template <int KIND>
__device__ __forceinline__ uint32_t value_code(float r) {
  if (KIND == SEEDQ_KV_INT8) return (uint32_t)(int)fminf(fmaxf(rintf(r), -127.f), 127.f) & 0xffu;
  return (uint32_t)__nv_cvt_float_to_fp8(r, __NV_SATFINITE, __NV_E4M3);
}

// The smallest power of two s >= 2^-126 with a <= 127 s (int8) or 448 s (E4M3),
// from the bits of a >= 0: 127 = 1.984375 * 2^6 and 448 = 1.75 * 2^8, so the
// exponent is a's less 6 or 8, one more if a's fraction is above theirs.
// 0 for a = 0; NaN for an infinity or a NaN.
template <int KIND>
__device__ __forceinline__ float block_scale(uint32_t abits) {
  if (abits == 0) return 0.f;
  if (abits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  constexpr int shift = KIND == SEEDQ_KV_INT8 ? 6 : 8;
  constexpr uint32_t top = KIND == SEEDQ_KV_INT8 ? 0x7e0000u : 0x600000u;
  int e = (int)(abits >> 23) - shift + ((abits & 0x7fffffu) > top ? 1 : 0);  // biased
  if (e < 1) e = 1;
  return __uint_as_float((uint32_t)e << 23);
}

inline bool rope_ok(int32_t layout, int32_t rot_dim, int32_t head_dim) {
  return (layout == SEEDQ_ROPE_HALF || layout == SEEDQ_ROPE_PAIRS) && head_dim <= SEEDQ_ROPE_MAX_DIM && rot_dim >= 2 &&
         rot_dim <= head_dim && rot_dim % 2 == 0;
}

inline int log2_of(int x) {  // -1 if x is no power of two
  if (x & (x - 1)) return -1;
  int n = 0;
  while (x >>= 1) ++n;
  return n;
}

// What the cache calls refuse.
inline seedq_status kv_check(const seedq_kv_cache *c) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return SEEDQ_ERR_INVALID_ARG;
  if (c->kind != SEEDQ_KV_INT8 && c->kind != SEEDQ_KV_E4M3) return SEEDQ_ERR_INVALID_ARG;
  if (c->n_kv_heads < 1 || c->n_pages < 1 || c->n_pages > INT32_MAX) return SEEDQ_ERR_INVALID_ARG;
  if (c->n_kv_heads > 1024) return SEEDQ_ERR_UNSUPPORTED;
  if (c->head_dim < 16 || c->head_dim > 256 || c->head_dim % 16) return SEEDQ_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || c->page_size % 16) return SEEDQ_ERR_UNSUPPORTED;
  for (int64_t s : {c->page_stride, c->head_stride, c->token_stride})
    if (s < c->head_dim || s % 16) return SEEDQ_ERR_UNSUPPORTED;
  if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) return SEEDQ_ERR_UNSUPPORTED;
  return SEEDQ_OK;
}

}  // namespace seedq
