// Logits in order: whole numbers that sort as they do, and sorted lists of 32 in
// a warp's lanes.
#pragma once

#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

namespace seedq {

// A logit's place in the order as a whole number: larger logits first, NaN
// before all, -0 equal to +0, the lower index first among equals.  Never 0.
__device__ __forceinline__ uint32_t order_word(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return isnan(x) ? 0xffffffffu : (b >> 31) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_key(float x, int i) { return ((uint64_t)order_word(x) << 32) | (uint32_t)~i; }
__device__ __forceinline__ float key_value(uint64_t key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return u == 0xffffffffu ? CUDART_NAN_F : __uint_as_float((u >> 31) ? (u & 0x7fffffffu) : ~u);
}
__device__ __forceinline__ int key_index(uint64_t key) { return (int)~(uint32_t)key; }

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float y;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b, float c) {
  float y;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// The largest of a warp's, in all lanes; NaN if any is.
__device__ __forceinline__ float warp_max_nan(float x) {
  float y;
  asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A load past the L1 cache: sees what other SMs wrote.
template <typename T>
__device__ __forceinline__ T fresh_load(const T *x) { return *(const volatile T *)x; }

// Both lists' first 32 keys in order: of two descending lists, the larger of a's
// i-th and b's (31 - i)-th are the 32 largest, a bitonic sequence.
static __device__ __noinline__ uint64_t merge_lists(uint64_t a, uint64_t b, int lane) {
  b = __shfl_sync(~0u, b, 31 - lane);
  uint64_t x = a > b ? a : b;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const uint64_t y = __shfl_xor_sync(~0u, x, o);
    x = (lane & o) == 0 ? (x > y ? x : y) : (x < y ? x : y);
  }
  return x;
}

// A warp's keys in descending order (bitonic).
static __device__ __noinline__ uint64_t sort_keys(uint64_t x, int lane) {
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int o = size >> 1; o; o >>= 1) {
      const uint64_t y = __shfl_xor_sync(~0u, x, o);
      const bool larger = ((lane & o) == 0) == ((lane & size) == 0);
      x = (x > y) == larger ? x : y;
    }
  return x;
}

}  // namespace seedq
