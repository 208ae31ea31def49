// Rotary positions: cos and sin of a step's positions (seedq_rotary_angles), and
// queries and keys turned by them (seedq_rotate).
//
// An angle is position * frequency, of which only the fraction of a turn matters.
// Frequencies are kept in turns as whole numbers F = round(w / 2 pi * 2^64), so the
// fraction is the product modulo 2^64: exact for that F at any position, where a float32
// product of position 131072 is off by 2^-8.  All 64 bits of it are used: of the slowest
// pair of base 5e5 the first position's angle is 1678 units of 2^-32 turns.
//
// Bytes bound the rotation (8192 tokens of 72 heads of 128, bfloat16: 50 us, 6.0 TB/s,
// 91% of the copy rate), launch a step's (16 tokens of 40 heads: 2.4 us, the angles
// 1.6).  A thread moves 16 bytes (8 pairs of 16-bit numbers in two pieces, or 8
// neighbouring pairs); 8 bytes took 72 us.
#include "rotary.cuh"

#include <algorithm>

namespace seedq {
namespace {

// cos and sin of f turns, f in units of 2^-64: the nearest quarter of a turn comes off as a
// whole number, and the rest, at most an eighth, rounds to float32 once: the sine of a small
// angle is as exact, relative to itself, as that of a large one.
__device__ __forceinline__ float2 cos_sin_of(uint64_t f) {
  const uint32_t quarter = (uint32_t)((f + (1ull << 61)) >> 62);
  const int64_t rest = (int64_t)(f - ((uint64_t)quarter << 62));  // -2^61 .. 2^61 - 1 of 2^64 to the turn
  float s, c;
  sincospif((float)rest * 0x1p-63f, &s, &c);
  switch (quarter & 3) {
    case 0: return make_float2(c, s);
    case 1: return make_float2(-s, c);
    case 2: return make_float2(-c, -s);
    default: return make_float2(s, -c);
  }
}

__global__ void __launch_bounds__(256) k_rotary_angles(const uint64_t *__restrict__ turns, int half, float scale,
                                                       const int32_t *__restrict__ positions, int64_t n, float2 *__restrict__ cs) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = i >> 32 ? i / half : (int64_t)((uint32_t)i / (uint32_t)half);
  if (t >= n) return;
  const float2 y = cos_sin_of((uint64_t)(int64_t)positions[t] * turns[i - t * half]);
  cs[i] = make_float2(scale * y.x, scale * y.y);
}

template <int IN, int OUT, int N>
__global__ void __launch_bounds__(256) k_rotate(const __grid_constant__ RotateArgs a, const __grid_constant__ RotateSplit s) {
  rotate_item<IN, OUT, N>(a, s, (int64_t)blockIdx.x * blockDim.x + threadIdx.x);
}

int64_t rotate_ctas(const RotateArgs &a, const RotateSplit &s) { return (a.n * s.pieces * s.groups + 255) / 256; }

template <int IN, int OUT>
seedq_status launch(const RotateArgs &a, cudaStream_t st) {
  const RotateSplit s = rotate_split(a, IN, OUT);
  const int64_t ctas = rotate_ctas(a, s);
  if (ctas > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  if (s.wide == 8) k_rotate<IN, OUT, 8><<<(unsigned)ctas, 256, 0, st>>>(a, s);
  else if (s.wide == 4) k_rotate<IN, OUT, 4><<<(unsigned)ctas, 256, 0, st>>>(a, s);
  else k_rotate<IN, OUT, 1><<<(unsigned)ctas, 256, 0, st>>>(a, s);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // namespace

seedq_status rotate_launch(const RotateArgs &a, int32_t in, cudaStream_t st) {
  using Launch = seedq_status (*)(const RotateArgs &, cudaStream_t);
  static constexpr Launch kLaunch[3][3] = {{launch<0, 0>, launch<0, 1>, launch<0, 2>},
                                           {launch<1, 0>, launch<1, 1>, launch<1, 2>},
                                           {launch<2, 0>, launch<2, 1>, launch<2, 2>}};
  return kLaunch[in][a.out_dtype](a, st);
}

}  // namespace seedq

using namespace seedq;

extern "C" {

seedq_status seedq_rotary_angles(const uint64_t *turns, int32_t half, float scale, const int32_t *positions, int64_t n_tokens,
                                 float *cos_sin, void *cuda_stream) {
  if (half < 1 || half > SEEDQ_ROPE_MAX_DIM / 2 || n_tokens < 0 || n_tokens > INT32_MAX || !(scale - scale == 0.f))
    return SEEDQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return SEEDQ_OK;
  if (!turns || !positions || !cos_sin || (uintptr_t)cos_sin % 8) return SEEDQ_ERR_INVALID_ARG;
  const int64_t ctas = (n_tokens * half + 255) / 256;
  if (ctas > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  const ByteRows out = byte_rows(cos_sin, (Wide)n_tokens * half * 8);
  if (overlap(out, byte_rows(positions, (Wide)n_tokens * 4)) || overlap(out, byte_rows(turns, (Wide)half * 8))) return SEEDQ_ERR_INVALID_ARG;
  k_rotary_angles<<<(unsigned)ctas, 256, 0, (cudaStream_t)cuda_stream>>>(turns, half, scale, positions, n_tokens, (float2 *)cos_sin);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

seedq_status seedq_rotate(const void *x, int32_t x_dtype, int64_t x_token_stride, int64_t x_head_stride, int64_t n_tokens,
                          int32_t n_heads, int32_t head_dim, int32_t rot_dim, int32_t layout, const float *cos_sin, void *out,
                          int32_t out_dtype, int64_t out_token_stride, int64_t out_head_stride, void *cuda_stream) {
  if (!dtype_ok(x_dtype) || !dtype_ok(out_dtype) || !rope_ok(layout, rot_dim, head_dim) || n_tokens < 0 || n_tokens > INT32_MAX ||
      n_heads < 0 || n_heads > SEEDQ_ROPE_MAX_HEADS)
    return SEEDQ_ERR_INVALID_ARG;
  if (n_tokens == 0 || n_heads == 0) return SEEDQ_OK;
  if (!x || !out || !cos_sin || (uintptr_t)cos_sin % 8) return SEEDQ_ERR_INVALID_ARG;
  if (x == out && (x_dtype != out_dtype || x_token_stride != out_token_stride || x_head_stride != out_head_stride))
    return SEEDQ_ERR_INVALID_ARG;
  const RotateArgs a{x, out, x_token_stride, x_head_stride, out_token_stride, out_head_stride, n_tokens, n_heads, head_dim,
                     rot_dim / 2, layout, out_dtype, (const float2 *)cos_sin};
  if (rotate_ctas(a, rotate_split(a, x_dtype, out_dtype)) > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  if (rotate_overlaps(a, x_dtype)) return SEEDQ_ERR_INVALID_ARG;
  return rotate_launch(a, x_dtype, (cudaStream_t)cuda_stream);
}

}  // extern "C"
