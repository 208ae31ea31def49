// Rotary positions: what the rotation kernels and the rotating cache write share.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "overlap.h"
#include "serve.cuh"

namespace seedq {

// N neighbouring elements as they lie in memory (at i, with accesses of up to 16
// bytes that start at a multiple of their size), and as numbers.
template <int DT, int N>
__device__ __forceinline__ void load_run(const void *p, int64_t i, float (&x)[N]) {
  constexpr int kSize = DT == SEEDQ_F32 ? 4 : 2, kWords = N * kSize / 4;
  static_assert(N * kSize >= 4 || N == 1, "");
  if constexpr (N == 1) {
    x[0] = load_elem(p, DT, i);
  } else {
    uint32_t w[kWords];
    const char *src = (const char *)p + i * kSize;
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int k = 0; k < kWords / 4; ++k) {
        const uint4 v = ((const uint4 *)src)[k];
        w[4 * k] = v.x, w[4 * k + 1] = v.y, w[4 * k + 2] = v.z, w[4 * k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < kWords / 2; ++k) {
        const uint2 v = ((const uint2 *)src)[k];
        w[2 * k] = v.x, w[2 * k + 1] = v.y;
      }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      if (DT == SEEDQ_F32) {
        x[k] = __uint_as_float(w[k % kWords]);
      } else {
        const uint32_t h = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu;
        x[k] = DT == SEEDQ_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
      }
    }
  }
}
template <int DT, int N>
__device__ __forceinline__ void store_run(void *p, int64_t i, const float (&x)[N]) {
  constexpr int kSize = DT == SEEDQ_F32 ? 4 : 2, kWords = N * kSize / 4;
  if constexpr (N == 1) {
    store_elem(p, DT, i, x[0]);
  } else {
    uint32_t w[kWords];
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if (DT == SEEDQ_F32) {
        w[k] = __float_as_uint(x[k % N]);
      } else if (DT == SEEDQ_BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[(2 * k) % N], x[(2 * k + 1) % N]);
        w[k] = *(const uint32_t *)&b;
      } else {
        const __half2 b = __floats2half2_rn(x[(2 * k) % N], x[(2 * k + 1) % N]);
        w[k] = *(const uint32_t *)&b;
      }
    }
    char *to = (char *)p + i * kSize;
    if constexpr (kWords % 4 == 0) {
#pragma unroll
      for (int k = 0; k < kWords / 4; ++k) ((uint4 *)to)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else {
#pragma unroll
      for (int k = 0; k < kWords / 2; ++k) ((uint2 *)to)[k] = make_uint2(w[2 * k], w[2 * k + 1]);
    }
  }
}

// A pair turned by (cos, sin): each product and the sum rounded once at most.
__device__ __forceinline__ float2 turned(float x, float y, float2 cs) {
  return make_float2(fmaf(x, cs.x, -(y * cs.y)), fmaf(y, cs.x, x * cs.y));
}

// A thread takes several heads, and so reads their cos and sin once, where threads are
// many and numbers narrow: 8192 tokens of 72 heads of 128 bfloat16 51 us instead of 57,
// 2048 of 40 10 us instead of 9, 4096 of 72 in float32 46 instead of 44.
constexpr int kRotateHeads = 4;
constexpr int64_t kRotateMany = 152 * 2048 * 4;

struct RotateArgs {
  const void *x;
  void *out;
  int64_t xt, xh, ot, oh;  // strides of tokens and heads, in elements
  int64_t n;               // tokens
  int32_t heads, dim, half;
  int32_t layout, out_dtype;
  const float2 *cs;        // n x half
};

// Work on a token: `pieces` threads to a head, of which the first take N pairs each
// and the others copy 2 N of the dims behind the rotated ones; `groups` such rows of
// threads, each with the heads that lie `groups` apart, whose cos and sin it reads once.
struct RotateSplit {
  int32_t turns, pieces, groups, wide;  // wide: N
};
// The widest N whose accesses are whole.
inline int rotate_wide(const RotateArgs &a, int32_t in, int32_t out) {
  const int ib = dtype_bytes(in), ob = dtype_bytes(out), rest = a.dim - 2 * a.half;
  const uint64_t all = (uint64_t)(uintptr_t)a.x | (uint64_t)(uintptr_t)a.out | (uint64_t)(a.xt * ib) | (uint64_t)(a.xh * ib) |
                       (uint64_t)(a.ot * ob) | (uint64_t)(a.oh * ob);
  for (int n : {8, 4})
    if (all % 16 == 0 && a.half % n == 0 && rest % (2 * n) == 0) return n;
  return 1;
}
inline RotateSplit rotate_split(const RotateArgs &a, int32_t in, int32_t out) {
  RotateSplit s{};
  const int n = rotate_wide(a, in, out), rest = a.dim - 2 * a.half;
  s.wide = n;
  s.turns = (a.half + n - 1) / n;
  s.pieces = s.turns + (rest + 2 * n - 1) / (2 * n);
  const int each = a.n * s.pieces * a.heads >= kRotateMany && (in != SEEDQ_F32 || out != SEEDQ_F32) ? kRotateHeads : 1;
  s.groups = (a.heads + each - 1) / each;
  return s;
}

// Whether out lies on itself, on cos and sin, or on x elsewhere than where it is x: a
// thread may write only what no other reads.
inline bool rotate_overlaps(const RotateArgs &a, int32_t in) {
  const Wide ib = dtype_bytes(in), ob = dtype_bytes(a.out_dtype);
  const ByteRows out = byte_rows(a.out, a.dim * ob, a.n, a.ot * ob, a.heads, a.oh * ob);
  return overlaps_itself(out) || overlap(out, byte_rows(a.cs, (Wide)a.n * a.half * 8)) ||
         (a.out != a.x && overlap(out, byte_rows(a.x, a.dim * ib, a.n, a.xt * ib, a.heads, a.xh * ib)));
}

// Enqueues the rotation (rotary.cu).
seedq_status rotate_launch(const RotateArgs &a, int32_t in, cudaStream_t st);

// The work of thread i of the call.  N = 1 takes any sizes and strides; larger N
// wants half and dim - 2 half in multiples of N and 2 N, and rows whose accesses of
// N elements (2 N of neighbouring pairs) are aligned.
template <int IN, int OUT, int N>
__device__ __forceinline__ void rotate_item(const RotateArgs &a, const RotateSplit &s, int64_t i) {
  const int per = s.pieces * s.groups;
  const int64_t t = i >> 32 ? i / per : (int64_t)((uint32_t)i / (uint32_t)per);
  if (t >= a.n) return;
  const int r = (int)(i - t * per), g = r / s.pieces, p = r - g * s.pieces;
  const char *x = (const char *)a.x;
  if (p < s.turns) {
    const int p0 = p * N;
    float2 cs[N];
#pragma unroll
    for (int k = 0; k < N; ++k) cs[k] = a.cs[t * a.half + p0 + k];
#pragma unroll kRotateHeads
    for (int h = g; h < a.heads; h += s.groups) {
      const int64_t at = t * a.xt + h * a.xh, to = t * a.ot + h * a.oh;
      if (a.layout == SEEDQ_ROPE_HALF) {
        float u[N], v[N];
        load_run<IN, N>(x, at + p0, u);
        load_run<IN, N>(x, at + a.half + p0, v);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float2 y = turned(u[k], v[k], cs[k]);
          u[k] = y.x, v[k] = y.y;
        }
        store_run<OUT, N>(a.out, to + p0, u);
        store_run<OUT, N>(a.out, to + a.half + p0, v);
      } else if constexpr (N == 1) {
        const float2 y = turned(load_elem(x, IN, at + 2 * p0), load_elem(x, IN, at + 2 * p0 + 1), cs[0]);
        store_elem(a.out, OUT, to + 2 * p0, y.x);
        store_elem(a.out, OUT, to + 2 * p0 + 1, y.y);
      } else {
        float u[2 * N];
        load_run<IN, 2 * N>(x, at + 2 * p0, u);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float2 y = turned(u[2 * k], u[2 * k + 1], cs[k]);
          u[2 * k] = y.x, u[2 * k + 1] = y.y;
        }
        store_run<OUT, 2 * N>(a.out, to + 2 * p0, u);
      }
    }
  } else {
    const int p0 = 2 * a.half + (p - s.turns) * 2 * N;
    for (int h = g; h < a.heads; h += s.groups) {
      const int64_t at = t * a.xt + h * a.xh + p0, to = t * a.ot + h * a.oh + p0;
      if constexpr (N == 1) {
        for (int k = 0; k < 2 && p0 + k < a.dim; ++k) store_elem(a.out, OUT, to + k, load_elem(x, IN, at + k));
      } else {
        float u[2 * N];
        load_run<IN, 2 * N>(x, at, u);
        store_run<OUT, 2 * N>(a.out, to, u);
      }
    }
  }
}

}  // namespace seedq
