// The 8-bit paged key/value cache: append (seedq_kv_append) and its inverse
// (seedq_kv_gather).
#include <cuda_runtime.h>
#include <stdint.h>

#include "serve.cuh"

namespace seedq {
namespace {

struct CacheArgs {
  seedq_kv_cache c;
  void *x[2];          // the tokens' keys and values
  int64_t ts, hs, n;   // their strides (elements) and number
  const int64_t *slots;
  int32_t vec;         // rows of x allow 16-byte accesses
  int32_t group_shift; // append: log2 of the tokens of a CTA
  int32_t page_shift;  // log2 of the page size, -1 if it is no power of two
};

__device__ __forceinline__ int64_t page_of(const CacheArgs &a, int64_t slot) {  // -1 for a negative slot
  if (slot < 0) return -1;
  return a.page_shift >= 0 ? slot >> a.page_shift : slot / a.c.page_size;
}

// Eight elements in a row, as they lie in memory and as numbers.
template <int DT>
struct Eight {
  static constexpr int kWords = DT == SEEDQ_F32 ? 8 : 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void *p, int64_t i, bool vec) {
    if (vec) {
      const uint4 *src = (const uint4 *)((const char *)p + i * (DT == SEEDQ_F32 ? 4 : 2));
#pragma unroll
      for (int k = 0; k < kWords / 4; ++k) {
        const uint4 v = __ldg(src + k);
        w[4 * k] = v.x, w[4 * k + 1] = v.y, w[4 * k + 2] = v.z, w[4 * k + 3] = v.w;
      }
    } else if (DT == SEEDQ_F32) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) w[k] = ((const uint32_t *)p)[i + k];
    } else {
#pragma unroll
      for (int k = 0; k < kWords; ++k)
        w[k] = (uint32_t)((const uint16_t *)p)[i + 2 * k] | (uint32_t)((const uint16_t *)p)[i + 2 * k + 1] << 16;
    }
  }
  __device__ __forceinline__ float get(int k) const {
    if (DT == SEEDQ_F32) return __uint_as_float(w[k]);
    const uint32_t h = k & 1 ? w[k / 2] >> 16 : w[k / 2] & 0xffffu;
    if (DT == SEEDQ_BF16) return __uint_as_float(h << 16);
    return __half2float(__ushort_as_half((unsigned short)h));
  }
  __device__ __forceinline__ void store(void *p, int64_t i, const float (&v)[8], bool vec) const {
    uint32_t y[kWords];
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if (DT == SEEDQ_F32) {
        y[k] = __float_as_uint(v[k]);
      } else if (DT == SEEDQ_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k % 8], v[(2 * k + 1) % 8]);
        y[k] = *(const uint32_t *)&h;
      } else {
        const __half2 h = __floats2half2_rn(v[2 * k % 8], v[(2 * k + 1) % 8]);
        y[k] = *(const uint32_t *)&h;
      }
    }
    if (vec) {
      uint4 *dst = (uint4 *)((char *)p + i * (DT == SEEDQ_F32 ? 4 : 2));
#pragma unroll
      for (int k = 0; k < kWords / 4; ++k) dst[k] = make_uint4(y[4 * k], y[4 * k + 1], y[4 * k + 2], y[4 * k + 3]);
    } else if (DT == SEEDQ_F32) {
#pragma unroll
      for (int k = 0; k < kWords; ++k) ((uint32_t *)p)[i + k] = y[k];
    } else {
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        ((uint16_t *)p)[i + 2 * k] = (uint16_t)y[k];
        ((uint16_t *)p)[i + 2 * k + 1] = (uint16_t)(y[k] >> 16);
      }
    }
  }
};

// ---------------------------------------------------------------- append
//
// A page's tokens are read, their largest magnitude is found over a warp, and
// the codes are written.  Bytes bound it for prompts, latency for a decode step
// (slots, then scale and tokens, then codes), so the work is cut for many warps
// and no barrier: a warp owns one head and tensor of the stretches of tokens on
// one page that begin among 2^group_shift tokens.  A lane takes 8 elements of a
// token; the first kHeld steps of the warp stay in registers between the maximum
// and the codes (16 tokens of 128 head dims, 8 in float32), longer runs are read
// again, from cache.
constexpr int kAppendWarps = 4;
constexpr int kAppendBlocks = 7;  // per SM: 28 warps of up to 73 registers

template <int KIND, int DT>
__global__ void __launch_bounds__(kAppendWarps * 32, kAppendBlocks) k_kv_append(const __grid_constant__ CacheArgs a) {
  constexpr int kHeld = DT == SEEDQ_F32 ? 4 : 8;
  const int lane = threadIdx.x & 31;
  const int P = a.c.page_size, D = a.c.head_dim, per = D / 8;  // pieces of a token
  int64_t id = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  const int pair = (int)(id % (2 * a.c.n_kv_heads)), h = pair >> 1, which = pair & 1;
  const int64_t g0 = id / (2 * a.c.n_kv_heads) << a.group_shift;
  const int64_t g1 = min(g0 + (1 << a.group_shift), a.n);
  if (g0 >= a.n) return;
  // Stretches begin where the page differs from the token's before: a lane per token.
  uint32_t starts;
  {
    const int64_t t = g0 + lane;
    const int64_t page = t < g1 ? page_of(a, a.slots[t]) : -1;
    int64_t before = __shfl_up_sync(~0u, page, 1);
    if (lane == 0) before = g0 > 0 ? page_of(a, a.slots[g0 - 1]) : -1;
    starts = __ballot_sync(~0u, page >= 0 && page < a.c.n_pages && page != before);
  }
  const void *x = a.x[which];
  const int step = 32 / per, t_first = lane / per, d = (lane - t_first * per) * 8;  // tokens of a step; the lane's piece
  const bool idle = t_first >= step;
  const int64_t ts = a.c.token_stride;

  for (; starts; starts &= starts - 1) {
    int64_t t0 = g0 + __ffs(starts) - 1;
    int64_t slot = a.slots[t0];
    const int64_t page = page_of(a, slot);
    float *scale = (which ? a.c.v_scale : a.c.k_scale) + page * a.c.n_kv_heads + h;
    uint8_t *code = (uint8_t *)(which ? a.c.v : a.c.k) + page * a.c.page_stride + h * a.c.head_stride + d;
    float old = *scale;
    do {  // runs of consecutive slots on the page
      const int off = (int)(slot - page * P);
      // the run's length: up to the first of the next tokens whose slot does not follow, found 32 at a time
      int m = 1;
      const int most = (int)min((int64_t)(P - off), a.n - t0);
      while (m < most) {
        const bool follows = m + lane < most && a.slots[t0 + m + lane] == slot + m + lane;
        const uint32_t stop = __ballot_sync(~0u, !follows);
        m += stop ? __ffs(stop) - 1 : 32;
        if (stop) break;
      }
      const int64_t at = t0 * a.ts + h * a.hs + d;
      const int mine = idle ? 0 : m;
      Eight<DT> held[kHeld];
      uint32_t amax = 0;
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (t_first + k * step < mine) held[k].load(x, at + (t_first + k * step) * a.ts, a.vec);
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (t_first + k * step < mine)
#pragma unroll
          for (int y = 0; y < 8; ++y) amax = max(amax, __float_as_uint(held[k].get(y)) & 0x7fffffffu);
#pragma unroll 4
      for (int t = t_first + kHeld * step; t < mine; t += step) {
        Eight<DT> e;
        e.load(x, at + t * a.ts, a.vec);
#pragma unroll
        for (int y = 0; y < 8; ++y) amax = max(amax, __float_as_uint(e.get(y)) & 0x7fffffffu);
      }
      const float want = block_scale<KIND>(__reduce_max_sync(~0u, amax));
      float now = want;
      if (off > 0 && !(want > old) && !isnan(want)) now = old;  // a NaN scale stays
      if (off > 0 && now > old) {
        const float r = __fdiv_rn(old, now);
#pragma unroll 4
        for (int t = t_first; t < (idle ? 0 : off); t += step) {
          uint2 *p = (uint2 *)(code + t * ts);
          const uint2 v = *p;
          const uint32_t y[2] = {v.x, v.y};
          uint32_t z[2] = {0, 0};
#pragma unroll
          for (int k = 0; k < 8; ++k)
            z[k / 4] |= value_code<KIND>(code_value<KIND>(y[k / 4] >> 8 * (k & 3) & 0xffu) * r) << 8 * (k & 3);
          *p = make_uint2(z[0], z[1]);
        }
      }
      // x / now; by the reciprocal where that is exact: now a power of two whose reciprocal is a normal number
      const uint32_t nb = __float_as_uint(now);
      const bool exact = (nb & 0x7fffffu) == 0 && nb < 0x7f000000u && nb != 0;
      const float inv = exact ? __uint_as_float(0x7f000000u - nb) : 0.f;
      auto write = [&](const Eight<DT> &e, int t) {
        uint32_t z[2] = {0, 0};
        if (exact) {
#pragma unroll
          for (int k = 0; k < 8; ++k) z[k / 4] |= value_code<KIND>(e.get(k) * inv) << 8 * (k & 3);
        } else if (now > 0.f) {
#pragma unroll 1
          for (int k = 0; k < 8; ++k) {
            const uint32_t c = value_code<KIND>(__fdiv_rn(load_elem(x, DT, at + t * a.ts + k), now)) << 8 * (k & 3);
            if (k < 4) z[0] |= c;
            else z[1] |= c;
          }
        }
        *(uint2 *)(code + (off + t) * ts) = make_uint2(z[0], z[1]);
      };
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (t_first + k * step < mine) write(held[k], t_first + k * step);
#pragma unroll 2
      for (int t = t_first + kHeld * step; t < mine; t += step) {
        Eight<DT> e;
        e.load(x, at + t * a.ts, a.vec);
        write(e, t);
      }
      old = now;
      t0 += m;
      slot = t0 < a.n ? a.slots[t0] : -1;
      __syncwarp();
    } while (page_of(a, slot) == page);
    if (lane == 0) *scale = old;
  }
}

// ---------------------------------------------------------------- gather
//
// A thread takes 16 codes of a key and of a value; bytes bound it.
template <int KIND, int DT>
__global__ void __launch_bounds__(256) k_kv_gather(const __grid_constant__ CacheArgs a) {
  const int P = a.c.page_size, per = a.c.head_dim / 16;
  const int row = a.c.n_kv_heads * per;  // threads of a token
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = i >> 32 ? i / row : (int64_t)((uint32_t)i / (uint32_t)row);
  if (t >= a.n) return;
  const int r = (int)(i - t * row), h = r / per, d = (r - h * per) * 16;
  const int64_t slot = a.slots[t];
  const int64_t page = page_of(a, slot);
  uint4 code[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  float scale[2] = {0.f, 0.f};
  if (page >= 0 && page < a.c.n_pages) {
    const int64_t at = page * a.c.page_stride + h * a.c.head_stride + (slot - page * P) * a.c.token_stride + d;
    const int64_t s = page * a.c.n_kv_heads + h;
    code[0] = *(const uint4 *)((const uint8_t *)a.c.k + at);
    code[1] = *(const uint4 *)((const uint8_t *)a.c.v + at);
    scale[0] = a.c.k_scale[s];
    scale[1] = a.c.v_scale[s];
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint32_t w[4] = {code[which].x, code[which].y, code[which].z, code[which].w};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = code_value<KIND>(w[half * 2 + k / 4] >> 8 * (k & 3) & 0xffu) * scale[which];
      Eight<DT>().store(a.x[which], t * a.ts + h * a.hs + d + half * 8, v, a.vec);
    }
  }
}

bool rows_aligned(const void *k, const void *v, int32_t dtype, int64_t ts, int64_t hs) {
  const int64_t per = 16 / dtype_bytes(dtype);
  return ((uintptr_t)k | (uintptr_t)v) % 16 == 0 && ts % per == 0 && hs % per == 0;
}

template <int KIND, int DT>
void launch_append(const CacheArgs &a, cudaStream_t st) {
  const int64_t warps = ((a.n + (1 << a.group_shift) - 1) >> a.group_shift) * a.c.n_kv_heads * 2;
  k_kv_append<KIND, DT><<<(unsigned)((warps + kAppendWarps - 1) / kAppendWarps), kAppendWarps * 32, 0, st>>>(a);
}
template <int KIND, int DT>
void launch_gather(const CacheArgs &a, cudaStream_t st) {
  const int64_t threads = a.n * a.c.n_kv_heads * (a.c.head_dim / 16);
  k_kv_gather<KIND, DT><<<(unsigned)((threads + 255) / 256), 256, 0, st>>>(a);
}
using Launch = void (*)(const CacheArgs &, cudaStream_t);
constexpr Launch kAppend[2][3] = {
    {launch_append<0, 0>, launch_append<0, 1>, launch_append<0, 2>}, {launch_append<1, 0>, launch_append<1, 1>, launch_append<1, 2>}};
constexpr Launch kGather[2][3] = {
    {launch_gather<0, 0>, launch_gather<0, 1>, launch_gather<0, 2>}, {launch_gather<1, 0>, launch_gather<1, 1>, launch_gather<1, 2>}};

// What both calls check and set up; a.n is 0 where there is nothing to do.
seedq_status prepare(const seedq_kv_cache *c, const void *k, const void *v, int32_t dtype, int64_t ts, int64_t hs,
                     const int64_t *slots, int64_t n, CacheArgs &a) {
  const seedq_status st = kv_check(c);
  if (st != SEEDQ_OK) return st;
  if (!dtype_ok(dtype) || n < 0 || n > INT32_MAX) return SEEDQ_ERR_INVALID_ARG;
  if (n > 0 && (!k || !v || !slots)) return SEEDQ_ERR_INVALID_ARG;
  a = CacheArgs{*c, {(void *)k, (void *)v}, ts, hs, n, slots, rows_aligned(k, v, dtype, ts, hs), 0, log2_of(c->page_size)};
  return SEEDQ_OK;
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

seedq_status seedq_kv_append(const seedq_kv_cache *cache, const void *k, const void *v, int32_t dtype,
                             int64_t token_stride, int64_t head_stride, const int64_t *slots, int64_t n_tokens,
                             void *cuda_stream) {
  CacheArgs a;
  const seedq_status st = prepare(cache, k, v, dtype, token_stride, head_stride, slots, n_tokens, a);
  if (st != SEEDQ_OK || n_tokens == 0) return st;
  // One token per warp until the warps fill the GPU twice over, then more.  Each may
  // be a page of its own (32 heads, 256 single tokens: 13 us, 14 with one token per
  // warp, 17 at half the threshold, 57 with 32 tokens), or all on a page (4 prompts
  // of 1024, pages of 64: 39 us, with one token per warp 100).
  a.group_shift = 0;
  while (a.group_shift < 5 && (n_tokens >> a.group_shift) * cache->n_kv_heads * 2 > 2 * 152 * 48) ++a.group_shift;
  kAppend[cache->kind][dtype](a, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

seedq_status seedq_kv_gather(const seedq_kv_cache *cache, const int64_t *slots, int64_t n_tokens, void *k, void *v,
                             int32_t dtype, int64_t token_stride, int64_t head_stride, void *cuda_stream) {
  CacheArgs a;
  const seedq_status st = prepare(cache, k, v, dtype, token_stride, head_stride, slots, n_tokens, a);
  if (st != SEEDQ_OK || n_tokens == 0) return st;
  kGather[cache->kind][dtype](a, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
