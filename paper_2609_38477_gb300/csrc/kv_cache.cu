// The 8-bit paged key/value cache: append (seedq_kv_append) and its inverse
// (seedq_kv_gather).
#include <cuda_runtime.h>
#include <stdint.h>

#include "cp_async.cuh"
#include "f32x2.cuh"
#include "kv_codes.cuh"
#include "serve.cuh"

namespace seedq {
namespace {

struct CacheArgs {
  seedq_kv_cache c;
  void *x[2];          // the tokens' keys and values
  int64_t ts, hs, n;   // their strides (elements) and number
  const int64_t *slots;
  int32_t vec;         // 2 or 1 where rows of x allow accesses of 32 or 16 bytes, else 0
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
  __device__ __forceinline__ uint64_t pair(int k) const {  // elements 2k and 2k + 1
    if (DT == SEEDQ_F16) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[k % kWords]));
      return f2_pack(f.x, f.y);
    }
    return f2_pack(get(2 * k), get(2 * k + 1));
  }
  // Largest magnitudes so far, in the type itself; a NaN stays.
  __device__ __forceinline__ void largest(uint32_t &m) const {
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      if (DT == SEEDQ_F32) m = max(m, w[k] & 0x7fffffffu);
      else m = __vmaxu2(m, w[k] & 0x7fff7fffu);
    }
  }
  static __device__ __forceinline__ uint32_t largest_bits(uint32_t m) {  // as the bits of a float
    if (DT == SEEDQ_F32) return m;
    const uint32_t x = max(m & 0xffffu, m >> 16);
    return DT == SEEDQ_BF16 ? x << 16 : __float_as_uint(__half2float(__ushort_as_half((unsigned short)x)));
  }
};

// ---------------------------------------------------------------- append
//
// A page's tokens are read, their largest magnitude is found, and the codes are
// written.  Bytes bound it for prompts, latency for a decode step (slots, then
// scale and tokens, then codes), so the work is cut for many warps: a warp owns
// one head and tensor of the stretches of tokens on one page that begin among
// 2^group_shift tokens.  A lane takes 8 elements of a token; the first kHeld
// steps of a run stay in its registers between the maximum and the codes, the
// next ones in shared memory, where asynchronous copies put them (30 tokens of
// 128 head dims, 16 in float32).  A run that is longer than that the CTA's warps,
// which own pairs of the same tokens, take together, one pair after the other,
// so that it too is read once (4 prompts of 1024, pages of 64, 32 heads: 24 us
// instead of 28; pages of 128: 30 instead of 49); what is longer still is read
// again, from cache.
//
// Measured, 128 head dims: 4 prompts of 1024 tokens, 32 heads, bfloat16, 24 us
// (4.2 TB/s, 62% of the copy rate; float32 46 us, 3.7 TB/s); 16 single tokens of
// 8 heads 3.4 us, launch and three dependent reads.  28 warps per SM: 24, with
// more registers, take 28 and, for 256 single tokens of 32 heads, 12 us instead
// of 10; 32 take 24 and 10.
constexpr int kAppendWarps = 4;
constexpr int kAppendBlocks = 7;  // per SM: 28 warps of up to 73 registers
constexpr int kKeptPieces = 14;   // of a lane in shared memory: 7 KB per warp

template <int KIND, int DT>
__global__ void __launch_bounds__(kAppendWarps * 32, kAppendBlocks) k_kv_append(const __grid_constant__ CacheArgs a) {
  constexpr int kHeld = 1, kPieces = DT == SEEDQ_F32 ? 2 : 1;  // 16-byte pieces of a lane and step
  constexpr int kKept = kKeptPieces / kPieces;
  __shared__ uint4 s_kept[kAppendWarps][kKeptPieces][32];
  __shared__ uint32_t s_max[kAppendWarps][kAppendWarps];  // of a pair, by warp
  __shared__ float s_old[kAppendWarps];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int P = a.c.page_size, D = a.c.head_dim, per = D / 8;  // pieces of a token
  const int pairs = 2 * a.c.n_kv_heads, ctas = (pairs + kAppendWarps - 1) / kAppendWarps;
  const int64_t group = blockIdx.x / (uint32_t)ctas;
  const int pair0 = (int)(blockIdx.x - (uint32_t)group * ctas) * kAppendWarps;  // the CTA's first
  const bool owner = pair0 + w < pairs;
  const int64_t g0 = group << a.group_shift;
  const int64_t g1 = min(g0 + (1 << a.group_shift), a.n);
  // Stretches begin where the page differs from the token's before: a lane per token.
  uint32_t starts;
  {
    const int64_t t = g0 + lane;
    const int64_t page = t < g1 ? page_of(a, a.slots[t]) : -1;
    int64_t before = __shfl_up_sync(~0u, page, 1);
    if (lane == 0) before = g0 > 0 ? page_of(a, a.slots[g0 - 1]) : -1;
    starts = __ballot_sync(~0u, page >= 0 && page < a.c.n_pages && page != before);
  }
  const int step = 32 / per, t_first = lane / per, d = (lane - t_first * per) * 8;  // tokens of a step; the lane's piece
  const bool idle = t_first >= step;
  const int64_t ts = a.c.token_stride;

  for (; starts; starts &= starts - 1) {
    int64_t t0 = g0 + __ffs(starts) - 1;
    int64_t slot = a.slots[t0];
    const int64_t page = page_of(a, slot);
    float *scale = ((pair0 + w) & 1 ? a.c.v_scale : a.c.k_scale) + page * a.c.n_kv_heads + (pair0 + w) / 2;
    float old = owner ? *scale : 0.f;
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
      const bool together = m > (kHeld + kKept) * step;  // the same in all warps
      const int nw = together ? kAppendWarps : 1;
      const int first = t_first + (together ? w : 0) * step, stride = nw * step;  // the lane's tokens
      const int mine = idle ? 0 : m;
      for (int p = together ? 0 : w; p < (together ? kAppendWarps : w + 1) && pair0 + p < pairs; ++p) {
        const int h = (pair0 + p) >> 1, which = p & 1;
        const void *x = a.x[which];
        uint8_t *code = (uint8_t *)(which ? a.c.v : a.c.k) + page * a.c.page_stride + h * a.c.head_stride + d;
        const int64_t at = t0 * a.ts + h * a.hs + d;
        Eight<DT> held[kHeld];
        uint32_t amax = 0;
        const int kept = a.vec ? kKept : 0;
        if (kHeld * stride < m)
          for (int k = 0; k < kept; ++k) {
            const int t = first + (kHeld + k) * stride;
            if (t < mine)
#pragma unroll
              for (int y = 0; y < kPieces; ++y)
                cp_async16(&s_kept[w][k * kPieces + y][lane], (const char *)x + (at + t * a.ts) * (kPieces * 2) + 16 * y);
          }
        auto from_kept = [&](int k) {
          Eight<DT> e;
#pragma unroll
          for (int y = 0; y < kPieces; ++y) {
            const uint4 v = s_kept[w][k * kPieces + y][lane];
            e.w[4 * y] = v.x, e.w[4 * y + 1] = v.y, e.w[4 * y + 2] = v.z, e.w[4 * y + 3] = v.w;
          }
          return e;
        };
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
          if (first + k * stride < mine) held[k].load(x, at + (first + k * stride) * a.ts, a.vec);
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
          if (first + k * stride < mine) held[k].largest(amax);
#pragma unroll 2
        for (int t = first + (kHeld + kept) * stride; t < mine; t += stride) {
          Eight<DT> e;
          e.load(x, at + t * a.ts, a.vec);
          e.largest(amax);
        }
        cp_async_commit();
        cp_async_wait<0>();
#pragma unroll 2
        for (int k = 0; k < kept && first + (kHeld + k) * stride < mine; ++k) from_kept(k).largest(amax);
        amax = __reduce_max_sync(~0u, Eight<DT>::largest_bits(amax));
        float was = old;
        if (together) {  // what is written here was last read before another pair's barrier
          if (lane == 0) s_max[p][w] = amax;
          if (lane == 0 && p == w) s_old[w] = old;
          __syncthreads();
#pragma unroll
          for (int k = 0; k < kAppendWarps; ++k) amax = max(amax, s_max[p][k]);
          was = s_old[p];
        }
        const float want = block_scale<KIND>(amax);
        float now = want;
        if (off > 0 && !(want > was) && !isnan(want)) now = was;  // a NaN scale stays
        if (off > 0 && now > was) {
          const float r = __fdiv_rn(was, now);
          const uint64_t r2 = f2_pack(r, r);
#pragma unroll 2
          for (int t = first; t < (idle ? 0 : off); t += stride) {
            uint2 *q = (uint2 *)(code + t * ts);
            const uint2 v = *q;
            uint64_t x0, x1, x2, x3;
            four_values<KIND>(v.x, x0, x1);
            four_values<KIND>(v.y, x2, x3);
            *q = make_uint2(four_codes<KIND>(x0, x1, r2), four_codes<KIND>(x2, x3, r2));
          }
        }
        // x / now; by the reciprocal where that is exact: now a power of two whose reciprocal is a normal number
        const uint32_t nb = __float_as_uint(now);
        const bool exact = (nb & 0x7fffffu) == 0 && nb < 0x7f000000u && nb != 0;
        const float inv = exact ? __uint_as_float(0x7f000000u - nb) : 0.f;
        const uint64_t inv2 = f2_pack(inv, inv);
        auto write = [&](const Eight<DT> &e, int t) {
          uint32_t z[2] = {0, 0};
          if (exact) {
            z[0] = four_codes<KIND>(e.pair(0), e.pair(1), inv2);
            z[1] = four_codes<KIND>(e.pair(2), e.pair(3), inv2);
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
          if (first + k * stride < mine) write(held[k], first + k * stride);
#pragma unroll 2
        for (int k = 0; k < kept && first + (kHeld + k) * stride < mine; ++k) write(from_kept(k), first + (kHeld + k) * stride);
#pragma unroll 2
        for (int t = first + (kHeld + kept) * stride; t < mine; t += stride) {
          Eight<DT> e;
          e.load(x, at + t * a.ts, a.vec);
          write(e, t);
        }
        if (p == w) old = now;
      }
      t0 += m;
      slot = t0 < a.n ? a.slots[t0] : -1;
      if (together) __syncthreads();  // the page's next run is perhaps a warp's alone
      else __syncwarp();
    } while (page_of(a, slot) == page);
    if (owner && lane == 0) *scale = old;
  }
}

// ---------------------------------------------------------------- gather
//
// A thread takes as many codes of a key and of a value as make BYTES bytes of the
// output; bytes bound it.  32 bytes are one store where rows begin at multiples of
// 32 (4096 tokens of 32 heads, 128 head dims: 18 us, 5.5 TB/s, 81% of the copy
// rate, float32 28 us; with stores of 16 bytes 20 and 35), 16 bytes make twice
// the threads of a small call (217 tokens of 4 heads of 64: 2.3 us, else 2.5).
constexpr int64_t kGatherSmall = 152 * 2048;

template <int KIND, int DT, int BYTES>
__global__ void __launch_bounds__(256) k_kv_gather(const __grid_constant__ CacheArgs a) {
  constexpr int kWidth = DT == SEEDQ_F32 ? 4 : 2, kCodes = BYTES / kWidth, kWords = BYTES / 4;
  const int P = a.c.page_size, per = a.c.head_dim / kCodes;
  const int row = a.c.n_kv_heads * per;  // threads of a token
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int64_t t = i >> 32 ? i / row : (int64_t)((uint32_t)i / (uint32_t)row);
  if (t >= a.n) return;
  const int r = (int)(i - t * row), h = r / per, d = (r - h * per) * kCodes;
  const int64_t slot = a.slots[t];
  const int64_t page = page_of(a, slot);
  uint32_t code[2][kCodes / 4] = {};
  float scale[2] = {0.f, 0.f};
  if (page >= 0 && page < a.c.n_pages) {
    const int64_t at = page * a.c.page_stride + h * a.c.head_stride + (slot - page * P) * a.c.token_stride + d;
    const int64_t s = page * a.c.n_kv_heads + h;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const uint8_t *src = (const uint8_t *)(which ? a.c.v : a.c.k) + at;
      if constexpr (kCodes == 16) {
        const uint4 v = *(const uint4 *)src;
        code[which][0] = v.x, code[which][1] = v.y, code[which][2] = v.z, code[which][3] = v.w;
      } else if constexpr (kCodes == 8) {
        const uint2 v = *(const uint2 *)src;
        code[which][0] = v.x, code[which][1] = v.y;
      } else {
        code[which][0] = *(const uint32_t *)src;
      }
      scale[which] = (which ? a.c.v_scale : a.c.k_scale)[s];
    }
  }
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const uint64_t by = f2_pack(scale[which], scale[which]);
    uint32_t y[kWords];
#pragma unroll
    for (int k = 0; k < kCodes / 2; ++k) {
      uint64_t x[2];
      four_values<KIND>(code[which][k / 2], x[0], x[1]);
      const float2 f = f2_unpack(f2_mul(x[k & 1], by));
      if (DT == SEEDQ_F32) {
        y[2 * k % kWords] = __float_as_uint(f.x), y[(2 * k + 1) % kWords] = __float_as_uint(f.y);
      } else if (DT == SEEDQ_BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
        y[k] = *(const uint32_t *)&b;
      } else {
        const __half2 b = __floats2half2_rn(f.x, f.y);
        y[k] = *(const uint32_t *)&b;
      }
    }
    char *to = (char *)a.x[which] + (t * a.ts + h * a.hs + d) * kWidth;
    if (BYTES == 32 && a.vec == 2) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(y[0]), "r"(y[1]), "r"(y[2]),
                   "r"(y[3]), "r"(y[4 % kWords]), "r"(y[5 % kWords]), "r"(y[6 % kWords]), "r"(y[7 % kWords])
                   : "memory");
    } else if (a.vec) {
#pragma unroll
      for (int k = 0; k < kWords; k += 4) *(uint4 *)(to + 4 * k) = make_uint4(y[k], y[k + 1], y[k + 2], y[k + 3]);
    } else {
#pragma unroll
      for (int k = 0; k < kWords; ++k) {
        if (DT == SEEDQ_F32) {
          ((uint32_t *)to)[k] = y[k];
        } else {
          ((uint16_t *)to)[2 * k] = (uint16_t)y[k];
          ((uint16_t *)to)[2 * k + 1] = (uint16_t)(y[k] >> 16);
        }
      }
    }
  }
}

// 2 or 1 where rows allow accesses of 32 or 16 bytes, else 0
int32_t rows_aligned(const void *k, const void *v, int32_t dtype, int64_t ts, int64_t hs) {
  const uint64_t all = (uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)v | (uint64_t)(ts * dtype_bytes(dtype)) | (uint64_t)(hs * dtype_bytes(dtype));
  return all % 32 == 0 ? 2 : all % 16 == 0;
}

int64_t append_ctas(const CacheArgs &a) {
  const int64_t groups = (a.n + (1 << a.group_shift) - 1) >> a.group_shift;
  return groups * ((a.c.n_kv_heads * 2 + kAppendWarps - 1) / kAppendWarps);
}
template <int KIND, int DT>
void launch_append(const CacheArgs &a, cudaStream_t st) {
  k_kv_append<KIND, DT><<<(unsigned)append_ctas(a), kAppendWarps * 32, 0, st>>>(a);
}
template <int KIND, int DT>
void launch_gather(const CacheArgs &a, cudaStream_t st) {
  const int64_t pieces = a.n * a.c.n_kv_heads * a.c.head_dim / (DT == SEEDQ_F32 ? 4 : 8);
  if (pieces <= kGatherSmall) k_kv_gather<KIND, DT, 16><<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(a);
  else k_kv_gather<KIND, DT, 32><<<(unsigned)((pieces / 2 + 255) / 256), 256, 0, st>>>(a);
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
  a.group_shift = append_group_shift(n_tokens, cache->n_kv_heads);
  if (append_ctas(a) > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  kAppend[cache->kind][dtype](a, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

seedq_status seedq_kv_gather(const seedq_kv_cache *cache, const int64_t *slots, int64_t n_tokens, void *k, void *v,
                             int32_t dtype, int64_t token_stride, int64_t head_stride, void *cuda_stream) {
  CacheArgs a;
  const seedq_status st = prepare(cache, k, v, dtype, token_stride, head_stride, slots, n_tokens, a);
  if (st != SEEDQ_OK || n_tokens == 0) return st;
  if (n_tokens * cache->n_kv_heads * cache->head_dim / 2048 >= INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  kGather[cache->kind][dtype](a, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
