// Log probability, rank, entropy and top alternatives of a token under a row of
// logits (seedq_token_logprobs).
//
// Mathematics, one pass over the logits x with c = scale * log2(e):
//   m = max x,  d = c (x - m),  s1 = sum 2^d,  s2 = sum d 2^d,
//   logprob = scale (x_t - m) - ln s1,  entropy = ln2 (log2 s1 - s2 / s1);
// when the running maximum rises by e / c, s1 and s2 become s1 2^-e and
// (s2 - e s1) 2^-e.  Differences come first: nothing overflows, and a large
// common part of the logits does not cost precision.  The rank counts logits
// above the target's; equal ones count where their index is lower.
//
// The first top_k tokens are kept as a sorted list, one 64-bit key per lane of a
// warp (the logit as an ordered integer, then the inverted index: equal logits
// go by the lower index).  A tile of logits is looked at only if its maximum
// reaches the list's last entry, which happens about top_k * ln(vocab) times
// per list; a list starts from the top_k-th largest of the lanes' own maxima of
// its first tile instead of from nothing.  Where few lanes hold logits that
// reach it, the whole warp looks at one lane's logits at a time and inserts what
// passes (about 75 cycles a key); else they are packed in shared memory, sorted
// 32 at a time and merged (about 600 cycles).
//
// What bounds it: many rows, the bytes of the logits (about 9 instructions and
// one 2^x per logit leave the SMs at half their rate for float32); few rows, the
// latency of the joins.  Measured, 128256 logits: 2048 rows of float32 153 us
// without targets and alternatives (6.9 TB/s, 101% of the copy rate), 171 with
// targets and 5 alternatives (90%), 213 with 20; of bfloat16 86 us (90%), 117 with
// targets, 191 with 20 alternatives as well, where instructions bound it; 16 rows
// of float32 with 20 alternatives 12 us.
//
// Split.  All rows' tiles form one sequence, cut into equal ranges, one per warp
// (at least one tile each).  A warp that holds a whole row writes its results;
// parts of rows cut between warps are joined by the CTA, those cut between CTAs
// by the last CTA to arrive (a counter per CTA, reset by that CTA), in the order
// of the tokens.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "cp_async.cuh"
#include "device_once.h"
#include "f32x2.cuh"
#include "serve.cuh"

namespace seedq {
namespace {

// 16 warps per SM: 24 take 124 us instead of 117 for 2048 rows of bfloat16 with
// targets (fewer registers), 12 as much and 194 instead of 171 in float32 with 5
// alternatives (too few copies under way); one CTA of 16, 17 us instead of 11 for
// 2000 rows of 600.
constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kCtasPerSm = 2;
constexpr int kMaxCtas = 152 * kCtasPerSm;
constexpr int kMaxTop = 32;
// k_score_few: threads, the most CTAs of a call, candidates that a CTA sorts
constexpr int kFewThreads = 256;
constexpr int kFewWarps = kFewThreads / 32, kFewEach = 32 / kFewWarps;
constexpr int kFewMax = 16 * 152;
constexpr int kFewKeys = 512;
constexpr int kStages = 3;       // tiles in a warp's ring (5: 160 us instead of 153 without targets and alternatives)
constexpr int kTileBytes = 2048; // 64 bytes per lane
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct ScoreArgs {
  const void *x;
  int64_t stride, rows;
  int32_t vocab, tiles;  // tiles of a row
  float scale, c;        // c = scale * log2(e)
  const int64_t *targets;
  float *logprob, *entropy;
  int32_t *rank;
  int32_t top_k;
  float *top_logprob;
  int32_t *top_index;
  void *workspace;
  int32_t ctas;
  int64_t share;  // tiles per CTA
};

// What a range of a row's logits comes to.
struct Part {
  float m, s1, s2;  // as above
  int32_t count;    // logits before the target
  uint64_t key[kMaxTop];
};

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
// x >= xt as x > the number before xt; for -inf every x: no x is <= NaN.
__device__ __forceinline__ float number_before(float xt) {
  if (xt == -CUDART_INF_F) return CUDART_NAN_F;
  return xt == 0.f ? __uint_as_float(0x80000001u) : __uint_as_float(__float_as_uint(xt) + (xt > 0.f ? -1 : 1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A load past the L1 cache: sees what other SMs wrote.
template <typename T>
__device__ __forceinline__ T fresh_load(const T *x) { return *(const volatile T *)x; }

// A target's logit, -0 as +0: count_above would take every +0 for larger than -0.
__device__ __forceinline__ float target_logit(const void *p, int dt, int64_t i) { return load_elem(p, dt, i) + 0.f; }

// How many of x are above thr, all of them if thr is NaN: the signs of thr - x,
// shifted into a word (a compare and an add per number cost twice as much).  thr
// is not -0.
template <int N>
__device__ __forceinline__ int count_above(const float (&x)[N], float thr) {
  static_assert(N <= 32, "");
  if (isnan(thr)) return N;
  const uint64_t thr2 = f2_pack(thr, thr), minus = f2_pack(-1.f, -1.f);
  uint32_t signs = 0;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    const float2 d = f2_unpack(f2_fma(f2_pack(x[e], x[e + 1]), minus, thr2));
    signs = __funnelshift_l(__float_as_uint(d.x), signs, 1);
    signs = __funnelshift_l(__float_as_uint(d.y), signs, 1);
  }
  return __popc(signs);
}

// The sums relative to a maximum `to` that is no smaller.
__device__ __forceinline__ void rebase(float &m, float &s1, float &s2, float to, float c) {
  const float d = m == -CUDART_INF_F ? 0.f : max_nan((m - to) * c, -1e4f), e = exp2_fast(d);
  s2 = (s2 + d * s1) * e;
  s1 *= e;
  m = to;
}

// Both lists' first 32 keys in order: of two descending lists, the larger of a's
// i-th and b's (31 - i)-th are the 32 largest, a bitonic sequence.
__device__ __noinline__ uint64_t merge_lists(uint64_t a, uint64_t b, int lane) {
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
__device__ __noinline__ uint64_t sort_keys(uint64_t x, int lane) {
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

// scale (x - m); by halves where the difference alone passes float32's largest.
__device__ __forceinline__ float scaled_difference(float scale, float x, float m) {
  const float d = x - m;
  return d == -CUDART_INF_F && x > -CUDART_INF_F ? 2.f * (scale * (0.5f * x - 0.5f * m)) : scale * d;
}

// Writes a row's results: key is the lane's entry of the list, the rest is the
// same in all lanes.
__device__ __noinline__ void write_row(const ScoreArgs &a, int64_t row, float m, float s1, float s2, int count, uint64_t key,
                                          int64_t t, float xt) {
  const int lane = threadIdx.x & 31;
  const bool bad = isnan(m) || m == CUDART_INF_F, empty = m == -CUDART_INF_F;
  const float lg = log2f(s1), ln_s1 = kLn2 * lg;  // differences by scale itself: c would carry a mask's value past the type
  if (lane == 0) {
    if (a.entropy) a.entropy[row] = bad ? CUDART_NAN_F : empty ? 0.f : kLn2 * (lg - s2 / s1);
    if (a.targets) {
      const bool has = t >= 0 && t < a.vocab;
      a.logprob[row] = t == -1          ? 0.f
                       : !has || bad    ? CUDART_NAN_F
                       : empty          ? -CUDART_INF_F
                                        : scaled_difference(a.scale, xt, m) - ln_s1;
      a.rank[row] = has && !isnan(m) ? count : -1;
    }
  }
  if (lane < a.top_k) {
    const float x = key_value(key);
    a.top_index[row * a.top_k + lane] = key ? key_index(key) : -1;
    a.top_logprob[row * a.top_k + lane] = !key || empty ? -CUDART_INF_F : bad ? CUDART_NAN_F : scaled_difference(a.scale, x, m) - ln_s1;
  }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_score(const __grid_constant__ ScoreArgs a) {
  constexpr int kPer = DT == SEEDQ_F32 ? 16 : 32;  // logits of a lane and tile
  constexpr int kVec = DT == SEEDQ_F32 ? 4 : 8;    // in one 16-byte load
  constexpr int kTile = 32 * kPer;
  constexpr int kSize = DT == SEEDQ_F32 ? 4 : 2;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  // at a multiple of 128 bytes: a copy whose 32-byte sectors straddle those of
  // shared memory is fetched twice from L2
  uint8_t *smem = smem_raw + (128 - ((uint32_t)__cvta_generic_to_shared(smem_raw) & 127)) % 128;
  __shared__ Part s_part[2 * kWarps];
  __shared__ int64_t s_row[2 * kWarps];  // its row, or -1
  __shared__ uint64_t s_buffer[kWarps][64];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  if (lane < 2) s_row[2 * w + lane] = -1;

  const int64_t total = a.rows * a.tiles;
  const int64_t c0 = a.share * blockIdx.x, c1 = min(c0 + a.share, total);
  const uint32_t mine = (uint32_t)(c1 - c0), each = mine / kWarps, rest = mine - each * kWarps;
  const int64_t w0 = c0 + each * (uint32_t)w + min((uint32_t)w, rest);
  const int64_t w1 = w0 + each + (w < (int)rest);

  uint64_t *buffer = s_buffer[w];
  uint8_t *ring = smem + w * (kStages * kTileBytes) + lane * 16;
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  int64_t row = w0 / a.tiles, prow = row;
  int tile = (int)(w0 - row * a.tiles), ptile = tile;
  int64_t left = w1 - w0;
  int pstage = 0, stage = 0;
  int64_t pleft = left;
  const char *psrc = (const char *)a.x + (prow * a.stride + (int64_t)ptile * kTile + lane * kVec) * kSize;
  auto issue = [&]() {
    if (VEC && pleft > 0) {
      const uint32_t dst = ring_s + pstage * kTileBytes;
      if ((ptile + 1) * kTile <= a.vocab) {
#pragma unroll
        for (int v = 0; v < 4; ++v)
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + v * 512), "l"(psrc + v * 512) : "memory");
      } else {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          // what lies past the row's end is not read
          const int i = ptile * kTile + v * (32 * kVec) + lane * kVec;
          const int bytes = min(max(a.vocab - i, 0) * kSize, 16);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + v * 512),
                       "l"(bytes ? psrc + v * 512 : (const char *)a.x), "r"(bytes)
                       : "memory");
        }
      }
      --pleft;
      pstage = pstage + 1 == kStages ? 0 : pstage + 1;
      psrc += kTile * kSize;
      if (++ptile == a.tiles) {
        ptile = 0;
        ++prow;
        psrc = (const char *)a.x + (prow * a.stride + lane * kVec) * kSize;
      }
    }
    cp_async_commit();
  };
  if (left > 0)
    for (int i = 0; i < kStages - 1; ++i) issue();

  // The targets of this row and the next two, and the logits of the first two,
  // are on their way before they are needed.
  auto target = [&](int64_t r) -> int64_t { return a.targets && r < a.rows ? a.targets[r] : -1; };
  auto logit = [&](int64_t r, int64_t t) -> float {
    return t >= 0 && t < a.vocab ? target_logit(a.x, DT, r * a.stride + t) : 0.f;
  };
  int64_t t = target(row), t1 = target(row + 1);
  float xt = logit(row, t), xt1 = logit(row + 1, t1);

  float m = 0.f, s1 = 0.f, s2 = 0.f, tau = 0.f;
  float above = 0.f, from = 0.f;  // logits greater than these come before the target: past it and ahead of it
  int count = 0;
  uint64_t key = 0, last = 0;  // the lane's entry of the list; the list's last
  bool fresh = true;           // the row begins for this warp
  const int64_t row0 = row;

  for (; left > 0; --left) {
    if (fresh) {
      if (row != row0) {
        t = t1, xt = xt1;
        t1 = target(row + 1);
        xt1 = logit(row + 1, t1);
      }
      m = -CUDART_INF_F;
      s1 = s2 = 0.f;
      count = 0;
      key = last = 0;
    }
    issue();
    float x[kPer];
    const int base = tile * kTile;
    if (VEC) {
      cp_async_wait<kStages - 1>();
      const uint8_t *src = ring + stage * kTileBytes;
      stage = stage + 1 == kStages ? 0 : stage + 1;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const uint4 y = *(const uint4 *)(src + v * 512);
        const uint32_t z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (DT == SEEDQ_F32) {
            x[v * 4 + k] = __uint_as_float(z[k]);
          } else if (DT == SEEDQ_BF16) {
            x[v * 8 + 2 * k] = __uint_as_float(z[k] << 16);
            x[v * 8 + 2 * k + 1] = __uint_as_float(z[k] & 0xffff0000u);
          } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&z[k]));
            x[v * 8 + 2 * k] = f.x, x[v * 8 + 2 * k + 1] = f.y;
          }
        }
      }
    }
    const uint8_t *held = ring + (stage == 0 ? kStages - 1 : stage - 1) * kTileBytes;
    // index of element e: rows that allow wide loads give a lane 16 bytes in a row, others single logits
    auto index = [&](int e) -> int {
      return base + (VEC ? (e / kVec) * (32 * kVec) + lane * kVec + e % kVec : e * 32 + lane);
    };
    // element e again, for the rare loops that are not unrolled
    auto fetch = [&](int e) -> float {
      if (index(e) >= a.vocab) return -CUDART_INF_F;
      return VEC ? load_elem(held + (e / kVec) * 512, DT, e % kVec) : load_elem(a.x, DT, row * a.stride + index(e));
    };
    const bool partial = base + kTile > a.vocab;
    if (!VEC) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) x[e] = index(e) < a.vocab ? load_elem(a.x, DT, row * a.stride + index(e)) : -CUDART_INF_F;
    } else if (partial) {
#pragma unroll
      for (int e = 0; e < kPer; ++e)
        if (index(e) >= a.vocab) x[e] = -CUDART_INF_F;
    }

    // the sums
    float mx = max_nan(x[0], x[1]), mo = max_nan(x[2], x[3]);
#pragma unroll
    for (int e = 4; e < kPer; e += 4) {
      mx = max_nan(mx, x[e], x[e + 1]);
      mo = max_nan(mo, x[e + 2], x[e + 3]);
    }
    mx = max_nan(mx, mo);
    const float to = max_nan(m, mx);
    rebase(m, s1, s2, to, a.c);
    const float off = to == -CUDART_INF_F ? 0.f : -to;
    const uint64_t off2 = f2_pack(off, off), c2 = f2_pack(a.c, a.c);
    uint64_t p1 = 0, p2 = 0;
#pragma unroll
    for (int e = 0; e < kPer; e += 2) {
      const float2 d = f2_unpack(f2_mul(f2_add(f2_pack(x[e], x[e + 1]), off2), c2));
      const float d0 = max_nan(d.x, -1e4f), d1 = max_nan(d.y, -1e4f);  // 2^-10000 is 0, and so is its product with d
      const uint64_t y = f2_pack(exp2_fast(d0), exp2_fast(d1));
      p1 = f2_add(p1, y);
      p2 = f2_fma(y, f2_pack(d0, d1), p2);
    }
    const float2 q1 = f2_unpack(p1), q2 = f2_unpack(p2);
    s1 += q1.x + q1.y;
    s2 += q2.x + q2.y;

    // the list
    if (a.top_k) {
      if (fresh) {  // the top_k-th largest of the lanes' maxima: at least top_k logits reach it
        int before = 0;
#pragma unroll 4
        for (int o = 0; o < 32; ++o) {
          const float y = __shfl_sync(~0u, mx, o);
          before += !(y <= mx) || (y == mx && o < lane);
        }
        tau = __shfl_sync(~0u, mx, __ffs(__ballot_sync(~0u, before == a.top_k - 1) | 0x80000000u) - 1);
        if (!__any_sync(~0u, before == a.top_k - 1)) tau = -CUDART_INF_F;  // NaN among them
      }
      uint32_t lanes = __ballot_sync(~0u, !(mx < tau));  // whose logits reach the list
      if (lanes) {
        __syncwarp();
        if (__popc(lanes) <= 8) {
          // a lane's logits are looked at by the whole warp
          do {
            const int from_lane = __ffs(lanes) - 1;
            const int i = base + (VEC ? (lane / kVec) * (32 * kVec) + from_lane * kVec + lane % kVec : lane * 32 + from_lane);
            const bool there = lane < kPer && i < a.vocab;
            float y = -CUDART_INF_F;
            if (there)
              y = VEC ? load_elem(held + (from_lane - lane) * 16 + (lane / kVec) * 512, DT, lane % kVec)
                      : load_elem(a.x, DT, row * a.stride + i);
            const uint64_t own = order_key(y, i);
            uint32_t todo = __ballot_sync(~0u, there && !(y < tau) && own > last);
            lanes &= lanes - 1;
            if (todo == 0) continue;
            do {
              const uint64_t cand = __shfl_sync(~0u, own, __ffs(todo) - 1), up = __shfl_up_sync(~0u, key, 1);
              if (key < cand) key = lane > 0 && up < cand ? up : cand;
              todo &= todo - 1;
            } while (todo);
            last = __shfl_sync(~0u, key, a.top_k - 1);
            if (last) tau = key_value(last);
            lanes &= __ballot_sync(~0u, !(mx < tau));
          } while (lanes);
        } else {
          int packed = 0;
          auto flush = [&]() {
            __syncwarp();
            for (int at = 0; at < packed; at += 32)
              key = merge_lists(key, sort_keys(at + lane < packed ? buffer[at + lane] : 0, lane), lane);
            packed = 0;
            last = __shfl_sync(~0u, key, a.top_k - 1);
            if (last) tau = key_value(last);
            __syncwarp();
          };
#pragma unroll 1
          for (int e = 0; e < kPer; ++e) {
            const float y = fetch(e);
            const uint64_t own = order_key(y, index(e));
            const bool in = !(y < tau) && own > last && index(e) < a.vocab;
            const uint32_t todo = __ballot_sync(~0u, in);
            if (todo == 0) continue;
            if (in) buffer[packed + __popc(todo & ((1u << lane) - 1))] = own;
            packed += __popc(todo);
            if (packed > 32) flush();
          }
          if (packed) flush();
        }
        __syncwarp();
      }
    }

    // the rank
    if (a.targets) {
      if (fresh) {
        above = xt;
        from = number_before(xt);
      }
      const float thr = base < t ? from : above;
      if ((partial && isnan(thr)) || (t >= base && t < base + kTile)) {  // what is past the row's end is -inf
#pragma unroll 1
        for (int e = 0; e < kPer; ++e) count += index(e) < a.vocab && !(fetch(e) <= (index(e) < t ? from : above));
      } else if (__any_sync(~0u, !(mx <= thr))) {  // else no logit of the tile comes before the target
        count += count_above<kPer>(x, thr);
      }
    }
    fresh = false;

    if (++tile < a.tiles && left > 1) continue;

    // ---- the end of this warp's part of a row
    const int64_t begin = row * a.tiles;
    const bool whole = begin >= w0 && begin + a.tiles <= w1;
    float M = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) M = max_nan(M, __shfl_xor_sync(~0u, M, o));
    rebase(m, s1, s2, M, a.c);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      s1 += __shfl_xor_sync(~0u, s1, o);
      s2 += __shfl_xor_sync(~0u, s2, o);
    }
    count = __reduce_add_sync(~0u, count);
    if (whole) {
      write_row(a, row, m, s1, s2, count, key, t, xt);
    } else {
      const int at = 2 * w + (left == 1);
      s_part[at].key[lane] = key;
      if (lane == 0) {
        s_part[at].m = m, s_part[at].s1 = s1, s_part[at].s2 = s2, s_part[at].count = count;
        s_row[at] = row;
      }
    }
    tile = 0;
    ++row;
    fresh = true;
  }
  cp_async_wait<0>();
  __syncthreads();

  // ---- joins.  Parts are taken in order; a join of few is one warp's work, so
  // that many rows are joined at a time, one of many the whole CTA's.
  Part *slots = (Part *)((uint8_t *)a.workspace + kFewMax * 4);  // two per CTA
  int *counters = (int *)a.workspace;
  __shared__ Part s_sum[kWarps];
  __shared__ int s_last[2];
  float fm, f1, f2;
  int fc;
  uint64_t fk;
  auto clear = [&]() { fm = -CUDART_INF_F, f1 = f2 = 0.f, fc = 0, fk = 0; };
  auto add = [&](const Part *q) {
    float qm = fresh_load(&q->m), q1 = fresh_load(&q->s1), q2 = fresh_load(&q->s2);
    const uint64_t qk = a.top_k ? fresh_load(&q->key[lane]) : 0;
    fc += fresh_load(&q->count);
    const float to = max_nan(fm, qm);
    rebase(fm, f1, f2, to, a.c);
    rebase(qm, q1, q2, to, a.c);
    f1 += q1, f2 += q2;
    if (a.top_k) fk = merge_lists(fk, qk, lane);
  };
  auto put = [&](Part *q) {
    q->key[lane] = fk;
    if (lane == 0) q->m = fm, q->s1 = f1, q->s2 = f2, q->count = fc;
  };
  auto finish = [&](int64_t r, Part *to) {
    if (to) return put(to);
    const int64_t tr = target(r);
    write_row(a, r, fm, f1, f2, fc, fk, tr, logit(r, tr));
  };
  auto tree = [&]() {  // the warps' sums into warp 0's
    for (int o = 1; o < kWarps; o <<= 1) {
      __syncthreads();
      if (w & o) put(&s_sum[w]);
      __syncthreads();
      if ((w & (2 * o - 1)) == 0 && w + o < kWarps) add(&s_sum[w + o]);
    }
  };

  // rows cut between the warps of this CTA
  const int64_t part_row = lane < 2 * kWarps ? s_row[lane] : -1;
  const uint32_t valid = __ballot_sync(~0u, part_row >= 0);
  if (valid == 0) return;
  const uint32_t below = valid & ((1u << lane) - 1);
  const int64_t row_before = __shfl_sync(~0u, part_row, below ? 31 - __clz(below) : 0);
  const uint32_t heads = __ballot_sync(~0u, part_row >= 0 && (below == 0 || row_before != part_row));
  int64_t cross[2];  // rows cut between CTAs: the one that came from before, the one that goes on
  cross[0] = __shfl_sync(~0u, part_row, __ffs(valid) - 1);
  cross[1] = __shfl_sync(~0u, part_row, 31 - __clz(valid));
  if (cross[1] * a.tiles < c0 || (cross[1] + 1) * a.tiles <= c1) cross[1] = -1;
  if (cross[0] * a.tiles >= c0) cross[0] = -1;
  auto slot_of = [&](int64_t r) -> Part * {
    return r == cross[0] ? slots + 2 * blockIdx.x : r == cross[1] ? slots + 2 * blockIdx.x + 1 : nullptr;
  };
  const bool alone = __popc(heads) > 2;  // joins by single warps
  uint32_t todo = heads;
  for (int g = 0; todo; ++g, todo &= todo - 1) {
    if (alone && g % kWarps != w) continue;
    const int64_t r = __shfl_sync(~0u, part_row, __ffs(todo) - 1);
    uint32_t same = __ballot_sync(~0u, part_row == r);
    clear();
    const int n = __popc(same);
    const int lo = alone ? 0 : n * w / kWarps, hi = alone ? n : n * (w + 1) / kWarps;
    for (int j = 0; same; ++j, same &= same - 1)
      if (j >= lo && j < hi) add(&s_part[__ffs(same) - 1]);
    if (!alone) tree();
    if (alone || w == 0) finish(r, slot_of(r));
  }
  if (cross[0] < 0 && cross[1] < 0) return;

  // rows cut between CTAs: the last to arrive joins
  __threadfence();
  __syncthreads();
  if (lane == 0 && w < 2) {
    const int64_t r = w ? cross[1] : cross[0];
    int last_one = 0;
    if (r >= 0) {
      const int first = (int)(r * a.tiles / a.share), n = (int)(((r + 1) * a.tiles - 1) / a.share) - first + 1;
      last_one = atomicAdd(counters + first, 1) == n - 1 ? n : 0;
      if (last_one) counters[first] = 0;
    }
    s_last[w] = last_one;
  }
  __syncthreads();
  __threadfence();
  for (int side = 0; side < 2; ++side) {
    const int n = s_last[side];
    const bool single = n <= 8;
    if (n == 0 || (single && w != side)) continue;
    const int64_t r = cross[side];
    // the first CTA's part is its second slot, the others' their first
    const Part *from_slot = slots + 2 * (int)(r * a.tiles / a.share);
    const int lo = single ? 0 : n * w / kWarps, hi = single ? n : n * (w + 1) / kWarps;
    clear();
    for (int j = lo; j < hi; ++j) add(from_slot + (j ? 2 * j : 1));
    if (!single) tree();
    if (single || w == 0) finish(r, nullptr);
  }
}

// ---------------------------------------------------------------- few rows
//
// A row's chunk per CTA, held in registers.  With few rows latency is all: the
// lists of k_score would each be built from one or two tiles.  Here every warp
// finds the four largest of its lanes' maxima; at least top_k logits of the CTA
// reach the top_k-th of these 32, and few more do, so these few are packed and put
// in order by counting, for each, how many come before it.  The last CTA of a row
// to arrive does the same with the chunks' lists.

// The n-th largest of the lanes' words (1 <= n <= 32), in all lanes.
template <typename T>
__device__ __forceinline__ T nth_of_warp(T x, int n) {
  const int lane = threadIdx.x & 31;
  int before = 0;
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const T y = __shfl_sync(~0u, x, j);
    before += y > x || (y == x && j < lane);
  }
  return __shfl_sync(~0u, x, __ffs(__ballot_sync(~0u, before == n - 1)) - 1);
}

// Puts the first 32 of n <= kFewKeys distinct keys in order into list (zeroed).
__device__ __forceinline__ void order_keys(const uint64_t *keys, int n, uint64_t *list) {
  for (int i = threadIdx.x; i < n; i += kFewThreads) {
    const uint64_t own = keys[i];
    int before = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) before += keys[j] > own;
    if (before < kMaxTop) list[before] = own;
  }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(kFewThreads, 4) k_score_few(const __grid_constant__ ScoreArgs a) {
  constexpr int kPer = DT == SEEDQ_F32 ? 16 : 32, kVec = DT == SEEDQ_F32 ? 4 : 8;
  __shared__ uint64_t s_keys[kFewKeys], s_list[kMaxTop], s_best[kFewWarps];
  __shared__ float s_1[kFewWarps], s_2[kFewWarps];
  __shared__ uint32_t s_reach[32];
  __shared__ int s_count[kFewWarps], s_n, s_last;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int64_t row = blockIdx.x / a.tiles;
  const int chunk = blockIdx.x - (int)row * a.tiles;
  const int base = chunk * (kFewThreads * kPer);

  auto index = [&](int e) -> int {
    return base + (VEC ? (e / kVec) * (kFewThreads * kVec) + tid * kVec + e % kVec : e * kFewThreads + tid);
  };
  float x[kPer];
  if (VEC) {
    const char *src = (const char *)a.x + (row * a.stride + base + tid * kVec) * (16 / kVec);
    uint4 y[4];
#pragma unroll
    for (int v = 0; v < 4; ++v)
      y[v] = index(v * kVec) + kVec <= a.vocab ? __ldg((const uint4 *)(src + v * (kFewThreads * 16))) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const uint32_t z[4] = {y[v].x, y[v].y, y[v].z, y[v].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (DT == SEEDQ_F32) {
          x[v * 4 + k] = __uint_as_float(z[k]);
        } else if (DT == SEEDQ_BF16) {
          x[(v * 8 + 2 * k) % kPer] = __uint_as_float(z[k] << 16);
          x[(v * 8 + 2 * k + 1) % kPer] = __uint_as_float(z[k] & 0xffff0000u);
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&z[k]));
          x[(v * 8 + 2 * k) % kPer] = f.x, x[(v * 8 + 2 * k + 1) % kPer] = f.y;
        }
      }
    }
  }
  if (!VEC || base + kFewThreads * kPer > a.vocab) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = index(e);
      // of a piece that the row's end cuts, what is there is read alone
      if (i >= a.vocab) x[e] = -CUDART_INF_F;
      else if (!VEC || i - e % kVec + kVec > a.vocab) x[e] = load_elem(a.x, DT, row * a.stride + i);
    }
  }
  const int64_t t = a.targets ? a.targets[row] : -1;
  const float xt = t >= 0 && t < a.vocab ? target_logit(a.x, DT, row * a.stride + t) : 0.f;

  if (tid < kMaxTop) s_list[tid] = 0;
  if (tid == 0) s_n = 0;
  float mx = max_nan(x[0], x[1]);
#pragma unroll
  for (int e = 2; e < kPer; e += 2) mx = max_nan(mx, x[e], x[e + 1]);
  const uint32_t um = index(0) < a.vocab ? order_word(mx) : 0;
  uint32_t rest = um;
  const int each = a.top_k ? kFewEach : 1;
#pragma unroll 1
  for (int j = 0; j < each; ++j) {
    const uint32_t word = __reduce_max_sync(~0u, rest);
    if (lane == __ffs(__ballot_sync(~0u, rest == word)) - 1) rest = 0;
    if (lane == 0) s_reach[w * kFewEach + j] = word;
  }
  __syncthreads();
  const uint32_t word = lane % kFewEach < each ? s_reach[lane] : 0;
  const float m = key_value((uint64_t)__reduce_max_sync(~0u, word) << 32);
  const uint32_t reach = a.top_k ? nth_of_warp(word, a.top_k) : 0;

  if (a.top_k && um && um >= reach) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const uint64_t key = order_key(x[e], index(e));
      if ((uint32_t)(key >> 32) >= reach && index(e) < a.vocab) {
        const int at = atomicAdd(&s_n, 1);
        if (at < kFewKeys) s_keys[at] = key;
      }
    }
  }
  const float off = m == -CUDART_INF_F ? 0.f : -m;
  const uint64_t off2 = f2_pack(off, off), c2 = f2_pack(a.c, a.c);
  uint64_t p1 = 0, p2 = 0;
#pragma unroll
  for (int e = 0; e < kPer; e += 2) {
    const float2 d = f2_unpack(f2_mul(f2_add(f2_pack(x[e], x[e + 1]), off2), c2));
    const float d0 = max_nan(d.x, -1e4f), d1 = max_nan(d.y, -1e4f);
    const uint64_t y = f2_pack(exp2_fast(d0), exp2_fast(d1));
    p1 = f2_add(p1, y);
    p2 = f2_fma(y, f2_pack(d0, d1), p2);
  }
  float s1 = f2_unpack(p1).x + f2_unpack(p1).y, s2 = f2_unpack(p2).x + f2_unpack(p2).y;
  int count = 0;
  if (a.targets) {
    const float from = number_before(xt);
    if (base + kFewThreads * kPer > a.vocab || (t >= base && t < base + kFewThreads * kPer)) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) count += index(e) < a.vocab && !(x[e] <= (index(e) < t ? from : xt));
    } else {
      count += count_above<kPer>(x, base < t ? from : xt);
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    s1 += __shfl_xor_sync(~0u, s1, o);
    s2 += __shfl_xor_sync(~0u, s2, o);
  }
  count = __reduce_add_sync(~0u, count);
  if (lane == 0) s_1[w] = s1, s_2[w] = s2, s_count[w] = count;
  __syncthreads();
  if (s_n <= kFewKeys) {
    order_keys(s_keys, s_n, s_list);
  } else {
    // more than fit reach it (equal logits): one key after another
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top_k; ++k) {
      uint64_t best = 0;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const uint64_t key = order_key(x[e], index(e));
        if (key < last && key > best && index(e) < a.vocab) best = key;
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) best = max(best, __shfl_xor_sync(~0u, best, o));
      if (lane == 0) s_best[w] = best;
      __syncthreads();
      last = 0;
      for (int j = 0; j < kFewWarps; ++j) last = max(last, s_best[j]);
      if (tid == 0) s_list[k] = last;
      __syncthreads();
    }
  }
  __syncthreads();

  Part *parts = (Part *)((uint8_t *)a.workspace + kFewMax * 4) + row * a.tiles;
  int *counter = (int *)a.workspace + row;
  if (w == 0) {
    s1 = s2 = 0.f;
    count = 0;
    for (int k = 0; k < kFewWarps; ++k) s1 += s_1[k], s2 += s_2[k], count += s_count[k];
    if (a.tiles == 1) {
      write_row(a, row, m, s1, s2, count, s_list[lane], t, xt);
    } else {
      Part &q = parts[chunk];
      q.key[lane] = s_list[lane];
      if (lane == 0) q.m = m, q.s1 = s1, q.s2 = s2, q.count = count;
      __syncwarp();
      if (lane == 0) {
        __threadfence();
        s_last = atomicAdd(counter, 1) == a.tiles - 1;
        if (s_last) *counter = 0;
        __threadfence();
        s_n = 0;
      }
    }
  }
  if (a.tiles == 1) return;
  __syncthreads();
  if (!s_last) return;

  // the row's chunks
  const int n = a.tiles;
  if (tid < kMaxTop) s_list[tid] = 0;
  if (a.top_k) {
    // the first keys are on their way meanwhile
    constexpr int kAhead = 4;
    uint64_t ahead[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const int i = tid + r * kFewThreads, q = i / a.top_k;
      ahead[r] = i < n * a.top_k ? fresh_load(&parts[q].key[i - q * a.top_k]) : 0;
    }
    // 32 keys of the row: the chunks' first, second, ..., or the largest of every 32nd chunk's first
    uint64_t some = n < 32 ? fresh_load(&parts[lane % n].key[lane / n]) : 0;
    if (n >= 32)
      for (int i = lane; i < n; i += 32) some = max(some, fresh_load(&parts[i].key[0]));
    const uint64_t low = max(nth_of_warp(some, a.top_k), (uint64_t)1);
    auto push = [&](uint64_t key) {
      if (key < low) return;
      const int at = atomicAdd(&s_n, 1);
      if (at < kFewKeys) s_keys[at] = key;
    };
#pragma unroll
    for (int r = 0; r < kAhead; ++r) push(ahead[r]);
    for (int i = tid + kAhead * kFewThreads; i < n * a.top_k; i += kFewThreads) {
      const int q = i / a.top_k;
      push(fresh_load(&parts[q].key[i - q * a.top_k]));
    }
    __syncthreads();
    if (s_n <= kFewKeys) {
      order_keys(s_keys, s_n, s_list);
    } else if (w == 0) {
      uint64_t key = 0;
      for (int i = 0; i < n; ++i) key = merge_lists(key, fresh_load(&parts[i].key[lane]), lane);
      s_list[lane] = key;
    }
    __syncthreads();
  }
  if (w == 0) {
    float fm = -CUDART_INF_F, f1 = 0.f, f2 = 0.f;
    int fc = 0;
    for (int i = lane; i < n; i += 32) {
      float qm = fresh_load(&parts[i].m), q1 = fresh_load(&parts[i].s1), q2 = fresh_load(&parts[i].s2);
      fc += fresh_load(&parts[i].count);
      const float to = max_nan(fm, qm);
      rebase(fm, f1, f2, to, a.c);
      rebase(qm, q1, q2, to, a.c);
      f1 += q1, f2 += q2;
    }
    float to = fm;
#pragma unroll
    for (int o = 16; o; o >>= 1) to = max_nan(to, __shfl_xor_sync(~0u, to, o));
    rebase(fm, f1, f2, to, a.c);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      f1 += __shfl_xor_sync(~0u, f1, o);
      f2 += __shfl_xor_sync(~0u, f2, o);
    }
    fc = __reduce_add_sync(~0u, fc);
    write_row(a, row, fm, f1, f2, fc, s_list[lane], t, xt);
  }
}

DeviceOnce g_once[6];

template <int DT, bool VEC>
seedq_status launch(ScoreArgs &a, int sms, int dev, cudaStream_t st) {
  constexpr int kPer = DT == SEEDQ_F32 ? 16 : 32, kTile = 32 * kPer, kChunk = kFewThreads * kPer;
  a.tiles = (a.vocab + kChunk - 1) / kChunk;
  // Few rows: 16 of 128256 with 20 alternatives take 12 us there and 23 below, 64
  // take 27 and 36, 256 with 5 take 78 and 44; rows of a tile or two are one
  // warp's work below (2000 of 1000: 21 and 13 us).
  if (a.vocab > 2 * kTile && a.rows * a.tiles <= kFewMax) {
    k_score_few<DT, VEC><<<(unsigned)(a.rows * a.tiles), kFewThreads, 0, st>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
  }
  a.tiles = (a.vocab + kTile - 1) / kTile;
  const int64_t total = a.rows * a.tiles;
  const int ctas = std::min(sms * kCtasPerSm, kMaxCtas);
  a.share = std::max<int64_t>((total + ctas - 1) / ctas, kWarps);
  a.ctas = (int)((total + a.share - 1) / a.share);
  constexpr size_t smem = (size_t)kWarps * kStages * kTileBytes + 128;
  const int rc = g_once[DT * 2 + VEC].run(dev, [] {
    return (int)cudaFuncSetAttribute(k_score<DT, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  });
  if (rc) return cuda_fail((cudaError_t)rc);
  k_score<DT, VEC><<<a.ctas, kThreads, smem, st>>>(a);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_token_logprobs_workspace_bytes(int64_t n_rows, int64_t vocab) {
  if (n_rows < 0 || vocab < 1) return 0;
  static_assert(kMaxCtas * 2 <= kFewMax, "");
  return kFewMax * 4 + (uint64_t)kFewMax * sizeof(Part);  // arrival counters and parts of rows
}

seedq_status seedq_token_logprobs(const void *logits, int32_t dtype, int64_t n_rows, int64_t vocab, int64_t row_stride,
                                  float scale, const int64_t *targets, float *logprob, float *entropy, int32_t *rank,
                                  int32_t top_k, float *top_logprob, int32_t *top_index, void *workspace,
                                  uint64_t workspace_bytes, void *cuda_stream) {
  if (!dtype_ok(dtype) || n_rows < 0 || n_rows > INT32_MAX || vocab < 1 || vocab > (1 << 30) || row_stride < vocab ||
      !std::isfinite(scale * kLog2e) || scale <= 0.f || top_k < 0 || top_k > kMaxTop)
    return SEEDQ_ERR_INVALID_ARG;
  if (n_rows == 0) return SEEDQ_OK;
  if (!logits || (targets && (!logprob || !rank)) || (top_k && (!top_logprob || !top_index)) || !workspace ||
      (uintptr_t)workspace % 16 || workspace_bytes < seedq_token_logprobs_workspace_bytes(n_rows, vocab))
    return SEEDQ_ERR_INVALID_ARG;
  ScoreArgs a{};
  a.x = logits, a.stride = row_stride, a.rows = n_rows, a.vocab = (int32_t)vocab, a.scale = scale, a.c = scale * kLog2e;
  a.targets = targets, a.logprob = logprob, a.entropy = entropy, a.rank = rank;
  a.top_k = top_k, a.top_logprob = top_logprob, a.top_index = top_index, a.workspace = workspace;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool vec = (uintptr_t)logits % 16 == 0 && (n_rows == 1 || row_stride * dtype_bytes(dtype) % 16 == 0);
  switch (dtype) {
    case SEEDQ_F32: return vec ? launch<SEEDQ_F32, true>(a, sms, dev, st) : launch<SEEDQ_F32, false>(a, sms, dev, st);
    case SEEDQ_BF16: return vec ? launch<SEEDQ_BF16, true>(a, sms, dev, st) : launch<SEEDQ_BF16, false>(a, sms, dev, st);
    default: return vec ? launch<SEEDQ_F16, true>(a, sms, dev, st) : launch<SEEDQ_F16, false>(a, sms, dev, st);
  }
}

}  // extern "C"
