// Beam search's choice over beams and vocabulary (seedq_beam_select).
//
// Mathematics.  With m the largest of a live beam's logits x, candidate (b, v) has
// the total score_b - ln sum exp(scale (x - m)) + scale (x_v - m), and a request's
// first n candidates by weight_b * total are wanted.  Within a beam the order is that of
// the logits themselves; between beams it is that of pairs of floats made from the
// logit, the score and the log sum, so candidates that lie close together are not
// swapped by a float32 sum.
//
// One pass over the logits keeps, per chunk of a row, the sum and the largest, and the
// largest per segment of 256 logits.  The first n candidates lie in the n segments
// whose largest logits come first in the same order: each of those n alone brings a
// candidate that precedes all of the others.  So the last CTA to arrive for a request
// chooses n segments from the maxima (of the chunks that can hold them), reads them
// again, and chooses from their logits.  Each choice is by a float32 bound that at
// least n reach, then by counting, for each of the few that do, how many precede it.
//
// Measured, n = twice the beams (the first: as many): a request of 4 beams of 32000
// logits 8.8 us, 4 requests of 4 beams of 128256 10.3 (the pass over the logits 3.9:
// launch, one trip to memory, an arrival), 64 of 8 beams of 128256 bfloat16 35 us (the
// pass 24, 4.4 TB/s).  The join is a chain of about fifteen trips to L2 or shared memory
// and barriers of one CTA, 5 to 7 us alone and 8.3 beside sixty others (sorted lists of
// 32 took 9 to 19), and many requests' joins fall at the end.  Segments of 256: what is
// read again is 1 KB a candidate, and a row of 128256 has 501 maxima, one look of a CTA
// at 4 beams.
//
// Where live beams have fewer segments than candidates are wanted, nothing bounds the
// chosen segments' logits; more than 256 of them are chosen one after another (one live
// beam of 300 logits, 4 chosen: 27 us; of 1000, 8 chosen: 44; of 7900, 32 chosen: 769,
// and 8000 10.9), as are about equal totals and numbers whose bounds float32 does not
// hold.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <cmath>

#include "cp_async.cuh"
#include "device_once.h"
#include "f32x2.cuh"
#include "order.cuh"
#include "overlap.h"
#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kSegment = 256;  // logits: 8 of each lane
constexpr int kMaxBeams = SEEDQ_MAX_BEAMS, kMaxTop = SEEDQ_MAX_BEAMS;
static_assert(kMaxBeams == 32, "a lane per beam and per candidate");
constexpr int kTokenBits = 27;
constexpr uint32_t kTokenMask = (1u << kTokenBits) - 1;
constexpr float kLog2e = 1.4426950408889634f;
constexpr uint64_t kHeader = 2 * SEEDQ_MAX_REQUESTS * 4 + 16;  // arrival counters of requests and of rows, a request on offer
// Logits from which on warps stream: 512 rows of 128256 bfloat16 (131 MB) take 35 us
// so and 42 by a CTA per chunk, 128 of float32 (66 MB) 25 and 22.
constexpr int64_t kStreamBytes = 96 << 20, kStreamVocab = 16384;

struct SelectArgs {
  const void *x;
  int64_t stride;
  int32_t vocab, beams, groups, segments, chunks, chunk_shift;  // of a row; segments of a chunk, a power of two
  float scale, c;                                  // c = scale * log2(e)
  const float *scores, *weights;
  const uint8_t *done;
  int32_t end_token, n_out;
  float *out_score;
  int32_t *out_beam, *out_token;
  int *counters;
  float2 *parts;  // maximum and sum of a row's chunks
  float *most;    // maximum of a row's segments
};

enum { kNone = 0, kLive = 1, kDone = 2 };  // what a beam brings

__device__ __forceinline__ int row_kind(const SelectArgs &a, int64_t row) {
  if (!(a.scores[row] > -CUDART_INF_F)) return kNone;  // a NaN is told apart at the join
  return a.done && a.done[row] ? kDone : kLive;
}

// A segment's logits as they lie in memory.  VEC: rows allow loads of 16 bytes;
// else lanes take single logits.  All rows of a call go one way, so that equal
// rows have equal sums, whatever their addresses.
template <int DT, bool VEC>
struct Segment {
  static constexpr int kSize = DT == SEEDQ_F32 ? 4 : 2, kVec = 16 / kSize, kPieces = 8 / kVec;
  uint32_t w[kPieces * 4];
  // The lane's element e of 8 within the segment.
  static __device__ __forceinline__ int place(int e, int lane) {
    return VEC ? (e / kVec) * (32 * kVec) + lane * kVec + e % kVec : e * 32 + lane;
  }
  static __device__ __forceinline__ uint32_t one(const char *row, int i, int vocab) {
    if (DT == SEEDQ_F32) return i < vocab ? ((const uint32_t *)row)[i] : 0xff800000u;
    return i < vocab ? ((const uint16_t *)row)[i] : DT == SEEDQ_BF16 ? 0xff80u : 0xfc00u;
  }
  __device__ __forceinline__ void load(const char *row, int first, int vocab, int lane) {
#pragma unroll
    for (int v = 0; v < kPieces; ++v) {
      const int i = first + place(v * kVec, lane);
      if (VEC && i + kVec <= vocab) {
        const uint4 y = __ldg((const uint4 *)(row + (int64_t)i * kSize));
        w[4 * v] = y.x, w[4 * v + 1] = y.y, w[4 * v + 2] = y.z, w[4 * v + 3] = y.w;
      } else {  // of a piece that the row's end cuts, what is there is read alone
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
          const uint32_t x = one(row, first + place(v * kVec + k, lane), vocab);
          if (DT == SEEDQ_F32) w[(4 * v + k) % (kPieces * 4)] = x;
          else if (k & 1) w[k / 2] |= x << 16;
          else w[k / 2] = x;
        }
      }
    }
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (DT == SEEDQ_F32) {
        x[e] = __uint_as_float(w[e % (kPieces * 4)]);
      } else {
        const uint32_t h = e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu;
        x[e] = DT == SEEDQ_BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
      }
    }
  }
};

// ---------------------------------------------------------------- candidates
//
// A candidate as two words that sort as candidates do: the weighted total as ordered
// numbers; then beam, logit and token, each such that what comes first is larger.  No
// candidate is (0, 0).
//
// Totals are pairs of floats, the nearest and the rest (46 bits; by the error-free
// sums and products of Knuth and Dekker): float64 instructions, few as they are, made
// the join 0.3 to 1 us longer.  Where a pair would overflow or underflow, the choice is
// made again in float64.
struct alignas(16) Item {
  uint64_t key, rest;
  __device__ __forceinline__ bool before(const Item &o) const { return (key > o.key) | ((key == o.key) & (rest > o.rest)); }
};
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair quick_sum(float a, float b) {  // |a| >= |b|
  const float s = __fadd_rn(a, b);
  return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ Pair exact_sum(float a, float b) {
  const float s = __fadd_rn(a, b), c = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, c)), __fsub_rn(b, c))};
}
__device__ __forceinline__ Pair exact_product(float a, float b) {
  const float p = __fmul_rn(a, b);
  return {p, __fmaf_rn(a, b, -p)};
}
__device__ __forceinline__ Pair sum(Pair a, Pair b) {
  const Pair s = exact_sum(a.hi, b.hi);
  return quick_sum(s.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)));
}
__device__ __forceinline__ Pair product(float a, Pair b) {
  const Pair p = exact_product(a, b.hi);
  return quick_sum(p.hi, __fmaf_rn(a, b.lo, p.lo));
}
__device__ __forceinline__ uint64_t order_double(double x) {
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
  return b >> 63 ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ uint64_t rest_word(int beam, uint32_t word, int index) {
  return (uint64_t)(31 - beam) << 59 | (uint64_t)word << kTokenBits | (kTokenMask - (uint32_t)index);
}
__device__ __forceinline__ int rest_beam(uint64_t rest) { return 31 - (int)(rest >> 59); }
__device__ __forceinline__ float rest_logit(uint64_t rest) { return key_value((rest >> kTokenBits) << 32); }
__device__ __forceinline__ int rest_index(uint64_t rest) { return (int)(kTokenMask - ((uint32_t)rest & kTokenMask)); }

constexpr int kMaxFound = 256;   // candidates of a choice: one of each thread
constexpr int kMaxChunks = 1024; // of a request, that the first look takes
constexpr int kAhead = 8;        // maxima that a thread has under way
constexpr int kLanesOfRow = 8;

struct Join {
  // total = base + scale * (logit - most): the difference first, or a large common part would take the sum's digits
  Pair base[kMaxBeams];
  float weight[kMaxBeams], most[kMaxBeams];
  float4 line[kMaxBeams];  // the same weighted, in float32: x * (logit - y) + z, and w = 2^-21 |z|; for a finished beam z alone
  int kind[kMaxBeams];
  alignas(16) float group[64];
  uint32_t words[kWarps];
  float chunk_most[kMaxChunks];
  uint32_t chunk[kMaxChunks];  // those that are looked at: beam << 16 and number
  Item found[kMaxFound], chosen[32];
  float found_x[kMaxFound];
  uint32_t found_at[kMaxFound];  // beam << 27 and index
  int n_chunks, n_found, n_chosen, spoiled, slow;  // slow: numbers too large for float32 bounds
};

__device__ __forceinline__ double total_of(const SelectArgs &a, const Join &s, int b, float x) {
  const double base = (double)s.base[b].hi + (double)s.base[b].lo;
  return s.kind[b] == kDone ? base : base + (double)a.scale * ((double)x - (double)s.most[b]);
}
__device__ __forceinline__ Item item_of(const SelectArgs &a, const Join &s, int b, float x, int index) {
  return {order_double((double)s.weight[b] * total_of(a, s, b, x)), rest_word(b, order_word(x), index)};
}
__device__ __forceinline__ Pair quick_total(const SelectArgs &a, const Join &s, int b, float x) {
  const Pair base = s.base[b];
  return s.kind[b] == kDone ? base : sum(base, product(a.scale, exact_sum(x, -s.most[b])));
}
// fine: false where a pair has no room, by its size or its smallness.
__device__ __forceinline__ Item quick_item(const SelectArgs &a, const Join &s, int b, float x, int index, bool &fine) {
  const Pair total = quick_total(a, s, b, x), y = product(s.weight[b], total);
  fine = fabsf(y.hi) < CUDART_INF_F && fabsf(y.lo) < CUDART_INF_F && (fabsf(y.hi) > 0x1p-70f || total.hi == 0.f);
  return {(uint64_t)order_word(y.hi) << 32 | order_word(y.lo), rest_word(b, order_word(x), index)};
}
// Bounds of the weighted total in float32: of its parts' few roundings, here 2^-21 of
// them.  What is far down is cut off, for all beams alike (their offsets are at most
// 1e29).  -inf of what is no candidate.
__device__ __forceinline__ float lower(const float4 l, float x) {
  const float d = fmaxf(l.x * (x - l.y), -1e37f), y = fmaf(fminf(d, 0.f), 0x1p-21f, d) + (l.z - l.w);  // d is at most 0 but for roundings
  return x > -CUDART_INF_F ? y : -CUDART_INF_F;
}
__device__ __forceinline__ float upper(const float4 l, float x) {
  const float d = fmaxf(l.x * (x - l.y), -1e37f), y = fmaf(fminf(d, 0.f), -0x1p-21f, d) + (l.z + l.w);
  return x > -CUDART_INF_F ? y : -CUDART_INF_F;
}
// Which of 256 items in a row a thread takes: such that the first 64 fall into 64
// different groups of four threads.
__device__ __forceinline__ int item_slot() { return (threadIdx.x & 3) * 64 + (threadIdx.x >> 2); }
// Of the threads' values (lower bounds of candidates' totals) the largest of every four:
// the n-th largest of those 64, -inf if fewer have any.  At least n candidates reach it.
__device__ __forceinline__ float nth_bound(Join &s, float mine, int n) {
  const int tid = threadIdx.x, lane = tid & 31;
  mine = fmaxf(mine, __shfl_xor_sync(~0u, mine, 1));
  mine = fmaxf(mine, __shfl_xor_sync(~0u, mine, 2));
  if (tid % 4 == 0) s.group[tid / 4] = mine;
  __syncthreads();
  int above = 0;  // each of the four looks at 16
#pragma unroll
  for (int k = 0; k < 16; k += 4) {
    const float4 v = *(const float4 *)(s.group + (tid & 3) * 16 + k);
    above += (v.x > mine) + (v.y > mine) + (v.z > mine) + (v.w > mine);
  }
  above += __shfl_xor_sync(~0u, above, 1);
  above += __shfl_xor_sync(~0u, above, 2);
  const uint32_t word = __reduce_min_sync(~0u, above < n ? order_word(mine) : ~0u);
  if (lane == 0) s.words[tid / 32] = word;
  __syncthreads();
  const uint32_t least = __reduce_min_sync(~0u, s.words[lane % kWarps]);
  return key_value((uint64_t)least << 32);
}
// The first n of the found candidates, in order, to chosen.  False if more were
// found than fit, or pairs do not hold some.
__device__ __forceinline__ bool rank_found(const SelectArgs &a, Join &s, int n) {
  __syncthreads();
  const int m = s.n_found;
  if (m > kMaxFound) return false;
  Item mine{0, 0};
  if (threadIdx.x < m) {
    const uint32_t at = s.found_at[threadIdx.x];
    bool fine;
    mine = quick_item(a, s, at >> kTokenBits, s.found_x[threadIdx.x], at & kTokenMask, fine);
    s.found[threadIdx.x] = mine;
    if (!fine) s.slow = 1;
  }
  __syncthreads();
  if (s.slow) return false;
  // several threads count for one candidate
  const int share = m <= 32 ? 8 : m <= 64 ? 4 : m <= 128 ? 2 : 1, i = threadIdx.x / share;
  mine = s.found[min(i, kMaxFound - 1)];
  int before = 0;
  if (i < m) {
#pragma unroll 4
    for (int k = threadIdx.x % share; k < m; k += share) {
      const ulonglong2 y = *(const ulonglong2 *)&s.found[k];
      before += Item{y.x, y.y}.before(mine);
    }
  }
  for (int o = share / 2; o; o >>= 1) before += __shfl_xor_sync(~0u, before, o);
  if (i < m && before < n && threadIdx.x % share == 0) s.chosen[before] = mine;
  if (threadIdx.x == 0) s.n_chosen = min(m, n);
  __syncthreads();
  return true;
}
__device__ __forceinline__ void push(Join &s, int b, float x, int index) {
  const int at = atomicAdd(&s.n_found, 1);
  if (at < kMaxFound) s.found_x[at] = x, s.found_at[at] = (uint32_t)b << kTokenBits | (uint32_t)index;
}

// For rows in which more than fit are about equal or nothing bounds them, or numbers
// too large or small for the bounds: the n first one after another.  each(f) calls
// f(beam, logit, index) for all that the thread sees.
template <typename Each>
__device__ __forceinline__ void choose_slowly(const SelectArgs &a, Join &s, Each each) {
  Item last = {~0ull, ~0ull};
  __syncthreads();
  if (threadIdx.x == 0) s.n_chosen = 0;
#pragma unroll 1
  for (int i = 0; i < a.n_out; ++i) {
    Item best = {0, 0};
    each([&](int b, float x, int index) {
      const Item y = item_of(a, s, b, x, index);
      if (last.before(y) && y.before(best)) best = y;
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const Item y{__shfl_xor_sync(~0u, best.key, o), __shfl_xor_sync(~0u, best.rest, o)};
      if (y.before(best)) best = y;
    }
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.found[threadIdx.x >> 5] = best;
    __syncthreads();
    best = s.found[0];
    for (int k = 1; k < kWarps; ++k)
      if (s.found[k].before(best)) best = s.found[k];
    if (!best.key) break;
    if (threadIdx.x == 0) s.chosen[i] = best, s.n_chosen = i + 1;
    last = best;
  }
  __syncthreads();
}

template <int DT, bool VEC>
__device__ __noinline__ void join_slowly(const SelectArgs a, Join &s, int64_t g) {  // by value: the kernel's own stay in constant memory
  using Seg = Segment<DT, VEC>;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  __syncthreads();
  if (threadIdx.x == 0) s.slow = 1;  // for who writes the results
  choose_slowly(a, s, [&](auto &&f) {
    for (int b = 0; b < a.beams; ++b) {
      if (s.kind[b] == kDone && threadIdx.x == 0) f(b, 0.f, a.end_token);
      if (s.kind[b] != kLive) continue;
      for (int i = threadIdx.x; i < a.segments; i += kThreads) {
        const float x = __ldcg(a.most + (g * a.beams + b) * a.segments + i);
        if (x > -CUDART_INF_F) f(b, x, i);
      }
    }
  });
  const Item mine = s.chosen[lane];
  const int n_chosen = s.n_chosen;
  choose_slowly(a, s, [&](auto &&f) {
    for (int i = w; i < n_chosen; i += kWarps) {
      const uint64_t rest = __shfl_sync(~0u, mine.rest, i);
      const int b = rest_beam(rest), first = rest_index(rest) * kSegment;
      if (s.kind[b] == kDone) {
        if (lane == 0) f(b, 0.f, a.end_token);
        continue;
      }
      Seg seg;
      seg.load((const char *)a.x + (g * a.beams + b) * a.stride * Seg::kSize, first, a.vocab, lane);
      float x[8];
      seg.get(x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (x[e] > -CUDART_INF_F) f(b, x[e], first + Seg::place(e, lane));
    }
  });
}

__device__ __forceinline__ bool by_chunks(const SelectArgs &a) {
  return a.beams * a.chunks <= kMaxChunks && a.beams * a.segments > kThreads * kAhead;
}
// The first segments' maxima, of all rows.
__device__ __forceinline__ void load_first(const SelectArgs &a, int64_t g, float (&ahead)[kAhead]) {
  const int total = a.beams * a.segments, slot = item_slot();
#pragma unroll
  for (int k = 0; k < kAhead; ++k) ahead[k] = k * kThreads + slot < total ? __ldcg(a.most + g * total + k * kThreads + slot) : -CUDART_INF_F;
}

template <int DT, bool VEC>
__device__ __forceinline__ void join_fast(const SelectArgs &a, Join &s, int64_t g, float (&ahead)[kAhead]) {
  using Seg = Segment<DT, VEC>;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, slot = item_slot();
  const int chunks = a.beams * a.chunks, shift = a.chunk_shift;
  const float per_chunk = 1.f / (float)a.chunks;
  auto beam_of = [&](int k) { return (int)(((float)k + 0.5f) * per_chunk); };  // off by 2^-17 at most, and 2^-11 from the next beam
  float bound = -CUDART_INF_F;
  // chunks, by their largest logits: of those whose upper bound reaches the n-th lower one the segments are looked at
  const bool few = by_chunks(a);
  if (few) {
    for (int k = slot; k < chunks; k += kThreads) {
      const int b = beam_of(k);
      if (s.kind[b] == kLive) bound = fmaxf(bound, lower(s.line[b], s.chunk_most[k]));
    }
    bound = nth_bound(s, bound, a.n_out);
    for (int k = slot; k < chunks; k += kThreads) {
      const int b = beam_of(k);
      if (s.kind[b] == kLive && s.chunk_most[k] > -CUDART_INF_F && upper(s.line[b], s.chunk_most[k]) >= bound)
        s.chunk[atomicAdd(&s.n_chunks, 1)] = (uint32_t)b << 16 | (uint32_t)(k - b * a.chunks);
    }
    __syncthreads();
  }
  // segments, by their largest logits; a finished beam is a segment of its one candidate
  const int total = few ? s.n_chunks << shift : a.beams * a.segments;
  int beam[kAhead], number[kAhead];
  const int step_b = kThreads / a.segments, step_i = kThreads - step_b * a.segments;
  auto load = [&](int first) {
    int b = 0, i = 0;  // of the item that k comes to
    if (!few) b = (first + slot) / a.segments, i = first + slot - b * a.segments;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int at = first + k * kThreads + slot;
      beam[k] = number[k] = 0;
      if (few) {
        const uint32_t c = at < total ? s.chunk[at >> shift] : 0;
        beam[k] = c >> 16, number[k] = (int)(c & 0xffffu) << shift | (at & ((1 << shift) - 1));
        ahead[k] = at < total && number[k] < a.segments ? __ldcg(a.most + (g * a.beams + beam[k]) * a.segments + number[k]) : -CUDART_INF_F;
      } else if (at < total) {
        beam[k] = b, number[k] = i;
        if (first) ahead[k] = __ldcg(a.most + g * a.beams * a.segments + at);
        if (s.kind[b] != kLive) ahead[k] = -CUDART_INF_F;  // the row holds anything
      } else {
        ahead[k] = -CUDART_INF_F;
      }
      b += step_b, i += step_i;
      if (i >= a.segments) i -= a.segments, ++b;
    }
  };
  const bool ends = tid < a.beams && s.kind[tid] == kDone;
  bound = ends ? s.line[tid].z - s.line[tid].w : -CUDART_INF_F;
  for (int first = 0; first < total; first += kThreads * kAhead) {
    load(first);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      bound = fmaxf(bound, lower(s.line[beam[k]], ahead[k]));
  }
  bound = nth_bound(s, bound, a.n_out);
  if (ends && s.line[tid].z + s.line[tid].w >= bound) push(s, tid, 0.f, a.end_token);
  for (int first = 0; first < total; first += kThreads * kAhead) {
    if (total > kThreads * kAhead) {
      if (!few && first == 0) load_first(a, g, ahead);
      load(first);
    }
    uint32_t in = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      in |= (uint32_t)((upper(s.line[beam[k]], ahead[k]) >= bound) & (ahead[k] > -CUDART_INF_F)) << k;
    while (in) {
      const int k = __ffs(in) - 1;
      in &= in - 1;
      float x = ahead[0];
      int b = beam[0], i = number[0];
#pragma unroll
      for (int z = 1; z < kAhead; ++z)
        if (k == z) x = ahead[z], b = beam[z], i = number[z];
      push(s, b, x, i);
    }
  }
  if (!rank_found(a, s, a.n_out)) return join_slowly<DT, VEC>(a, s, g);

  // their logits
  const int n_chosen = s.n_chosen;
  bound = -CUDART_INF_F;
  if (n_chosen == a.n_out) {  // no candidate comes behind the last segment's best
    const Item last = s.chosen[n_chosen - 1];
    const int b = rest_beam(last.rest);
    bound = s.kind[b] == kDone ? s.line[b].z - s.line[b].w : lower(s.line[b], rest_logit(last.rest));
  }
  constexpr int kEach = kMaxTop / kWarps;
  Seg seg[kEach];
  int of[kEach], at[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = w + k * kWarps;
    of[k] = -1;
    if (i < n_chosen) {
      const uint64_t rest = s.chosen[i].rest;
      of[k] = rest_beam(rest), at[k] = rest_index(rest) * kSegment;
      if (s.kind[of[k]] == kLive) seg[k].load((const char *)a.x + (g * a.beams + of[k]) * a.stride * Seg::kSize, at[k], a.vocab, lane);
    }
  }
  __syncthreads();
  if (tid == 0) s.n_found = 0;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    if (of[k] < 0) continue;
    const int b = of[k];
    if (s.kind[b] == kDone) {
      if (lane == 0) push(s, b, 0.f, a.end_token);
      continue;
    }
    float x[8];
    seg[k].get(x);
    const float4 line = s.line[b];
    uint32_t in = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) in |= (uint32_t)((upper(line, x[e]) >= bound) & (x[e] > -CUDART_INF_F)) << e;
    while (in) {
      const int e = __ffs(in) - 1;
      in &= in - 1;
      float y = x[0];
#pragma unroll
      for (int z = 1; z < 8; ++z) y = e == z ? x[z] : y;
      push(s, b, y, at[k] + Seg::place(e, lane));
    }
  }
  if (!rank_found(a, s, a.n_out)) return join_slowly<DT, VEC>(a, s, g);
}

template <int DT, bool VEC>
__device__ __forceinline__ void join_group(const SelectArgs &a, Join &s, int64_t g) {
  const int tid = threadIdx.x;
  if (tid == 0) s.spoiled = s.slow = s.n_found = s.n_chosen = s.n_chunks = 0;
  __syncthreads();
  // the sums of the beams, 8 lanes each: all at once
  static_assert(kThreads / kLanesOfRow == kMaxBeams, "");
  const int b = tid / kLanesOfRow, part = tid % kLanesOfRow;
  const bool there = b < a.beams;
  const int64_t row = g * a.beams + (there ? b : 0);
  const float score = a.scores[row];
  const float weight = a.weights ? a.weights[row] : 1.f;
  int kind = there ? row_kind(a, row) : kNone;
  const bool keep = a.beams * a.chunks <= kMaxChunks;
  float ahead[kAhead];
  if (!by_chunks(a)) load_first(a, g, ahead);  // on their way while the sums are made
  constexpr int kEarly = 4;  // parts under way before the beam's kind is known
  float2 early[kEarly];
#pragma unroll
  for (int k = 0; k < kEarly; ++k)
    if (part + k * kLanesOfRow < a.chunks) early[k] = __ldcg(a.parts + row * a.chunks + part + k * kLanesOfRow);
  float m = -CUDART_INF_F, sum = 0.f;
  if (kind == kLive) {
#pragma unroll 4
    for (int k = 0, i = part; i < a.chunks; i += kLanesOfRow, ++k) {
      float2 p = early[0];
      early[0] = early[1], early[1] = early[2], early[2] = early[3];
      if (k >= kEarly) p = __ldcg(a.parts + row * a.chunks + i);
      if (keep) s.chunk_most[b * a.chunks + i] = p.x;
      const float to = max_nan(m, p.x);
      if (to != -CUDART_INF_F) sum = sum * exp2_fast((m - to) * a.c) + p.y * exp2_fast((p.x - to) * a.c);
      m = to;
    }
  }
  float to = m;
#pragma unroll
  for (int o = kLanesOfRow / 2; o; o >>= 1) to = max_nan(to, __shfl_xor_sync(~0u, to, o));
  if (to != -CUDART_INF_F) sum *= exp2_fast((m - to) * a.c);
#pragma unroll
  for (int o = kLanesOfRow / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
  if (there && part == 0) {
    Pair base{score, 0.f};
    float high = 0.f;
    bool bad = isnan(score) || (kind != kNone && !(score < CUDART_INF_F && weight > 0.f && weight < CUDART_INF_F));
    if (kind == kLive) {
      if (to == -CUDART_INF_F) {
        kind = kNone;  // no token is allowed
      } else if (!(sum < CUDART_INF_F)) {
        bad = true;
      } else {
        // ln sum = e ln 2 + ln f, f within 0.7 and 1.42: float32 errors of the small logarithm alone
        const int e = (int)(__float_as_uint(sum * 1.41421356f) >> 23) - 127;
        const float f = sum * __uint_as_float((uint32_t)(127 - e) << 23);
        constexpr float kLn2 = 0.693147182f, kLn2Rest = -1.9046543e-9f;  // together ln 2 to 2^-50
        const Pair log_sum = seedq::sum(product((float)e, Pair{kLn2, kLn2Rest}), Pair{logf(f), 0.f});
        base = seedq::sum(base, Pair{-log_sum.hi, -log_sum.lo});
        high = to;
      }
    }
    const float offset = weight * base.hi, slope = kind == kLive ? weight * a.scale : 0.f;
    s.base[b] = base, s.weight[b] = weight, s.most[b] = high, s.kind[b] = kind;
    s.line[b] = kind == kNone ? make_float4(0.f, 0.f, -CUDART_INF_F, 0.f) : make_float4(slope, high, offset, 0x1p-21f * fabsf(offset));
    // the bounds' margins need room at both ends, an infinite slope times no difference is no number, and a logit
    // of -float32's largest must not lie infinitely far below the beam's own largest
    const float smallest = kind == kLive ? fminf(weight, slope) : weight;
    if (kind != kNone && !(fabsf(offset) <= 1e29f && smallest >= 0x1p-80f && slope < CUDART_INF_F && high <= 0x1p100f)) s.slow = 1;
    if (bad) s.spoiled = 1;
  }
  __syncthreads();
  const bool spoiled = s.spoiled;  // the same in all threads
  if (!spoiled) {
    if (s.slow) join_slowly<DT, VEC>(a, s, g);
    else join_fast<DT, VEC>(a, s, g, ahead);
  }
  if (tid < a.n_out) {
    const int64_t o = g * a.n_out + tid;
    const bool has = !spoiled && tid < s.n_chosen;
    const Item x = has ? s.chosen[tid] : Item{0, 0};
    const int from = rest_beam(x.rest);
    const float total = !has ? -CUDART_INF_F : s.slow ? (float)total_of(a, s, from, rest_logit(x.rest)) : quick_total(a, s, from, rest_logit(x.rest)).hi;
    a.out_score[o] = spoiled ? CUDART_NAN_F : total;
    a.out_beam[o] = has ? from : -1;
    a.out_token[o] = has ? rest_index(x.rest) : -1;
  }
  __syncthreads();
}

// Few logits: a CTA per chunk of a row, all of it read at once.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) k_beam_select(const __grid_constant__ SelectArgs a) {
  using Seg = Segment<DT, VEC>;
  constexpr int kEach = Seg::kSize == 4 ? 4 : 8;  // segments of a warp
  __shared__ Join s_join;
  __shared__ float2 s_part[kWarps];
  __shared__ bool s_last;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t row = blockIdx.x / (uint32_t)a.chunks;
  const int chunk = (int)(blockIdx.x - (uint32_t)row * a.chunks);
  if (row_kind(a, row) == kLive) {
    const char *base = (const char *)a.x + row * a.stride * Seg::kSize;
    const int s0 = chunk * (kEach * kWarps) + w;
    Seg seg[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) seg[j].load(base, (s0 + j * kWarps) * kSegment, a.vocab, lane);
    float m = -CUDART_INF_F;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      float x[8];
      seg[j].get(x);
      float mx = max_nan(x[0], x[1]);
#pragma unroll
      for (int e = 2; e < 8; e += 2) mx = max_nan(mx, x[e], x[e + 1]);
      mx = warp_max_nan(mx);
      m = max_nan(m, mx);
      if (lane == 0 && s0 + j * kWarps < a.segments) a.most[row * a.segments + s0 + j * kWarps] = mx;
    }
    const float off = m == -CUDART_INF_F ? 0.f : -m;
    const uint64_t off2 = f2_pack(off, off), c2 = f2_pack(a.c, a.c);
    uint64_t sums = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      float x[8];
      seg[j].get(x);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float2 d = f2_unpack(f2_mul(f2_add(f2_pack(x[e], x[e + 1]), off2), c2));
        sums = f2_add(sums, f2_pack(exp2_fast(d.x), exp2_fast(d.y)));
      }
    }
    float sum = f2_unpack(sums).x + f2_unpack(sums).y;
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) s_part[w] = make_float2(m, sum);
    __syncthreads();
    if (w == 0) {
      const float2 p = lane < kWarps ? s_part[lane] : make_float2(-CUDART_INF_F, 0.f);
      float to = p.x;
#pragma unroll
      for (int o = kWarps / 2; o; o >>= 1) to = max_nan(to, __shfl_xor_sync(~0u, to, o));
      float t = to == -CUDART_INF_F ? 0.f : p.y * exp2_fast((p.x - to) * a.c);
#pragma unroll
      for (int o = kWarps / 2; o; o >>= 1) t += __shfl_xor_sync(~0u, t, o);
      if (lane == 0) a.parts[row * a.chunks + chunk] = make_float2(to, t);
    }
  }
  const int64_t g = row / a.beams;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    s_last = atomicAdd(a.counters + g, 1) == a.beams * a.chunks - 1;
    if (s_last) a.counters[g] = 0;
    __threadfence();
  }
  __syncthreads();
  if (s_last) join_group<DT, VEC>(a, s_join, g);
}

// Many logits: warps stream through equal ranges of the live rows' chunks, a ring of
// copies ahead; a row's chunks are the same for all rows, so that equal rows have
// equal sums.  A row counts its chunks, a request its rows; the CTA of the warp that
// brings the last joins the request once its own range is done.  A CTA that has two
// to join, which would end 7 us after the others, offers one to those whose range ends
// later, and takes back what is still there after its own.
constexpr int kStages = 3;          // tiles in a warp's ring
constexpr int kTileBytes = 2048;    // 64 bytes of each lane
constexpr int kChunkTiles = 4;
constexpr int kMaxJoins = 128;
constexpr int kStreamCtas = 2;      // per SM
template <int DT>
__global__ void __launch_bounds__(kThreads, kStreamCtas) k_beam_stream(const __grid_constant__ SelectArgs a) {
  using Seg = Segment<DT, true>;
  constexpr int kSize = Seg::kSize, kVec = Seg::kVec, kTile = kTileBytes / kSize, kSegs = kTile / kSegment;
  extern __shared__ __align__(128) uint8_t s_ring[];
  uint16_t *live = (uint16_t *)(s_ring + kWarps * kStages * kTileBytes);  // the live rows
  __shared__ Join s_join;
  __shared__ int s_count[kWarps], s_joins[kMaxJoins], s_n_joins, s_offers;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  if (tid == 0) s_n_joins = 0;
  int n_live = 0;
  const int rows = a.groups * a.beams;
  constexpr int kRounds = 2;  // whose rows are looked at together
  bool ahead[kRounds];
#pragma unroll
  for (int k = 0; k < kRounds; ++k) ahead[k] = k * kThreads + tid < rows && row_kind(a, k * kThreads + tid) == kLive;
  for (int r0 = 0, k = 0; r0 < rows; r0 += kThreads, ++k) {
    const bool is = k < kRounds ? ahead[0] : r0 + tid < rows && row_kind(a, r0 + tid) == kLive;
    ahead[0] = ahead[1];
    const uint32_t mask = __ballot_sync(~0u, is);
    if (lane == 0) s_count[w] = __popc(mask);
    __syncthreads();
    int before = 0, all = 0;
    for (int k = 0; k < kWarps; ++k) {
      before += k < w ? s_count[k] : 0;
      all += s_count[k];
    }
    if (is) live[n_live + before + __popc(mask & ((1u << lane) - 1))] = (uint16_t)(r0 + tid);
    n_live += all;
    __syncthreads();
  }
  auto live_of_group = [&](int g) { return __popc(__ballot_sync(~0u, lane < a.beams && row_kind(a, (int64_t)g * a.beams + lane) == kLive)); };
  // requests without a live beam are nobody's last
  for (int g = blockIdx.x; g < a.groups; g += gridDim.x)
    if (w == 0 && live_of_group(g) == 0 && lane == 0) s_joins[s_n_joins++] = g;
  __syncthreads();

  const int64_t tasks = (int64_t)n_live * a.chunks, warps = (int64_t)gridDim.x * kWarps, me = (int64_t)blockIdx.x * kWarps + w;
  const int64_t t0 = tasks * me / warps, t1 = tasks * (me + 1) / warps;
  const int tiles = (a.vocab + kTile - 1) / kTile;  // of a row
  uint8_t *ring = s_ring + w * (kStages * kTileBytes) + lane * 16;
  // where the copies are: live row, tile
  int li = (int)(t0 / a.chunks), pi = li, ptile = (int)(t0 - (int64_t)li * a.chunks) * kChunkTiles, chunk = ptile / kChunkTiles, pstage = 0, stage = 0;
  // tiles left to copy
  int64_t pleft = 0;
  if (t0 < t1) {
    const int le = (int)((t1 - 1) / a.chunks), ce = (int)(t1 - 1 - (int64_t)le * a.chunks);
    pleft = (int64_t)(le - li) * tiles + min((ce + 1) * kChunkTiles, tiles) - ptile;
  }
  const char *psrc = t0 < t1 ? (const char *)a.x + (int64_t)live[pi] * a.stride * kSize : nullptr;
  auto issue = [&]() {
    if (pleft > 0) {
      const uint32_t dst = (uint32_t)__cvta_generic_to_shared(ring + pstage * kTileBytes);
      if ((ptile + 1) * kTile <= a.vocab) {
        const char *from = psrc + ptile * kTileBytes + lane * 16;
#pragma unroll
        for (int v = 0; v < 4; ++v) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + v * 512), "l"(from + v * 512) : "memory");
      } else
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int i = ptile * kTile + v * (32 * kVec) + lane * kVec;
        const int bytes = min(max(a.vocab - i, 0) * kSize, 16);  // what lies past the row's end is not read
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + v * 512),
                     "l"(bytes ? psrc + (int64_t)i * kSize : (const char *)a.x), "r"(bytes)
                     : "memory");
      }
      --pleft;
      pstage = pstage + 1 == kStages ? 0 : pstage + 1;
      if (++ptile == tiles && pleft > 0) {
        ptile = 0;
        psrc = (const char *)a.x + (int64_t)live[++pi] * a.stride * kSize;
      }
    }
    cp_async_commit();
  };
  for (int k = 0; k < kStages - 1; ++k) issue();
  int pending = 0;  // chunks of the row that nobody knows of yet
  auto arrive = [&](int64_t row) {
    __syncwarp();
    const int g = (int)(row / a.beams), n = live_of_group(g);
    if (lane == 0) {
      __threadfence();
      if (atomicAdd(a.counters + SEEDQ_MAX_REQUESTS + row, pending) + pending == a.chunks) {
        a.counters[SEEDQ_MAX_REQUESTS + row] = 0;
        __threadfence();
        if (atomicAdd(a.counters + g, 1) + 1 == n) {
          a.counters[g] = 0;
          s_joins[atomicAdd(&s_n_joins, 1)] = g;
        }
      }
    }
    pending = 0;
  };
  const uint64_t c2 = f2_pack(a.c, a.c);
  for (int64_t t = t0; t < t1; ++t) {
    const int64_t row = live[li];
    float m = -CUDART_INF_F;
    float sum = 0.f;
    const int last = min((chunk + 1) * kChunkTiles, tiles);
    for (int tile = chunk * kChunkTiles; tile < last; ++tile) {
      issue();
      cp_async_wait<kStages - 1>();
      const uint8_t *src = ring + stage * kTileBytes;
      stage = stage + 1 == kStages ? 0 : stage + 1;
      Seg seg[kSegs];
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const uint4 y = *(const uint4 *)(src + v * 512);
        uint32_t *to = seg[v / Seg::kPieces].w + (v % Seg::kPieces) * 4;
        to[0] = y.x, to[1] = y.y, to[2] = y.z, to[3] = y.w;
      }
      float x[kSegs][8];
#pragma unroll
      for (int k = 0; k < kSegs; ++k) seg[k].get(x[k]);
      if ((tile + 1) * kTile > a.vocab) {
#pragma unroll
        for (int k = 0; k < kSegs; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (tile * kTile + k * kSegment + Seg::place(e, lane) >= a.vocab) x[k][e] = -CUDART_INF_F;
      }
      float to = m, mine = 0.f;
#pragma unroll
      for (int k = 0; k < kSegs; ++k) {
        float mx = max_nan(x[k][0], x[k][1]);
#pragma unroll
        for (int e = 2; e < 8; e += 2) mx = max_nan(mx, x[k][e], x[k][e + 1]);
        mx = warp_max_nan(mx);
        to = max_nan(to, mx);
        if (lane == k) mine = mx;
      }
      if (lane < kSegs && tile * kSegs + lane < a.segments) a.most[row * a.segments + tile * kSegs + lane] = mine;
      if (to != -CUDART_INF_F) sum *= exp2_fast((m - to) * a.c);
      m = to;
      const float off = to == -CUDART_INF_F ? 0.f : -to;
      const uint64_t off2 = f2_pack(off, off);
      uint64_t sums = 0;
#pragma unroll
      for (int k = 0; k < kSegs; ++k)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float2 d = f2_unpack(f2_mul(f2_add(f2_pack(x[k][e], x[k][e + 1]), off2), c2));
          sums = f2_add(sums, f2_pack(exp2_fast(d.x), exp2_fast(d.y)));
        }
      sum += f2_unpack(sums).x + f2_unpack(sums).y;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
    if (lane == 0) a.parts[row * a.chunks + chunk] = make_float2(m, sum);
    ++pending;
    if (++chunk == a.chunks) {
      arrive(row);
      chunk = 0;
      ++li;
    }
  }
  if (pending) arrive(live[li]);
  cp_async_wait<0>();
  __syncthreads();
  int *const offer = a.counters + 2 * SEEDQ_MAX_REQUESTS;  // a request + 1, or 0
  if (tid == 0) {
    __threadfence();
    const int n = s_n_joins;
    s_offers = n > 1 && atomicCAS(offer, 0, s_joins[n - 1] + 1) == 0;
    if (s_offers) s_n_joins = n - 1;
    if (n == 0 && (s_joins[0] = atomicExch(offer, 0) - 1) >= 0) s_n_joins = 1;
  }
  __syncthreads();
  __threadfence();
  const int joins = s_n_joins, offers = s_offers;
  for (int k = 0; k < joins + offers; ++k) {
    if (k == joins) {
      if (tid == 0) s_joins[k] = atomicExch(offer, 0) - 1;  // its own, another's or none
      __syncthreads();
      if (s_joins[k] < 0) break;
      __threadfence();
    }
    join_group<DT, true>(a, s_join, s_joins[k]);
  }
}

int few_chunk_logits(int32_t dtype) { return (dtype == SEEDQ_F32 ? 4 : 8) * kWarps * kSegment; }
int stream_chunk_logits(int32_t dtype) { return kChunkTiles * kTileBytes / dtype_bytes(dtype); }
int64_t segments_of(int64_t vocab) { return (vocab + kSegment - 1) / kSegment; }

DeviceOnce g_stream[3];

template <int DT>
cudaError_t launch(SelectArgs &a, bool vec, cudaStream_t st) {
  const int64_t rows = (int64_t)a.groups * a.beams;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return e;
  const bool many = rows * a.vocab * dtype_bytes(DT) >= kStreamBytes && a.vocab >= kStreamVocab;
  if (vec && many && rows <= (int64_t)sms * kStreamCtas * kMaxJoins / 4) {  // a CTA meets a quarter as many rows, and as many requests without any
    constexpr size_t kSmem = kWarps * kStages * kTileBytes + SEEDQ_MAX_REQUESTS * sizeof(uint16_t);
    const int rc = g_stream[DT].run(dev, [] {
      return (int)cudaFuncSetAttribute(k_beam_stream<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    });
    if (rc) return (cudaError_t)rc;
    a.chunks = (a.vocab + stream_chunk_logits(DT) - 1) / stream_chunk_logits(DT);
    a.chunk_shift = __builtin_ctz(stream_chunk_logits(DT) / kSegment);
    a.most = (float *)(a.parts + rows * a.chunks);
    k_beam_stream<DT><<<sms * kStreamCtas, kThreads, kSmem, st>>>(a);
  } else {
    a.chunks = (a.vocab + few_chunk_logits(DT) - 1) / few_chunk_logits(DT);
    a.chunk_shift = __builtin_ctz(few_chunk_logits(DT) / kSegment);
    a.most = (float *)(a.parts + rows * a.chunks);
    const unsigned ctas = (unsigned)(rows * a.chunks);  // at most 2^13 * 2^14
    if (vec) k_beam_select<DT, true><<<ctas, kThreads, 0, st>>>(a);
    else k_beam_select<DT, false><<<ctas, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
}

bool sizes_ok(int64_t groups, int32_t beams, int64_t vocab) {
  return groups >= 0 && beams >= 1 && beams <= kMaxBeams && groups * beams <= SEEDQ_MAX_REQUESTS && groups <= SEEDQ_MAX_REQUESTS &&
         vocab >= 1 && vocab <= SEEDQ_BEAM_MAX_VOCAB;
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_beam_select_workspace_bytes(int64_t n_groups, int32_t n_beams, int64_t vocab) {
  if (!sizes_ok(n_groups, n_beams, vocab)) return 0;
  const uint64_t rows = (uint64_t)n_groups * n_beams, segments = (uint64_t)segments_of(vocab);
  const uint64_t chunks = ((uint64_t)vocab + stream_chunk_logits(SEEDQ_F32) - 1) / stream_chunk_logits(SEEDQ_F32);  // the smallest
  return kHeader + rows * (chunks * sizeof(float2) + segments * sizeof(float));
}

seedq_status seedq_beam_select(const seedq_beam_select_args *args, void *cuda_stream) {
  if (!args) return SEEDQ_ERR_INVALID_ARG;
  const seedq_beam_select_args &p = *args;
  if (!dtype_ok(p.dtype) || !sizes_ok(p.n_groups, p.n_beams, p.vocab) || p.row_stride < p.vocab || p.n_out < 1 || p.n_out > kMaxTop ||
      !(p.scale >= 0x1p-64f && p.scale <= 0x1p64f))
    return SEEDQ_ERR_INVALID_ARG;
  if (p.n_groups == 0) return SEEDQ_OK;
  if (!p.logits || !p.scores || !p.out_score || !p.out_beam || !p.out_token || !p.workspace || (uintptr_t)p.workspace % 16 ||
      p.workspace_bytes < seedq_beam_select_workspace_bytes(p.n_groups, p.n_beams, p.vocab) ||
      (p.done && (p.end_token < 0 || p.end_token >= p.vocab)) || (uintptr_t)p.logits % dtype_bytes(p.dtype))
    return SEEDQ_ERR_INVALID_ARG;
  // CTAs that begin late read the scores again, and segments' logits.
  const Wide rows_in = (Wide)p.n_groups * p.n_beams, results = (Wide)p.n_groups * p.n_out * 4;
  const ByteRows out[] = {byte_rows(p.out_score, results), byte_rows(p.out_beam, results), byte_rows(p.out_token, results)};
  const ByteRows x = byte_rows(p.logits, (Wide)p.vocab * dtype_bytes(p.dtype), rows_in, (Wide)p.row_stride * dtype_bytes(p.dtype));
  if (overlap(out[0], out[1]) || overlap(out[0], out[2]) || overlap(out[1], out[2])) return SEEDQ_ERR_INVALID_ARG;
  for (const ByteRows &o : out)
    if (overlap(o, x) || overlap(o, byte_rows(p.scores, rows_in * 4)) || (p.weights && overlap(o, byte_rows(p.weights, rows_in * 4))) ||
        (p.done && overlap(o, byte_rows(p.done, rows_in))))
      return SEEDQ_ERR_INVALID_ARG;
  SelectArgs a{};
  a.x = p.logits, a.stride = p.row_stride, a.vocab = (int32_t)p.vocab, a.beams = p.n_beams, a.groups = (int32_t)p.n_groups;
  a.scale = p.scale, a.c = p.scale * kLog2e, a.scores = p.scores, a.weights = p.weights, a.done = p.done, a.end_token = p.end_token;
  a.n_out = p.n_out, a.out_score = p.out_score, a.out_beam = p.out_beam, a.out_token = p.out_token;
  a.segments = (int32_t)segments_of(p.vocab);
  const int64_t rows = p.n_groups * p.n_beams;
  a.counters = (int *)p.workspace;
  a.parts = (float2 *)((char *)p.workspace + kHeader);
  const bool vec = (uintptr_t)p.logits % 16 == 0 && (rows == 1 || p.row_stride * dtype_bytes(p.dtype) % 16 == 0);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const cudaError_t e = p.dtype == SEEDQ_F32    ? launch<SEEDQ_F32>(a, vec, st)
                        : p.dtype == SEEDQ_BF16 ? launch<SEEDQ_BF16>(a, vec, st)
                                                : launch<SEEDQ_F16>(a, vec, st);
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
