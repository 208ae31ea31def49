// Beam search's choice over beams and vocabulary (seedq_beam_select).
//
// Mathematics.  With m the largest of a live beam's logits x, candidate (b, v) has
// the total score_b - ln sum exp(scale (x - m)) + scale (x_v - m), and a request's
// first n candidates by weight_b * total are wanted.  Within a beam the order is that of
// the logits themselves; between beams it is that of doubles made from the logit,
// the score and the log sum, so candidates that lie close together are not swapped by
// a float32 sum.
//
// One pass over the logits keeps the sums and, per segment of 256 logits, the
// largest.  The first n candidates lie in the n segments whose largest logits come
// first in the same order: each of those n alone brings a candidate that precedes
// all of the others.  So the last CTA to arrive for a request chooses n segments
// from the maxima, reads them again, and chooses from their logits.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <cmath>

#include "f32x2.cuh"
#include "order.cuh"
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
constexpr uint64_t kHeader = SEEDQ_MAX_REQUESTS * 4;  // arrival counters

struct SelectArgs {
  const void *x;
  int64_t stride;
  int32_t vocab, beams, groups, segments, chunks;  // segments, chunks: of a row
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
// A candidate as two words that sort as candidates do: the weighted total as an
// ordered double; then beam, logit and token, each such that what comes first is
// larger.  No candidate is (0, 0).
struct Item {
  uint64_t key, rest;
  __device__ __forceinline__ bool before(const Item &o) const { return key > o.key || (key == o.key && rest > o.rest); }
};
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

__device__ __forceinline__ Item shuffled(const Item &x, int from) { return {__shfl_sync(~0u, x.key, from), __shfl_sync(~0u, x.rest, from)}; }
// The first 32 of two lists in order, as merge_lists.
__device__ __noinline__ Item merge_items(Item a, Item b, int lane) {
  b = shuffled(b, 31 - lane);
  Item x = a.before(b) ? a : b;
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    const Item y = shuffled(x, lane ^ o);
    if (y.before(x) == ((lane & o) == 0)) x = y;
  }
  return x;
}

struct Join {
  // total = base + scale * (logit - most): the difference first, or a large common part would take the sum's digits
  double base[kMaxBeams], weight[kMaxBeams], most[kMaxBeams];
  int kind[kMaxBeams];
  uint32_t reach[kMaxBeams];  // the row's n-th largest segment maximum, as a word: no smaller logit is chosen
  Item list[kWarps][32];
  Item chosen[32];
  uint64_t keys[kWarps][kSegment];
  int spoiled;
};

__device__ __forceinline__ double total_of(const SelectArgs &a, const Join &s, int b, float x) {
  return s.kind[b] == kDone ? s.base[b] : s.base[b] + (double)a.scale * ((double)x - s.most[b]);
}
__device__ __forceinline__ Item item_of(const SelectArgs &a, const Join &s, int b, uint64_t key) {  // of an order_key
  if (!key) return {0, 0};
  return {order_double(s.weight[b] * total_of(a, s, b, key_value(key))), rest_word(b, (uint32_t)(key >> 32), key_index(key))};
}
// The CTA's lists, one per warp, as one; in warp 0.
__device__ __forceinline__ Item join_lists(Join &s, Item mine, int w, int lane) {
  s.list[w][lane] = mine;
#pragma unroll
  for (int n = kWarps / 2; n; n >>= 1) {
    __syncthreads();
    if (w < n) {
      mine = merge_items(mine, s.list[w + n][lane], lane);
      s.list[w][lane] = mine;
    }
  }
  return mine;
}

template <int DT, bool VEC>
__device__ __forceinline__ void join_group(const SelectArgs &a, Join &s, int64_t g) {
  using Seg = Segment<DT, VEC>;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (threadIdx.x == 0) s.spoiled = 0;
  __syncthreads();
  // the sums of the beams
  Item best = {0, 0};
  for (int b = w; b < a.beams; b += kWarps) {
    const int64_t row = g * a.beams + b;
    const float score = a.scores[row];
    const float weight = a.weights ? a.weights[row] : 1.f;
    int kind = row_kind(a, row);
    double base = (double)score, most_logit = 0.0;
    bool bad = isnan(score) || (kind != kNone && !(score < CUDART_INF_F && weight > 0.f && weight < CUDART_INF_F));
    if (kind == kLive) {
      float m = -CUDART_INF_F, sum = 0.f;
      for (int i = lane; i < a.chunks; i += 32) {
        const float2 *p = a.parts + row * a.chunks + i;
        const float pm = fresh_load(&p->x), ps = fresh_load(&p->y);
        const float to = max_nan(m, pm);
        if (to != -CUDART_INF_F) sum = sum * exp2_fast((m - to) * a.c) + ps * exp2_fast((pm - to) * a.c);
        m = to;
      }
      float to = m;
#pragma unroll
      for (int o = 16; o; o >>= 1) to = max_nan(to, __shfl_xor_sync(~0u, to, o));
      if (to != -CUDART_INF_F) sum *= exp2_fast((m - to) * a.c);
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
      if (to == -CUDART_INF_F) {
        kind = kNone;  // no token is allowed
      } else if (!(sum < CUDART_INF_F)) {
        bad = true;
      } else {
        // ln sum = e ln 2 + ln f, f within 0.7 and 1.42: float32 errors of the small logarithm alone
        const int e = (int)(__float_as_uint(sum * 1.41421356f) >> 23) - 127;
        const float f = sum * __uint_as_float((uint32_t)(127 - e) << 23);
        base -= (double)e * 0.69314718055994531 + (double)logf(f);
        most_logit = (double)to;
      }
    }
    if (lane == 0) {
      s.base[b] = base, s.weight[b] = (double)weight, s.most[b] = most_logit, s.kind[b] = kind;
      if (bad) s.spoiled = 1;
    }
    __syncwarp();
    // the beam's first segments
    uint64_t key = 0;
    if (kind == kLive && !bad) {
      const float *most = a.most + row * a.segments;
      uint64_t last = 0;
      for (int s0 = 0; s0 < a.segments; s0 += 32) {
        const int i = s0 + lane;
        const float x = i < a.segments ? fresh_load(most + i) : -CUDART_INF_F;
        const uint64_t k = x > -CUDART_INF_F ? order_key(x, i) : 0;
        if (!__any_sync(~0u, k > last)) continue;
        key = merge_lists(key, sort_keys(k, lane), lane);
        last = __shfl_sync(~0u, key, a.n_out - 1);
      }
      if (lane == 0) s.reach[b] = (uint32_t)(last >> 32);
    } else if (kind == kDone && !bad && lane == 0) {
      key = order_key(0.f, a.end_token);
    }
    best = merge_items(best, item_of(a, s, b, key), lane);
  }
  best = join_lists(s, best, w, lane);
  if (w == 0) s.chosen[lane] = lane < a.n_out ? best : Item{0, 0};
  __syncthreads();

  // the chosen segments' logits
  best = {0, 0};
  if (!s.spoiled) {
    for (int i = w; i < a.n_out; i += kWarps) {
      const Item at = s.chosen[i];
      if (!at.key) break;  // the same in all lanes
      const int b = rest_beam(at.rest);
      if (s.kind[b] == kDone) {
        best = merge_items(best, lane == 0 ? at : Item{0, 0}, lane);
        continue;
      }
      const int64_t row = g * a.beams + b;
      const char *base = (const char *)a.x + row * a.stride * Seg::kSize;
      const int first = rest_index(at.rest) * kSegment;
      Seg seg;
      seg.load(base, first, a.vocab, lane);
      float x[8];
      seg.get(x);
      const uint32_t reach = s.reach[b];
      int n = 0;
      __syncwarp();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint64_t k = order_key(x[e], first + Seg::place(e, lane));
        const bool in = x[e] > -CUDART_INF_F && (uint32_t)(k >> 32) >= reach;
        const uint32_t all = __ballot_sync(~0u, in);
        if (in) s.keys[w][n + __popc(all & ((1u << lane) - 1))] = k;
        n += __popc(all);
      }
      __syncwarp();
      uint64_t key = 0;
      for (int o = 0; o < n; o += 32) key = merge_lists(key, sort_keys(o + lane < n ? s.keys[w][o + lane] : 0, lane), lane);
      best = merge_items(best, item_of(a, s, b, key), lane);
    }
  }
  best = join_lists(s, best, w, lane);
  if (w == 0 && lane < a.n_out) {
    const int64_t o = g * a.n_out + lane;
    const bool there = best.key && !s.spoiled;
    const int b = rest_beam(best.rest);
    a.out_score[o] = s.spoiled ? CUDART_NAN_F : there ? (float)total_of(a, s, b, rest_logit(best.rest)) : -CUDART_INF_F;
    a.out_beam[o] = there ? b : -1;
    a.out_token[o] = there ? rest_index(best.rest) : -1;
  }
}

template <int DT, bool VEC>
__global__ void __launch_bounds__(kThreads) k_beam_select(const __grid_constant__ SelectArgs a) {
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
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      float x[8];
      seg[j].get(x);
      float mx = max_nan(x[0], x[1]);
#pragma unroll
      for (int e = 2; e < 8; e += 2) mx = max_nan(mx, x[e], x[e + 1]);
      const uint32_t most = __reduce_max_sync(~0u, order_word(mx));
      word = max(word, most);
      if (lane == 0 && s0 + j * kWarps < a.segments) a.most[row * a.segments + s0 + j * kWarps] = key_value((uint64_t)most << 32);
    }
    const float m = key_value((uint64_t)word << 32);
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

int chunk_segments(int32_t dtype) { return dtype == SEEDQ_F32 ? 4 * kWarps : 8 * kWarps; }
int64_t segments_of(int64_t vocab) { return (vocab + kSegment - 1) / kSegment; }

template <int DT>
void launch(const SelectArgs &a, bool vec, unsigned ctas, cudaStream_t st) {
  if (vec) k_beam_select<DT, true><<<ctas, kThreads, 0, st>>>(a);
  else k_beam_select<DT, false><<<ctas, kThreads, 0, st>>>(a);
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
  const uint64_t chunks = (segments + chunk_segments(SEEDQ_F32) - 1) / chunk_segments(SEEDQ_F32);
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
  SelectArgs a{};
  a.x = p.logits, a.stride = p.row_stride, a.vocab = (int32_t)p.vocab, a.beams = p.n_beams, a.groups = (int32_t)p.n_groups;
  a.scale = p.scale, a.c = p.scale * kLog2e, a.scores = p.scores, a.weights = p.weights, a.done = p.done, a.end_token = p.end_token;
  a.n_out = p.n_out, a.out_score = p.out_score, a.out_beam = p.out_beam, a.out_token = p.out_token;
  a.segments = (int32_t)segments_of(p.vocab);
  a.chunks = (a.segments + chunk_segments(p.dtype) - 1) / chunk_segments(p.dtype);
  const int64_t rows = p.n_groups * p.n_beams;
  a.counters = (int *)p.workspace;
  a.parts = (float2 *)((char *)p.workspace + kHeader);
  a.most = (float *)(a.parts + rows * a.chunks);
  const unsigned ctas = (unsigned)(rows * a.chunks);  // at most 2^13 * 2^14
  const bool vec = (uintptr_t)p.logits % 16 == 0 && (rows == 1 || p.row_stride * dtype_bytes(p.dtype) % 16 == 0);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  switch (p.dtype) {
    case SEEDQ_F32: launch<SEEDQ_F32>(a, vec, ctas, st); break;
    case SEEDQ_BF16: launch<SEEDQ_BF16>(a, vec, ctas, st); break;
    default: launch<SEEDQ_F16>(a, vec, ctas, st);
  }
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}

}  // extern "C"
