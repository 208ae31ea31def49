// The cache write with the keys rotated on the way (seedq_kv_append_rotary).
//
// Mathematics: a page's scale is the smallest power of two that brings the rotated
// keys within the codes' range, so every key is rotated before the first code is
// written.  Between the two a lane keeps the rotated numbers in registers, two tokens
// of 16 numbers each: two pieces of 8 that hold whole pairs, with SEEDQ_ROPE_HALF
// piece i of the first half of the rotated dims and piece i of the second, else of the
// head's halves.
//
// A CTA owns `share` heads of the keys or of the values, for the stretches of tokens on
// one page that begin among 2^group_shift tokens.  Its 8 warps form teams, the
// smallest that can keep the longest run of consecutive slots, and the tasks (a
// stretch, a head) are dealt to the teams in equal ranges.  A team has the next two
// heads' numbers under way by asynchronous copies, and the cos and sin of its lanes'
// tokens in registers for all heads.  Runs longer than 8 warps keep are read again.
// The step's queries are turned by CTAs behind those of the append, many by a launch
// of their own: the registers and shared memory of the append leave their CTAs too few
// of an SM's threads.
//
// Measured, 128 head dims: 16 single tokens of 8 key-value and 32 query heads, float32,
// 3.9 us (the plain append 3.0, a rotation 2.4); 4 prompts of 1024, 32 heads, bfloat16,
// 27.5 us without queries (3.7 TB/s; the plain append 23), 43 with them (3.9 TB/s).
// What bounds the prompts is the chain of a head (numbers, largest, the warps' largest,
// codes) and about 200 instructions per 16 numbers of a lane at 16 warps per SM, 43%
// of the issue slots of an active SM, and CTAs that begin apart: 3.4 to a place, 54
// thousand cycles on average of the longest SM's 59.  4 heads to a CTA instead of 8
// level that, and read cos and sin twice as often, 33 us; 16, 37.  24 warps want 80
// registers, and spill (61 us); cos and sin in registers instead of shared memory, 36
// us; as loads of every head, 50; the numbers kept as they came and rotated twice, 45.
#include <cuda_runtime.h>
#include <stdint.h>

#include "cp_async.cuh"
#include "device_once.h"
#include "f32x2.cuh"
#include "kv_codes.cuh"
#include "order.cuh"
#include "rotary.cuh"
#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kCtasPerSm = 2;
constexpr int kSteps = 2;   // tokens that a lane keeps
constexpr int kStages = 2;  // tasks whose numbers are under way
// Tokens times heads and tensors up to which a CTA takes one head of 8 tokens: a prompt
// of 512 tokens of 8 heads (8192) takes 10.8 us so, 15.5 with 8 heads to a CTA, 256
// single tokens of 32 heads (16384) 23.5 and 17.1.
constexpr int64_t kFewPairs = 8192;
constexpr int64_t kQueriesApart = 152 * 2048;  // threads from which on the queries have a launch of their own

struct AppendArgs {
  seedq_kv_cache c;
  const void *x[2];     // the tokens' keys and values
  int64_t ts, hs, n;    // their strides (elements) and number
  const int64_t *slots;
  const float2 *cs;
  int32_t half, layout;
  bool vec;             // rows of x allow accesses of 16 bytes
  bool wide_cs;         // pairs of cos and sin two at a time
  int32_t group_shift, page_shift;
  int32_t share;           // heads of a CTA
  unsigned ctas, ctas_of_group;  // of the append, and of a group of tokens and a tensor
  RotateArgs q;
  RotateSplit split;
};

__device__ __forceinline__ int64_t page_of(const AppendArgs &a, int64_t slot) {  // -1 for a negative slot
  if (slot < 0) return -1;
  return a.page_shift >= 0 ? slot >> a.page_shift : slot / a.c.page_size;
}

// 16 numbers of a token, in two pieces, as they lie in memory and as numbers.
template <int DT>
struct Unit {
  static constexpr int kSize = DT == SEEDQ_F32 ? 4 : 2, kLoads = kSize;  // of 16 bytes
  uint4 w[kLoads];
  __device__ __forceinline__ void get(float (&x)[16]) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint32_t v[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (DT == SEEDQ_F32) {
          x[(4 * i + k) % 16] = __uint_as_float(v[k]);
        } else if (DT == SEEDQ_BF16) {
          x[(8 * i + 2 * k) % 16] = __uint_as_float(v[k] << 16);
          x[(8 * i + 2 * k + 1) % 16] = __uint_as_float(v[k] & 0xffff0000u);
        } else {
          const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v[k]));
          x[(8 * i + 2 * k) % 16] = f.x, x[(8 * i + 2 * k + 1) % 16] = f.y;
        }
      }
    }
  }
};

// How pairs lie in a lane's two pieces: number k of the first with number k of the
// second, neighbours, or (SEEDQ_ROPE_HALF whose halves are no multiple of 8) across
// pieces of any lanes.
enum { kAcross = 0, kBeside = 1, kOdd = 2 };

// What a lane does to every token: its pieces begin at dims d0 and d1 (lanes of a token
// read each of them side by side), and hold n0 pairs from p0 on and n1 from p1 on, up
// to 4 each.
struct Lane {
  int d0, d1, p0, p1, n0, n1;
};

template <int PAIRS>
__device__ __forceinline__ Lane lane_of(const AppendArgs &a, int u) {
  const int D = a.c.head_dim;
  if (PAIRS == kOdd) return {8 * u, D / 2 + 8 * u, 0, 0, 0, 0};
  if (PAIRS == kBeside) {
    const int p0 = 4 * u, p1 = D / 4 + 4 * u;
    return {8 * u, D / 2 + 8 * u, p0, p1, min(max(a.half - p0, 0), 4), min(max(a.half - p1, 0), 4)};
  }
  const int turns = a.half / 8;
  if (u < turns) return {8 * u, a.half + 8 * u, 8 * u, 8 * u + 4, 4, 4};
  const int d = 2 * a.half + 8 * (u - turns);
  return {d, d + (D - 2 * a.half) / 2, 0, 0, 0, 0};
}

// cos and sin of the lane's pairs of token t; what it has none of is not used.
__device__ __forceinline__ void load_angles(const AppendArgs &a, const Lane &l, int64_t t, float2 (&c)[8]) {
  const float2 *cs = a.cs + t * a.half;
  if (a.wide_cs && l.n0 == 4 && l.n1 == 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 v = __ldg((const float4 *)(cs + (k < 2 ? l.p0 : l.p1)) + k % 2);
      c[2 * k] = make_float2(v.x, v.y), c[2 * k + 1] = make_float2(v.z, v.w);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) c[k] = k % 4 < (k < 4 ? l.n0 : l.n1) ? __ldg(cs + (k < 4 ? l.p0 : l.p1) + k % 4) : make_float2(1.f, 0.f);
  }
}

// A key's numbers turned; x, t: its first element and its token (for kOdd alone).
template <int DT, int PAIRS>
__device__ __forceinline__ void turn(const AppendArgs &a, const Lane &l, const float2 (&c)[8], float (&y)[16], const char *x, int64_t t) {
  if (PAIRS == kOdd) {
    const float2 *cs = a.cs + t * a.half;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int i = k < 8 ? l.d0 + k : l.d1 + k - 8;
      if (i < 2 * a.half) {
        const bool second = i >= a.half;
        const float o = load_elem(x, DT, i + (second ? -a.half : a.half));
        const float2 z = second ? turned(o, y[k], cs[i - a.half]) : turned(y[k], o, cs[i]);
        y[k] = second ? z.y : z.x;
      }
    }
  } else if (PAIRS == kAcross ? l.n0 > 0 : l.n0 + l.n1 == 8) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int i = PAIRS == kBeside ? 2 * k : k, j = PAIRS == kBeside ? 2 * k + 1 : 8 + k;
      const float2 z = turned(y[i], y[j], c[k]);
      y[i] = z.x, y[j] = z.y;
    }
  } else if (PAIRS == kBeside && l.n0 > 0) {  // pairs at the end of the rotated dims
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 z = turned(y[2 * k], y[2 * k + 1], c[k]);
      if (k % 4 < (k < 4 ? l.n0 : l.n1)) y[2 * k] = z.x, y[2 * k + 1] = z.y;
    }
  }
}

// Four codes of numbers times a power of two, none past the largest code: as
// four_codes, whose product is exact.
template <int KIND>
__device__ __forceinline__ uint32_t four_scaled(const float *x, uint64_t by2) {
  if (KIND == SEEDQ_KV_INT8) {
    const uint64_t one = f2_pack(12582912.f, 12582912.f);
    const float2 a = f2_unpack(f2_fma(f2_pack(x[0], x[1]), by2, one)), b = f2_unpack(f2_fma(f2_pack(x[2], x[3]), by2, one));
    return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                       __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
  }
  return four_codes<KIND>(f2_pack(x[0], x[1]), f2_pack(x[2], x[3]), by2);
}

template <int DT>
constexpr int ring_bytes() { return ((kStages * kSteps + 1) * Unit<DT>::kLoads + kSteps * 4) * kThreads * 16; }

// 16 numbers that lie at any address, to where a team's copies go.
template <int DT>
__device__ __noinline__ void copy_slowly(uint4 *to, int to_step, const char *x, int second) {
  using U = Unit<DT>;
#pragma unroll 1
  for (int i = 0; i < U::kLoads; ++i) {
    const char *from = x + (i < U::kLoads / 2 ? 0 : second) + i % (U::kLoads / 2) * 16;
    uint32_t y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      y[k] = DT == SEEDQ_F32 ? ((const uint32_t *)from)[k] : (uint32_t)((const uint16_t *)from)[2 * k] | (uint32_t)((const uint16_t *)from)[2 * k + 1] << 16;
    to[i * to_step] = make_uint4(y[0], y[1], y[2], y[3]);
  }
}

// A run of consecutive slots on a page.
struct Run {
  int64_t page, t0;  // its page and first token
  int off, m;        // its first place on the page, and its length
};
// What a team does to it: heads h0 .. h1 - 1 of the tensor.
struct Team {
  int warps, id, lead;  // of the CTA's 8; lead: the team's first warp
  int first, stride;    // the lane's tokens
  bool idle;            // the lane is left over
  int h0, h1;
};

__device__ __forceinline__ void team_barrier(const Team &t) {
  if (t.warps == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(t.id + 1), "r"(t.warps * 32) : "memory");
}

// Writes a run; the lane keeps STEPS of its tokens.
template <int KIND, int DT, int PAIRS, int TENSOR, int STEPS>
__device__ __forceinline__ void write_run(const AppendArgs &a, const Lane &l, const Team &team, const Run &run, float (*s_max)[kWarps], int &parity) {
  using U = Unit<DT>;
  constexpr int kHalf = U::kLoads / 2, kStageSize = kSteps * U::kLoads * kThreads;
  extern __shared__ __align__(128) uint4 s_ring[];  // [stage][step and load][thread]
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  uint4 *ring = s_ring + threadIdx.x;
  const int second_x = (l.d1 - l.d0) * U::kSize, second_c = l.d1 - l.d0;
  // The lane's kept tokens; where the run has fewer, its last once more: the same numbers to the same place.
  int64_t x_kept[STEPS], c_kept[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int t = min(team.first + k * team.stride, run.m - 1);
    x_kept[k] = (t * a.ts + l.d0) * U::kSize;
    c_kept[k] = t * a.c.token_stride + l.d0;
  }
  const int64_t x_head = a.hs * U::kSize;
  const char *x = (const char *)a.x[TENSOR] + (run.t0 * a.ts + team.h0 * a.hs) * U::kSize;
  uint8_t *code = (uint8_t *)(TENSOR ? a.c.v : a.c.k) + run.page * a.c.page_stride + team.h0 * a.c.head_stride + run.off * a.c.token_stride;
  float *scale = (TENSOR ? a.c.v_scale : a.c.k_scale) + run.page * a.c.n_kv_heads + team.h0;
  auto issue = [&](int h, const char *x_ahead) {  // the numbers of head h under way
    if (h < team.h1) {
      uint4 *to = ring + (h % kStages) * kStageSize;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        const char *from = x_ahead + x_kept[k];
        if (a.vec) {
#pragma unroll
          for (int i = 0; i < U::kLoads; ++i)
            cp_async16(to + (k * U::kLoads + i) * kThreads, from + (i < kHalf ? 0 : second_x) + (i % kHalf) * 16);
        } else {
          copy_slowly<DT>(to + k * U::kLoads * kThreads, kThreads, from, second_x);
        }
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int k = 0; k < kStages; ++k) issue(team.h0 + k, x + k * x_head);
  float4 *angles = (float4 *)(ring + (kStages * kSteps + 1) * U::kLoads * kThreads);  // [step and two pairs][thread]
  if (TENSOR == 0 && PAIRS != kOdd) {
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      float2 c[8];
      load_angles(a, l, run.t0 + min(team.first + k * team.stride, run.m - 1), c);
#pragma unroll
      for (int i = 0; i < 4; ++i) angles[(k * 4 + i) * kThreads] = make_float4(c[2 * i].x, c[2 * i].y, c[2 * i + 1].x, c[2 * i + 1].y);
    }
  }
#pragma unroll 1
  for (int h = team.h0; h < team.h1; ++h, x += x_head, code += a.c.head_stride, ++scale) {
    const float was = run.off > 0 ? *(volatile float *)scale : 0.f;  // another run of the page may have written it
    float high = 0.f, low = 0.f;  // a NaN stays
    auto largest = [&](const float (&y)[16]) {
#pragma unroll
      for (int k = 0; k < 16; k += 2) high = max_nan(high, y[k], y[k + 1]), low = min_nan(low, y[k], y[k + 1]);
    };
    float held[STEPS][16];
    cp_async_wait<kStages - 1>();
    const uint4 *from = ring + (h % kStages) * kStageSize;
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      U e;
#pragma unroll
      for (int i = 0; i < U::kLoads; ++i) e.w[i] = from[(k * U::kLoads + i) * kThreads];
      e.get(held[k]);
    }
    issue(h + kStages, x + kStages * x_head);  // into the stage just read
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
      float2 c[8];
      if (TENSOR == 0 && PAIRS != kOdd) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 v = angles[(k * 4 + i) * kThreads];
          c[2 * i] = make_float2(v.x, v.y), c[2 * i + 1] = make_float2(v.z, v.w);
        }
      }
      if (TENSOR == 0)
        turn<DT, PAIRS>(a, l, c, held[k], x + x_kept[k] - l.d0 * U::kSize, run.t0 + min(team.first + k * team.stride, run.m - 1));
      largest(held[k]);
    }
    const int mine = team.idle ? 0 : run.m;
    auto far = [&](int t, float (&y)[16]) {  // of the tokens that are not kept
      const char *from = x + ((int64_t)t * a.ts + l.d0) * U::kSize;
      U e;
      if (a.vec) {
#pragma unroll
        for (int k = 0; k < U::kLoads; ++k) e.w[k] = __ldg((const uint4 *)(from + (k < kHalf ? 0 : second_x)) + k % kHalf);
      } else {
        uint4 *to = ring + kStages * kStageSize;  // a place of the lane's own behind the stages
        copy_slowly<DT>(to, kThreads, from, second_x);
#pragma unroll
        for (int k = 0; k < U::kLoads; ++k) e.w[k] = to[k * kThreads];
      }
      e.get(y);
      if (TENSOR == 0) {
        float2 c[8];
        if (PAIRS != kOdd) load_angles(a, l, run.t0 + t, c);
        turn<DT, PAIRS>(a, l, c, y, x + (int64_t)t * a.ts * U::kSize, run.t0 + t);
      }
    };
#pragma unroll 1
    for (int t = team.first + STEPS * team.stride; t < mine; t += team.stride) {
      float y[16];
      far(t, y);
      largest(y);
    }
    uint32_t bits = __reduce_max_sync(~0u, __float_as_uint(max_nan(high, -low)) & 0x7fffffffu);  // a NaN above all
    if (team.warps > 1) {  // by turns: a warp that is one head ahead writes the other maxima
      if (lane == 0) s_max[parity][w] = __uint_as_float(bits);
      team_barrier(team);
      bits = __reduce_max_sync(~0u, __float_as_uint(s_max[parity][team.lead + lane % team.warps]));
      parity ^= 1;
    }
    const float want = block_scale<KIND>(bits);
    float now = want;
    if (run.off > 0) {
      if (!(want > was) && !isnan(want)) now = was;  // a NaN scale stays
      if (now > was) {
        const float r = __fdiv_rn(was, now);
        const uint64_t r2 = f2_pack(r, r);
#pragma unroll 1
        for (int t = team.first - run.off; t < (team.idle ? -run.off : 0); t += team.stride) {
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            uint2 *c = (uint2 *)(code + t * a.c.token_stride + (part ? l.d1 : l.d0));
            const uint2 v = *c;
            uint64_t x0, x1, x2, x3;
            four_values<KIND>(v.x, x0, x1);
            four_values<KIND>(v.y, x2, x3);
            *c = make_uint2(four_codes<KIND>(x0, x1, r2), four_codes<KIND>(x2, x3, r2));
          }
        }
      }
    }
    // x / now; by the reciprocal where that is exact: a power of two whose reciprocal is a normal number
    const uint32_t nb = __float_as_uint(now);
    const bool exact = (nb & 0x7fffffu) == 0 && nb < 0x7f000000u && nb != 0;
    const float inv = exact ? __uint_as_float(0x7f000000u - nb) : 0.f;
    const uint64_t inv2 = f2_pack(inv, inv);
    auto write = [&](const float (&y)[16], uint8_t *to) {
      uint2 c[2] = {make_uint2(0, 0), make_uint2(0, 0)};
      if (exact) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
          c[part] = make_uint2(four_scaled<KIND>(y + 8 * part, inv2), four_scaled<KIND>(y + 8 * part + 4, inv2));
      } else if (now > 0.f) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            c[part].x |= value_code<KIND>(__fdiv_rn(y[8 * part + k], now)) << 8 * k;
            c[part].y |= value_code<KIND>(__fdiv_rn(y[8 * part + 4 + k], now)) << 8 * k;
          }
      }
      *(uint2 *)to = c[0];
      *(uint2 *)(to + second_c) = c[1];
    };
#pragma unroll
    for (int k = 0; k < STEPS; ++k) write(held[k], code + c_kept[k]);
#pragma unroll 1
    for (int t = team.first + STEPS * team.stride; t < mine; t += team.stride) {
      float y[16];
      far(t, y);
      write(y, code + t * a.c.token_stride + l.d0);
    }
    if (lane == 0 && w == team.lead) *scale = now;
  }
  cp_async_wait<0>();
}

template <int KIND, int DT, int PAIRS, int TENSOR>
__device__ __forceinline__ void append(const AppendArgs &a, int64_t group, int h0) {
  __shared__ float s_max[2][kWarps];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int P = a.c.page_size, per = a.c.head_dim / 16;  // lanes of a token
  const int heads = min(a.share, a.c.n_kv_heads - h0);
  const int64_t g0 = group << a.group_shift;

  // A lane per token: stretches begin where the page differs from the token's before,
  // runs end where a slot does not follow.
  uint32_t starts;
  int64_t my_slot = -1;
  int my_run;
  {
    const int64_t t = g0 + lane;
    if (t < a.n) my_slot = a.slots[t];
    int64_t before = __shfl_up_sync(~0u, my_slot, 1);
    if (lane == 0) before = g0 > 0 ? a.slots[g0 - 1] : -1;
    const int64_t page = page_of(a, my_slot), page_before = page_of(a, before);
    starts = __ballot_sync(~0u, lane < (1 << a.group_shift) && page >= 0 && page < a.c.n_pages && page != page_before);
    const uint32_t breaks = __ballot_sync(~0u, my_slot != before + 1 || page != page_before) >> lane >> 1;
    my_run = breaks ? __ffs(breaks) : 32 - lane;
  }
  if (starts == 0) return;
  // The length of the run of tokens from t0 on, m of them known.
  auto run_length = [&](int64_t t0, int64_t slot, int m) {
    const int most = (int)min((int64_t)(P - (int)(slot - page_of(a, slot) * P)), a.n - t0);
    while (m < most) {
      const bool follows = m + lane < most && a.slots[t0 + m + lane] == slot + m + lane;
      const uint32_t stop = __ballot_sync(~0u, !follows);
      m += stop ? __ffs(stop) - 1 : 32;
      if (stop) break;
    }
    return m;
  };
  {
    const int last = 31 - __clz(starts);
    const int m = __shfl_sync(~0u, my_run, last);
    const int64_t slot = __shfl_sync(~0u, my_slot, last);
    if (last + m == 32) {  // it may go on behind the tokens looked at
      const int all = run_length(g0 + last, slot, m);
      if (lane == last) my_run = all;
    }
  }
  const int longest = __reduce_max_sync(~0u, (starts >> lane & 1) ? my_run : 0);

  const int step = 32 / per, t_first = lane / per;  // tokens of a warp's step; the lane's
  const Lane l = lane_of<PAIRS>(a, lane - t_first * per);
  Team team;
  team.warps = 1;
  while (team.warps < kWarps && team.warps * kSteps * step < longest) team.warps *= 2;
  const int teams = kWarps / team.warps;
  team.id = w / team.warps;
  team.lead = team.id * team.warps;
  team.first = (w - team.lead) * step + t_first;
  team.stride = team.warps * step;
  team.idle = t_first >= step;

  // Tasks are a stretch and a head; the team's are stretch after stretch, each for a range of heads.
  const int tasks = __popc(starts) * heads;
  int q = tasks * team.id / teams, parity = 0;
  const int q_end = tasks * (team.id + 1) / teams;
  uint32_t rest = starts;
  int first = q;
  for (; first >= heads; first -= heads) rest &= rest - 1;
  for (; q < q_end; q += heads - first, first = 0, rest &= rest - 1) {
    team.h0 = h0 + first;
    team.h1 = h0 + min(heads, first + q_end - q);
    const int s = __ffs(rest) - 1;
    int64_t slot = __shfl_sync(~0u, my_slot, s);
    Run run{page_of(a, slot), g0 + s, 0, __shfl_sync(~0u, my_run, s)};
    for (;;) {
      run.off = (int)(slot - run.page * P);
      if (run.m <= team.stride) write_run<KIND, DT, PAIRS, TENSOR, 1>(a, l, team, run, s_max, parity);
      else write_run<KIND, DT, PAIRS, TENSOR, kSteps>(a, l, team, run, s_max, parity);
      run.t0 += run.m;
      if (run.t0 >= a.n) break;
      slot = run.t0 - g0 < 32 ? __shfl_sync(~0u, my_slot, (int)(run.t0 - g0)) : a.slots[run.t0];
      if (page_of(a, slot) != run.page) break;
      run.m = run_length(run.t0, slot, 1);
      team_barrier(team);  // the scales are written
    }
  }
}

template <int DT, int N>
__device__ __forceinline__ void rotate_query(const AppendArgs &a, int64_t i) {
  switch (a.q.out_dtype) {
    case SEEDQ_F32: rotate_item<DT, SEEDQ_F32, N>(a.q, a.split, i); break;
    case SEEDQ_BF16: rotate_item<DT, SEEDQ_BF16, N>(a.q, a.split, i); break;
    default: rotate_item<DT, SEEDQ_F16, N>(a.q, a.split, i);
  }
}

template <int KIND, int DT, int PAIRS>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) k_kv_append_rotary(const __grid_constant__ AppendArgs a) {
  if (blockIdx.x < a.ctas) {
    // the keys first: they take longer
    const bool tensor = blockIdx.x >= a.ctas / 2;
    const unsigned i = tensor ? blockIdx.x - a.ctas / 2 : blockIdx.x;
    const int64_t group = i / a.ctas_of_group;
    const int h0 = (int)(i - (unsigned)group * a.ctas_of_group) * a.share;
    if (tensor) append<KIND, DT, PAIRS, 1>(a, group, h0);
    else append<KIND, DT, PAIRS, 0>(a, group, h0);
  } else {
    const int64_t i = (int64_t)(blockIdx.x - a.ctas) * blockDim.x + threadIdx.x;
    if (a.split.wide == 8) rotate_query<DT, 8>(a, i);
    else if (a.split.wide == 4) rotate_query<DT, 4>(a, i);
    else rotate_query<DT, 1>(a, i);
  }
}

DeviceOnce g_once[2][3][3];

template <int KIND, int DT, int PAIRS>
cudaError_t launch_as(const AppendArgs &a, unsigned ctas, cudaStream_t st) {
  if (ring_bytes<DT>() > 40 * 1024) {  // of 48 without being asked for, the static part among them
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const int rc = g_once[KIND][DT][PAIRS].run(dev, [] {
      return (int)cudaFuncSetAttribute(k_kv_append_rotary<KIND, DT, PAIRS>, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes<DT>());
    });
    if (rc) return (cudaError_t)rc;
  }
  k_kv_append_rotary<KIND, DT, PAIRS><<<ctas, kThreads, ring_bytes<DT>(), st>>>(a);
  return cudaGetLastError();
}
template <int KIND, int DT>
cudaError_t launch(const AppendArgs &a, unsigned ctas, cudaStream_t st) {
  if (a.layout == SEEDQ_ROPE_PAIRS) return launch_as<KIND, DT, kBeside>(a, ctas, st);
  return a.half % 8 ? launch_as<KIND, DT, kOdd>(a, ctas, st) : launch_as<KIND, DT, kAcross>(a, ctas, st);
}
using Launch = cudaError_t (*)(const AppendArgs &, unsigned, cudaStream_t);
constexpr Launch kLaunch[2][3] = {{launch<0, 0>, launch<0, 1>, launch<0, 2>}, {launch<1, 0>, launch<1, 1>, launch<1, 2>}};

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" seedq_status seedq_kv_append_rotary(const seedq_kv_cache *cache, const void *k, const void *v, int32_t dtype,
                                               int64_t token_stride, int64_t head_stride, const int64_t *slots, int64_t n_tokens,
                                               const seedq_append_rotary_args *args, void *cuda_stream) {
  const seedq_status st = kv_check(cache);
  if (st != SEEDQ_OK) return st;
  if (!dtype_ok(dtype) || n_tokens < 0 || n_tokens > INT32_MAX || !args || !rope_ok(args->layout, args->rot_dim, cache->head_dim) ||
      args->n_heads < 0 || args->n_heads > SEEDQ_ROPE_MAX_HEADS)
    return SEEDQ_ERR_INVALID_ARG;
  const bool queries = args->n_heads > 0;
  if (queries && !dtype_ok(args->out_dtype)) return SEEDQ_ERR_INVALID_ARG;
  if (n_tokens == 0) return SEEDQ_OK;
  if (!k || !v || !slots || !args->cos_sin || (uintptr_t)args->cos_sin % 8) return SEEDQ_ERR_INVALID_ARG;
  AppendArgs a{};
  a.c = *cache, a.x[0] = k, a.x[1] = v, a.ts = token_stride, a.hs = head_stride, a.n = n_tokens, a.slots = slots;
  a.cs = (const float2 *)args->cos_sin, a.half = args->rot_dim / 2, a.layout = args->layout;
  const uint64_t size = dtype_bytes(dtype);
  a.vec = ((uint64_t)(uintptr_t)k | (uint64_t)(uintptr_t)v | (uint64_t)token_stride * size | (uint64_t)head_stride * size) % 16 == 0;
  a.wide_cs = a.half % 2 == 0 && (uintptr_t)args->cos_sin % 16 == 0;
  const int64_t work = n_tokens * cache->n_kv_heads * 2;
  a.share = work <= kFewPairs ? 1 : kWarps;
  a.group_shift = work <= kFewPairs ? 3 : append_group_shift(n_tokens, cache->n_kv_heads);
  a.page_shift = log2_of(cache->page_size);
  const int64_t groups = (n_tokens + (1 << a.group_shift) - 1) >> a.group_shift;
  a.ctas_of_group = (unsigned)((cache->n_kv_heads + a.share - 1) / a.share);
  const int64_t ctas = 2 * groups * a.ctas_of_group;
  if (ctas > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  int64_t more = 0;
  if (queries) {
    if (!args->q || !args->q_out) return SEEDQ_ERR_INVALID_ARG;
    if (args->q == args->q_out && (args->out_dtype != dtype || args->q_token_stride != args->out_token_stride ||
                                   args->q_head_stride != args->out_head_stride))
      return SEEDQ_ERR_INVALID_ARG;
    a.q = RotateArgs{args->q, args->q_out, args->q_token_stride, args->q_head_stride, args->out_token_stride, args->out_head_stride,
                     n_tokens, args->n_heads, cache->head_dim, a.half, a.layout, args->out_dtype, a.cs};
    // keys, values and slots are read while queries are written
    const Wide row = (Wide)cache->head_dim * size, ob = dtype_bytes(args->out_dtype);
    const ByteRows out = byte_rows(args->q_out, cache->head_dim * ob, n_tokens, a.q.ot * ob, args->n_heads, a.q.oh * ob);
    for (const void *x : a.x)
      if (overlap(out, byte_rows(x, row, n_tokens, token_stride * (Wide)size, cache->n_kv_heads, head_stride * (Wide)size))) return SEEDQ_ERR_INVALID_ARG;
    if (rotate_overlaps(a.q, dtype) || overlap(out, byte_rows(slots, (Wide)n_tokens * 8))) return SEEDQ_ERR_INVALID_ARG;
    a.split = rotate_split(a.q, dtype, args->out_dtype);
    if (n_tokens * a.split.pieces * args->n_heads >= kQueriesApart) {
      const seedq_status rc = rotate_launch(a.q, dtype, (cudaStream_t)cuda_stream);
      if (rc != SEEDQ_OK) return rc;
    } else {
      more = (n_tokens * a.split.pieces * a.split.groups + kThreads - 1) / kThreads;
    }
  }
  if (ctas + more > INT32_MAX) return SEEDQ_ERR_UNSUPPORTED;
  a.ctas = (unsigned)ctas;
  const cudaError_t e = kLaunch[cache->kind][dtype](a, (unsigned)(ctas + more), (cudaStream_t)cuda_stream);
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}
