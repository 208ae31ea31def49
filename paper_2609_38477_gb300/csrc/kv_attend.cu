// Attention of the newest tokens over the 8-bit paged cache (seedq_kv_attend).
//
// Mathematics.  With codes c^k, c^v and block scales s^k, s^v a query row q of
// a head gives
//   z_j = scale * s^k_j (q . c^k_j),  out = sum_j p_j s^v_j c^v_j / sum_j p_j,
//   p_j = 2^(log2(e) z_j - m),  m a running maximum,
// one pass over the keys.  The products run on the tensor cores (m16n8k16,
// binary16 with float32 sums) with the cache as the 16-row operand: a decode
// step has few rows of its own (query heads that share a key-value head, times
// new tokens) and they fit the 8 columns.  Codes are exact in binary16; q and
// the weights p_j s^v_j, which are not, are held as a high and a low half (22
// bits; of q in a 16-bit type, scaled, the high half is all).  Up to 4 rows, the
// columns 0-3 carry the high and 4-7 the low halves of the same rows and the
// second half costs nothing; from 5 rows on the low halves are products of their
// own into the same sums.  q is scaled by a power of two per row, the weights
// p_j s^v_j of a row by one that brings the largest so far of its own (keys that it
// does not see count for nothing, whatever their scale) to 2^13, so binary16's
// range never cuts off more than 2^-37 of it.  Each unit's products start from
// zero and are added to float32 registers, so a long context is not accumulated
// inside the tensor cores, which truncate.
//
// What bounds it: the bytes of the cache, 2 head_dim per key and key-value
// head.  At 8 rows a byte costs 16 operations, far below the balance, but every
// code has to be widened (about 1.5 instructions) and multiplied.  Measured, 128
// head dims: 4 contexts of about 121000, 32 query on 8 key-value heads, 160 us (6.2
// TB/s, 91% of the copy rate); 64 of 2048 on 8 heads, 66 us with 32 query heads
// (4.0 TB/s) and 80 with 64, where the instructions bound it; 16 tokens of 32 heads
// over 32768 keys 93 us (tiles of 16 rows read and widen the keys four times), of 64
// heads 162 (eight times); one request of 1000 12 us, the latency of lengths, page numbers, keys and the joins.
//
// Layout.  For keys a product's row is a token and its inner index the head
// dim; the order of the inner index is free as long as q uses the same, so each
// lane takes 16 consecutive codes of a token and q's fragments are laid out to
// match.  For values the inner index is the token and a row a head dim, whose
// order is free again: lane (n, r) takes 16 consecutive codes of its four
// tokens.  A warp copies whole rows (cp.async, 16 bytes a lane: partial lines
// are fetched from L2 in 64-byte steps, and lane-private pieces of 32 bytes cost
// 1.75 times the traffic) into a ring of its own in shared memory, 16-byte pieces
// permuted so that neither the copies nor the lanes' reads meet in a bank.  Only
// the warp's own barrier is needed, strides are free, and what is past a
// request's end is filled with zeros instead of being read.
//
// Split.  The work list is every (request, key-value head, row tile) with its
// keys in units of kUnit tokens; it is cut into equal ranges of units, one per
// warp, so lengths need not be alike and nothing about them has to reach the
// host.  A warp that holds all units of an entry writes its output; the parts
// of entries cut between warps are joined by the CTA after one barrier, those
// cut between CTAs by the last CTA to arrive (a counter per CTA, reset by that
// CTA), always in the order of the keys: results do not depend on timing.
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cp_async.cuh"
#include "device_once.h"
#include "f32x2.cuh"
#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kMaxCtas = 152;      // one per SM
constexpr int kSmemMax = 227 * 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWeight = 13;  // a row's largest weight is held near 2^kWeight

// DP: head dim rounded up to 64, 128 or 256.  MODE: rows of a tile: 0: 4 (high
// and low halves share the 8 columns), 1: 8, 2: 16.  HALVES: of q, 1 where its
// type has no more than binary16's 11 bits.
template <int DP, int MODE, int HALVES>
struct Shape {
  static constexpr int kRows = 4 << MODE;
  static constexpr int kSets = MODE == 2 ? 2 : 1;    // sets of 8 columns
  static constexpr int kHalves = MODE == 0 ? 1 : 2;  // of the weights: operands per set
  static constexpr int kQHalves = MODE == 0 ? 1 : HALVES;  // of q
  static constexpr int kUnit = DP <= 128 ? 32 : 16;  // tokens of a unit
  static constexpr int kGroups = kUnit / 16;
  static constexpr int kChunks = DP / 64;            // 64 head dims: 16 codes of 4 lanes
  static constexpr int kVB = DP >= 128 ? 16 : 8;     // codes of a lane's value piece
  static constexpr int kLanes = DP / 16;             // lanes that copy a row
  static constexpr int kStep = 32 / kLanes;          // rows of a copy
  static constexpr int kVParts = DP / (8 * kVB);
  static constexpr int kTiles = DP / 16;             // output tiles of 16 head dims
  static constexpr int kValAt = kUnit * DP;
  static constexpr int kMetaAt = 2 * kUnit * DP;
  static constexpr int kStage = kMetaAt + 128;       // meta: per group both scales and a flag
  // 12 warps with a ring of 2 units or 8 with 3: tiles of 4 rows, few registers, take
  // 12 (64 requests of 2048, 32 heads on 8: 66 us, 8 warps 73); the work of 8 rows
  // is about as fast either way (64 on 8 heads: 80 us, 12 warps 77) and leaves fewer
  // parts to join (16 ragged requests up to 8192: 19.6 us, 12 warps 21.4).
  static constexpr int kWarps = MODE == 0 && DP <= 128 ? 12 : 8;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kStages = DP == 64 ? 4 : kWarps == 12 ? 2 : 3;  // units in a warp's ring
  // units, see the split of the work list
  static constexpr int kWhole = 8 * kWarps, kWholeLittle = 8, kWholeWarp = 6, kWholeWarpLittle = 2;
  static constexpr int kRequests = kThreads;                   // that the shared table holds
  static constexpr int kStats = 2 * 8 * kSets;                 // m and l of every column
  static constexpr int kSlot = kStats + kSets * kTiles * 128;  // floats of a part: stats, then lanes' products
  static_assert(kSlot * 4 <= kStages * kStage, "a part fits its warp's ring");
};

struct Args {
  seedq_kv_cache c;
  seedq_attend_args a;
  int32_t group;           // query heads per key-value head
  int32_t group_shift, gpp_shift;  // log2 of it, and of a page's groups of 16 tokens; -1 if there is none
  int32_t ctas;
  int32_t chunk;           // requests per entry of the table of units
  uint64_t ctas_inv;       // 2^64 / ctas, rounded up
  int32_t q_bytes;         // of an element of q
  int32_t q_vec, out_vec;  // q / out rows allow 16-byte accesses
};

// x / by for x >= 0, by > 0.  Below 2^20, (x + 1/2) / by is further from a whole
// number than the approximate quotient errs.
__device__ __forceinline__ int quotient(int64_t x, int by) {
  if (x < (1 << 20)) return (int)__fdividef((float)(int)x + 0.5f, (float)by);
  return x >> 31 ? (int)(x / by) : (int)((uint32_t)x / (uint32_t)by);
}
__device__ __forceinline__ int divide(int x, int by, int shift) { return shift >= 0 ? x >> shift : quotient(x, by); }

__device__ __forceinline__ void cp_async16z(uint32_t dst, const void *src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint32_t (&b)[2]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b[0]), "r"(b[1]));
}
// Transpose of an 8 x 8 matrix of binary16 over the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The whole number next to x, -127 at least, held as 1.5 * 2^23 more: differences
// are exact, and the low bits are the number.
__device__ __forceinline__ float exponent(float x) { return fmaxf(x, -127.f) + 12582912.f; }
__device__ __forceinline__ int exponent_bits(float x) { return (int)(__float_as_uint(x) - __float_as_uint(12582912.f)); }
__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t *>(&h); }

// x = hi + lo in binary16 (pairs).
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 f = __half22float2(h);
  hi = half2_bits(h);
  lo = half2_bits(__floats2half2_rn(x - f.x, y - f.y));
}

// Widen the codes in bytes (0, 1) and (2, 3) of w to binary16, exactly.  int8:
// byte + 128 placed under the exponent of 1024 is 1152 + code.
template <int KIND>
__device__ __forceinline__ uint32_t code_bias(uint32_t w) { return KIND == SEEDQ_KV_INT8 ? w ^ 0x80808080u : w; }
template <int KIND>
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) {
  if (KIND == SEEDQ_KV_E4M3) return e4m3x2_to_half2(w);
  const uint32_t x = __byte_perm(w, 0x64646464u, 0x4140u);
  return half2_bits(__hsub2(*reinterpret_cast<const __half2 *>(&x), __float2half2_rn(1152.f)));
}
template <int KIND>
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) {
  if (KIND == SEEDQ_KV_E4M3) return e4m3x2_to_half2(w >> 16);
  const uint32_t x = __byte_perm(w, 0x64646464u, 0x4342u);
  return half2_bits(__hsub2(*reinterpret_cast<const __half2 *>(&x), __float2half2_rn(1152.f)));
}

// A request's share of the work list.
struct __align__(16) Req {
  int first, fresh;  // its query tokens
  int len;           // cached tokens, the newest included
  int lo, hi;        // keys that any of its queries may see
  int tiles;         // row tiles
  int u0, units;     // its keys in units: u0 .. u0 + units - 1
};
template <typename S>
__device__ __forceinline__ Req request(const Args &p, int b) {
  Req r;
  const int n = (int)p.a.n_tokens;
  r.first = min(max(p.a.starts[b], 0), n);
  r.fresh = max(min(max(p.a.starts[b + 1], 0), n) - r.first, 0);
  r.len = p.a.seq_lens[b];
  const int64_t cap = (int64_t)p.a.table_width * p.c.page_size;  // below 2^29
  r.hi = min(max(r.len, 0), (int)cap);
  const int64_t lo = p.a.window > 0 ? (int64_t)r.len - r.fresh + 1 - p.a.window : 0;
  r.lo = (int)min(max(lo, (int64_t)0), (int64_t)r.hi);
  r.tiles = (int)(((int64_t)r.fresh * p.group + S::kRows - 1) / S::kRows);
  r.u0 = r.lo / S::kUnit;
  r.units = max((r.hi + S::kUnit - 1) / S::kUnit - r.u0, 1);
  return r;
}
// Steps of the work list: an entry's units and kStart more, the cost of its start
// (queries) and end, so that many short contexts weigh what they take (16 ragged
// contexts up to 8192: 26 us without, 20, 19 and 20 with 2 to 4; 64 up to 300: 23
// without, 18 with 2 to 4).
constexpr int kStart = 3;
constexpr int kOver = 24;
__device__ __forceinline__ int64_t steps_of(const Args &p, const Req &r) {
  return r.fresh ? (int64_t)(r.units + kStart) * r.tiles * p.c.n_kv_heads : 0;
}

// One entry of the work list: (request, key-value head, row tile).
struct Entry {
  Req r;
  int b, h, tile;
};  // its units are the steps after its first kStart
// The table of requests in shared memory: units before every chunk of
// requests, and, where a chunk is one request, the requests themselves.
template <typename S>
struct Table {
  int64_t before[S::kRequests];
  Req req[S::kRequests];
};
template <typename S>
__device__ __forceinline__ Req request(const Args &p, const Table<S> &t, int b) {
  return p.chunk == 1 ? t.req[b] : request<S>(p, b);
}
template <typename S>
__device__ __forceinline__ Entry entry_at(const Args &p, const Table<S> &t, int64_t u, int64_t &begin) {
  Entry e;
  int lo = 0, hi = (p.a.n_requests + p.chunk - 1) / p.chunk;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (t.before[mid] <= u) lo = mid;
    else hi = mid;
  }
  int64_t base = t.before[lo];
  e.b = lo * p.chunk;
  e.r = request<S>(p, t, e.b);
  for (int i = 1; i < p.chunk; ++i) {
    const int64_t n = steps_of(p, e.r);
    if (u < base + n) break;
    base += n;
    e.r = request<S>(p, ++e.b);
  }
  const int k = quotient(u - base, e.r.units + kStart);
  e.h = e.r.tiles == 1 ? k : quotient(k, e.r.tiles);
  e.tile = k - e.h * e.r.tiles;
  begin = base + (int64_t)k * (e.r.units + kStart);
  return e;
}
template <typename S>
__device__ __forceinline__ void next_entry(const Args &p, const Table<S> &t, Entry &e) {  // only where one follows
  if (++e.tile < e.r.tiles) return;
  e.tile = 0;
  if (++e.h < p.c.n_kv_heads) return;
  e.h = 0;
  do e.r = request<S>(p, t, ++e.b);
  while (e.r.fresh == 0);
}

// What the products and the joins need to know of an entry.
struct Desc {
  int first, fresh, len, hi;
  int h, tile;
  int token0;  // the first token of a warp's first unit of it
  int units;   // units of it that the warp holds
  int whole;   // whether these are all
  int64_t begin, end;  // the steps of its units
};

// Where a row of an entry's tile goes; false if it holds no query.
template <typename S>
__device__ __forceinline__ bool row_of(const Args &p, const Desc &e, int row, int64_t &token, int &head, int &pos) {
  const int r = e.tile * S::kRows + row, t = divide(r, p.group, p.group_shift);
  token = e.first + t;
  head = e.h * p.group + (r - t * p.group);
  pos = e.len - e.fresh + t;
  return t < e.fresh;
}

template <int N>  // N = 2 or 4 elements in a row from i on
__device__ __forceinline__ void store_row(void *out, int dt, int64_t i, const float (&x)[N], bool vec) {
  if (!vec) {
#pragma unroll
    for (int y = 0; y < N; ++y) store_elem(out, dt, i + y, x[y]);
  } else if (dt == SEEDQ_F32) {
    if constexpr (N == 4) *(float4 *)((float *)out + i) = make_float4(x[0], x[1], x[2], x[3]);
    else *(float2 *)((float *)out + i) = make_float2(x[0], x[1]);
  } else {
    uint32_t v[N / 2];
#pragma unroll
    for (int y = 0; y < N / 2; ++y) {
      if (dt == SEEDQ_BF16) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * y], x[2 * y + 1]);
        v[y] = *(const uint32_t *)&b;
      } else {
        v[y] = half2_bits(__floats2half2_rn(x[2 * y], x[2 * y + 1]));
      }
    }
    if constexpr (N == 4) *(uint2 *)((uint16_t *)out + i) = make_uint2(v[0], v[1]);
    else *(uint32_t *)((uint16_t *)out + i) = v[0];
  }
}

// A load that sees what other SMs wrote (generic address, past the L1 cache).
template <typename T>
__device__ __forceinline__ T load_fresh(const float *x) {
  T v;
  if constexpr (sizeof(T) == 8) asm volatile("ld.volatile.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(x) : "memory");
  else asm volatile("ld.volatile.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(x) : "memory");
  return v;
}

// Joins n parts of an entry into `to`, or, if to is null, writes the entry's
// output.  A part holds m (in units of log2) and l of every column and the
// columns' averages o = sum / l as the products' accumulators lie in the lanes;
// it weighs l 2^m.  Averages, not sums, are kept, of the parts and of what is
// joined so far, so nothing overflows on the way.  The parts are from[0..n-1],
// or, without `from`, the second of the two slots of the CTA at `slots` and the
// first ones of the n - 1 CTAs behind it.  The warp takes the tiles first, first +
// step, ...; a lane reads the statistics of its two columns itself, so no barrier
// is needed.
template <typename S, int MODE>
__device__ __forceinline__ void join(const Args &p, const Desc &e, int n, const float *const *from, const float *slots,
                                     float *to, int first, int step) {
  constexpr int kAtATime = 8;
  const int lane = threadIdx.x & 31, nn = lane >> 2, q4 = lane & 3;
#pragma unroll 1
  for (int tt = first; tt < S::kSets * S::kTiles; tt += step) {
    const int set = tt / S::kTiles, tile = tt - set * S::kTiles, col = set * 8 + 2 * q4;
    float m0 = -CUDART_INF_F, m1 = -CUDART_INF_F, l0 = 0.f, l1 = 0.f, c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int i = 0; i < n; i += kAtATime) {  // one latency
      float2 m[kAtATime], l[kAtATime];
      float4 o[kAtATime];
#pragma unroll
      for (int k = 0; k < kAtATime; ++k) {
        const int j = min(i + k, n - 1);
        const float *x = from ? from[j] : slots + (j ? 2 * j : 1) * S::kSlot;
        m[k] = load_fresh<float2>(x + col);
        l[k] = load_fresh<float2>(x + S::kStats / 2 + col);
        o[k] = load_fresh<float4>(x + S::kStats + (tt * 32 + lane) * 4);
      }
      const float was0 = m0, was1 = m1;
#pragma unroll
      for (int k = 0; k < kAtATime; ++k) {
        if (i + k >= n) l[k] = make_float2(0.f, 0.f);
        m0 = fmaxf(m0, m[k].x);
        m1 = fmaxf(m1, m[k].y);
      }
      const float u0 = m0 == -CUDART_INF_F ? 0.f : m0, u1 = m1 == -CUDART_INF_F ? 0.f : m1;
      const float s0 = l0 * exp2_fast(was0 - u0), s1 = l1 * exp2_fast(was1 - u1);
      l0 = s0, l1 = s1;
#pragma unroll
      for (int k = 0; k < kAtATime; ++k) {
        l[k].x = l[k].x == 0.f ? 0.f : l[k].x * exp2_fast(m[k].x - u0);
        l[k].y = l[k].y == 0.f ? 0.f : l[k].y * exp2_fast(m[k].y - u1);
        l0 += l[k].x;
        l1 += l[k].y;
      }
      const float i0 = l0 == 0.f ? 0.f : 1.f / l0, i1 = l1 == 0.f ? 0.f : 1.f / l1;
      c[0] *= s0 * i0, c[2] *= s0 * i0;
      c[1] *= s1 * i1, c[3] *= s1 * i1;
#pragma unroll
      for (int k = 0; k < kAtATime; ++k) {
        const float w0 = l[k].x * i0, w1 = l[k].y * i1;
        if (w0 != 0.f) c[0] = fmaf(w0, o[k].x, c[0]), c[2] = fmaf(w0, o[k].z, c[2]);
        if (w1 != 0.f) c[1] = fmaf(w1, o[k].y, c[1]), c[3] = fmaf(w1, o[k].w, c[3]);
      }
    }
    if (to) {
      if (tile == 0 && nn == 0) {
        *(float2 *)(to + col) = make_float2(m0, m1);
        *(float2 *)(to + S::kStats / 2 + col) = make_float2(l0, l1);
      }
      ((float4 *)(to + S::kStats))[tt * 32 + lane] = make_float4(c[0], c[1], c[2], c[3]);
      continue;
    }
    if (MODE == 0) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] += __shfl_xor_sync(~0u, c[k], 2);
      if (q4 >= 2) continue;
    }
    const int d = (2 * tile / S::kVB) * 128 + nn * S::kVB + 2 * tile % S::kVB;
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
      int64_t token;
      int head, pos;
      if (!row_of<S>(p, e, col + k, token, head, pos)) continue;
      const float x[2] = {k ? c[1] : c[0], k ? c[3] : c[2]};
      if (d < p.c.head_dim)
        store_row<2>(p.a.out, p.a.out_dtype, token * p.a.out_token_stride + head * p.a.out_head_stride + d, x, p.out_vec);
      if (p.a.lse && tile == 0 && nn == 0) {
        const float l = k ? l1 : l0, m = k ? m1 : m0;
        p.a.lse[token * p.a.n_heads + head] = l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * kLn2;
      }
    }
  }
}

// Rows of DP bytes in shared memory have their 16-byte pieces permuted, piece x
// of row r at x ^ swizzle(r): the rows (2a, 2a + 1) that the lanes of a key
// read share, and the rows 0, 2, 4, 6 of a value read, then lie in different
// banks.
template <int DP>
__host__ __device__ constexpr int swizzle(int r) {
  return DP >= 128 ? (r & 6) ^ ((r & 1) << 2) : (r >> 1) & 3;
}

template <int KIND, int DP, int MODE, int HALVES>
__global__ void __launch_bounds__(Shape<DP, MODE, HALVES>::kThreads, 1) k_attend(const __grid_constant__ Args p) {
  using S = Shape<DP, MODE, HALVES>;
  extern __shared__ __align__(128) uint8_t smem_raw[];
  uint8_t *smem = smem_raw + (128 - ((uint32_t)__cvta_generic_to_shared(smem_raw) & 127)) % 128;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int nn = lane >> 2, q4 = lane & 3;
  const int B = p.a.n_requests, D = p.c.head_dim;

  // ---- the work list: exclusive sums of the requests' units
  Table<S> &table = *(Table<S> *)smem;
  __shared__ int64_t s_sums[S::kWarps];
  __shared__ int s_most[S::kWarps], s_least[S::kWarps];
  int64_t total = 0, u = 0;
  int most = 0, least = INT32_MAX;  // units of the longest and of the shortest entry
  // With up to 32 requests every warp makes the sums, and all write the same
  // table; no barrier.
  const bool few = B <= 32;
  const int slot = few ? lane : tid;
  for (int b = slot * p.chunk; b < min((slot + 1) * p.chunk, B); ++b) {
    const Req r = request<S>(p, b);
    if (p.chunk == 1) table.req[b] = r;
    u += steps_of(p, r);
    if (r.fresh) most = max(most, r.units), least = min(least, r.units);
  }
  {
    int64_t x = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(~0u, x, o);
      if (lane >= o) x += y;
    }
    most = __reduce_max_sync(~0u, most);
    least = __reduce_min_sync(~0u, least);
    int64_t before = x - u;
    if (few) {
      total = __shfl_sync(~0u, x, 31);
      table.before[lane] = before;
      __syncwarp();
    } else {
      if (lane == 31) s_sums[w] = x, s_most[w] = most, s_least[w] = least;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < S::kWarps; ++k) {
        if (k < w) before += s_sums[k];
        total += s_sums[k];
        most = max(most, s_most[k]);
        least = min(least, s_least[k]);
      }
      table.before[tid] = before;
      __syncthreads();
    }
  }
  // Even shares of steps for the CTAs' warps, at least one each.  Little work goes
  // to 4 warps per CTA, one per scheduler, and so to more SMs (one request of 1000:
  // 12 us, with all warps 15).  Entries of one length (one request, or a batch in
  // step) are each cut for the same number of CTAs, so that no CTA has parts of two
  // (one request of 4096: 14.5 us, else 16).  Else, where no entry is longer than a
  // few units per warp and than a share by kOver, the shares' ends move to the
  // nearest entry's: a join between CTAs costs 3 to 4 us (40 ragged requests up to
  // 1000, 32 heads on 8: 19 us, without 22; 100: 26 and 30; but 16 up to 2048, whose
  // longest entry is twice a share, 22 with and 18 without; 256 up to 4096, 82 and
  // 78); with little work where none is longer than kWholeLittle (21 requests that
  // see a window of 33: 11 us, else 13).  Likewise between warps where no entry is
  // longer than kWholeWarp (200 requests up to 100: 19 us, else 25).
  const bool little = total <= (int64_t)p.ctas * 8;
  const int warps = little ? 4 : S::kWarps;
  const int64_t share = max((int64_t)__umul64hi((uint64_t)total, p.ctas_inv) + 1, (int64_t)warps);
  int cuts = 0;  // CTAs per entry, where all have as many
  if (most == least && total <= (int64_t)p.ctas * (most + kStart)) {
    const int entries = quotient(total, most + kStart);
    cuts = min(quotient(p.ctas, entries), little ? (most + 3) >> 2 : (most + S::kWarps - 1) / S::kWarps);
    if (!little && entries * cuts * 10 < p.ctas * 9) cuts = 0;
  }
  auto nearest = [&](int64_t u) -> int64_t {  // entry end nearest to u
    if (u >= total) return total;
    int64_t begin;
    const int length = entry_at<S>(p, table, u, begin).r.units + kStart;
    return u - begin <= begin + length - u ? begin : begin + length;
  };
  int64_t c0, c1;
  if (cuts) {
    const int entry = quotient(blockIdx.x, cuts), piece = blockIdx.x - entry * cuts;
    const int64_t at = (int64_t)entry * (most + kStart) + kStart;
    if (at >= total) return;
    c0 = at + quotient((int64_t)most * piece, cuts);
    c1 = at + quotient((int64_t)most * (piece + 1), cuts);
  } else {
    c0 = min(share * blockIdx.x, total), c1 = min(c0 + share, total);
    if (c0 >= total) return;
    if (little ? most <= S::kWholeLittle : most <= S::kWhole && most + kStart <= share + kOver) {
      const int64_t c = nearest(lane ? c1 : c0);
      c0 = __shfl_sync(~0u, c, 0);
      c1 = __shfl_sync(~0u, c, 1);
      if (c0 >= c1) return;
    }
  }
  const uint32_t mine = (uint32_t)(c1 - c0);  // split in even shares without passing 32 bits
  const uint32_t each = little ? mine / 4 : mine / S::kWarps, rest = mine - each * warps;
  int64_t w0 = c0 + each * (uint32_t)min(w, warps) + min((uint32_t)w, rest);
  int64_t w1 = w < warps ? w0 + each + (w < (int)rest) : w0;
  if (most <= (little ? S::kWholeWarpLittle : S::kWholeWarp)) {
    if (cuts == 1) {  // the CTA's only entry
      w0 = c0;
      w1 = w == 0 ? c1 : c0;
    } else if (cuts == 0) {
      const int64_t c = nearest(lane ? w1 : w0);
      w0 = __shfl_sync(~0u, c, 0);
      w1 = __shfl_sync(~0u, c, 1);
    }
  }

  // Rows begin at multiples of 128 bytes: a copy whose 32-byte sectors straddle
  // those of shared memory is fetched twice from L2.
  constexpr int ring_at = (sizeof(Table<S>) + 127) & ~127;
  uint8_t *ring = smem + ring_at + (size_t)w * S::kStages * S::kStage;
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  float *ws = (float *)((uint8_t *)p.a.workspace + kMaxCtas * 4);
  float *cta_slots = ws + (size_t)blockIdx.x * 2 * S::kSlot;
  // What the joins need again, so that it takes no registers until then.
  __shared__ struct { int64_t share, c0, c1; int cuts, length; } s_split;
  __shared__ int64_t s_first[S::kWarps];  // the warps' first steps
  if (tid == 0) s_split = {share, c0, c1, cuts, most + kStart};
  if (lane == 0) s_first[w] = w0;
  const int steps = (int)(w1 - w0);
  // Entries on their way from the copies to the products.
  __shared__ Desc s_desc[S::kWarps][S::kStages + 1];
  // Parts of cut entries, in the order of their keys: [2 w] a warp's first
  // entry if more follow, [2 w + 1] its last.
  __shared__ Desc s_cut[2 * S::kWarps];
  if (lane < 2) s_cut[2 * w + lane].units = 0;

  // ---- copies
  const int gpp = p.c.page_size >> 4;  // groups of 16 tokens per page
  const int64_t ts = p.c.token_stride, tstep = S::kStep * ts;
  const int crow = lane / S::kLanes, cat = lane % S::kLanes * 16;  // the lane's row and first code of a copy
  const int64_t clane = crow * ts + cat;
  // The place of 16-byte piece x of row r: x ^ swizzle(r).
  const uint32_t cdst = crow * DP + ((lane % S::kLanes) ^ swizzle<DP>(crow)) * 16;
  __shared__ Entry s_entry[S::kWarps];  // the entries being copied
  int pb = -1, ph = 0, plo = 0, phi = 0;  // of this warp's: its request, head and keys
  int plast = 0;                          // where it ends, in steps from the warp's first
  const int32_t *prow = nullptr;
  int pleft = 0;               // its units still to copy by this warp
  int copied = 0;              // units copied so far
  bool more = steps > 0;       // whether there are others
  int pg = 0, pgb = 0;         // the next group of 16 tokens; the group of lane 0's page
  int poff = 0;                // the next group's place in its page
  int ids = -1, ids_next = -1; // pages of the groups pgb + lane and pgb + 32 + lane
  int pstage = 0, pdesc = 0, cdesc = 0, stage = 0;
  auto load_ids = [&](int g) -> int {
    const int64_t gl = (int64_t)g + lane;
    return gl * 16 < phi ? __ldg(prow + divide((int)gl, gpp, p.gpp_shift)) : -1;
  };

  // ---- products
  uint32_t qf[S::kSets][S::kQHalves][S::kChunks * 4][2];  // q as the second operand
  float zf[S::kSets][2];      // z in units of log2 per unit of product, but for the key scale
  float m[S::kSets][2], l[S::kSets][2];
  float top[S::kSets][2];     // log2 of the row's largest p s^v so far, relative to 2^m (s^v as the power of two below it)
  uint64_t o[S::kSets][S::kTiles][2];  // sums of the columns (2 q4, 2 q4 + 1) for two head dims
  int cleft = 0, tok = 0, see_all = 0, see_from = 0;  // units of the tokens see_from < t <= see_all need no mask
  // and of a value tile: piece n (DP 64: half of piece n / 2) of row 2 q4
  const uint32_t vat = 2 * q4 * DP + (S::kVB == 16 ? (nn ^ swizzle<DP>(2 * q4)) * 16 : ((nn >> 1) ^ swizzle<DP>(2 * q4)) * 16 + (nn & 1) * 8);
  const uint32_t kat = nn * DP + (q4 ^ swizzle<DP>(nn)) * 16;  // the lane's first codes of a key tile

#pragma unroll 1
  for (int it = 1 - S::kStages;; ++it) {
    __syncwarp();  // all lanes are done with the stage that is filled next
    if (more && pleft == 0) {
      // The next entry with a unit in the warp's steps.
      if (copied > 0 && plast >= steps) {
        more = false;
      } else {
        Entry pe;
        int begin = plast;
        if (copied == 0) {
          int64_t at;
          pe = entry_at<S>(p, table, s_first[w], at);
          begin = (int)(at - s_first[w]);
        } else {
          pe = s_entry[w];
          next_entry<S>(p, table, pe);
        }
        __syncwarp();
        if (lane == 0) s_entry[w] = pe;
        plast = begin + kStart + pe.r.units;
        const int from = max(begin + kStart, 0);
        pleft = max(min(plast, steps) - from, 0);
        more = pleft > 0;  // else its start alone
        plo = pe.r.lo, phi = pe.r.hi, ph = pe.h;
        prow = p.a.block_table + (int64_t)pe.b * p.a.table_stride;
        pg = (pe.r.u0 + from - begin - kStart) * S::kGroups;
        poff = pg - divide(pg, gpp, p.gpp_shift) * gpp;
        if (pe.b != pb || pg != pgb) {  // the next head of a request reads the same pages
          pgb = pg;
          ids = load_ids(pgb);
          ids_next = load_ids(pgb + 32);
        }
        pb = pe.b;
        if (lane == 0) {
          Desc &x = s_desc[w][pdesc];
          x.first = pe.r.first, x.fresh = pe.r.fresh, x.len = pe.r.len, x.hi = pe.r.hi;
          x.h = pe.h, x.tile = pe.tile, x.token0 = pg * 16, x.units = pleft;
          x.begin = s_first[w] + begin + kStart, x.end = x.begin + pe.r.units;
          x.whole = pleft == pe.r.units;
        }
        pdesc = pdesc == S::kStages ? 0 : pdesc + 1;
        // its queries' first touch, while the page numbers are on their way
        const int r = pe.tile * S::kRows + lane, t = divide(r, p.group, p.group_shift);
        if (lane < S::kRows && t < pe.r.fresh) {
          const char *row = (const char *)p.a.q + ((int64_t)(pe.r.first + t) * p.a.q_token_stride +
                                                   (pe.h * p.group + r - t * p.group) * p.a.q_head_stride) * p.q_bytes;
          for (int x = 0; x < D * p.q_bytes; x += 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(row + x));
        }
      }
    }
    if (more) {
      __syncwarp();
      int my_page = -1;
      --pleft;
      ++copied;
      const uint32_t dst = ring_s + pstage * S::kStage;
      pstage = pstage + 1 == S::kStages ? 0 : pstage + 1;
      if (pg - pgb >= 32) {
        pgb += 32;
        ids = ids_next;
        ids_next = load_ids(pgb + 32);
      }
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
        const int page = __shfl_sync(~0u, ids, pg - pgb);
        const int t0 = pg * 16;
        const bool in = page >= 0 && page < p.c.n_pages && t0 + 16 > plo;  // ids is -1 past hi
        const int left = in ? phi - t0 : 0;                                // tokens of the group that exist
        const int64_t at = in ? page * p.c.page_stride + ph * p.c.head_stride + poff * 16 * ts : 0;
        ++pg;
        poff = poff + 1 == gpp ? 0 : poff + 1;
        const uint8_t *kp = (const uint8_t *)p.c.k + at + clane, *vp = (const uint8_t *)p.c.v + at + clane;
        const uint32_t to = dst + g * (16 * DP);
        const bool full = left >= 16 && D == DP;  // every copy is wanted
#pragma unroll
        for (int t = 0; t < 16 / S::kStep; ++t) {
          const int row = t * S::kStep;  // the lanes' rows begin here
          const uint32_t x = to + ((row * DP + cdst) ^ (swizzle<DP>(row) * 16));
          const bool ok = full || (row + crow < left && cat < D);
          cp_async16z(x, ok ? kp : (const uint8_t *)p.c.k, ok);
          cp_async16z(x + S::kValAt, ok ? vp : (const uint8_t *)p.c.v, ok);
          kp += tstep;
          vp += tstep;
        }
        if ((lane >> 1) == g) my_page = in ? page : -1;
      }
      // the groups' scales and flags, two lanes a group, after all copies: a warp
      // that has split up fetches lines twice
      if (lane < 2 * S::kGroups) {
        const uint32_t meta = dst + S::kMetaAt + (lane >> 1) * 16;
        if (my_page >= 0) {
          const float *sc = (lane & 1 ? p.c.v_scale : p.c.k_scale) + (int64_t)my_page * p.c.n_kv_heads + ph;
          asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(meta + (lane & 1) * 4), "l"(sc) : "memory");
        } else {
          asm volatile("st.shared.f32 [%0], %1;" ::"r"(meta + (lane & 1) * 4), "f"(0.f) : "memory");
        }
        if ((lane & 1) == 0) asm volatile("st.shared.s32 [%0], %1;" ::"r"(meta + 8), "r"(my_page >= 0 ? 1 : 0) : "memory");
      }
    }
    cp_async_commit();
    int ahead = it;
    asm volatile("" : "+r"(ahead));  // keeps the compiler from splitting the loop here and writing the copies out twice
    if (ahead < 0) continue;
    if (ahead == copied) break;  // the copies run ahead, so there is no other unit

    if (cleft == 0) {  // a new entry: its queries
      const Desc e = s_desc[w][cdesc];
      cleft = e.units;
      tok = e.token0;
      {
        const int r0 = e.tile * S::kRows, t0 = divide(r0, p.group, p.group_shift), t1 = divide(r0 + S::kRows - 1, p.group, p.group_shift);
        see_all = min(e.len - e.fresh + t0, e.hi - 1);
        see_from = p.a.window > 0 ? min(e.len - e.fresh + t1, e.len - 1) - p.a.window : -1;
      }
#pragma unroll
      for (int s = 0; s < S::kSets; ++s) {
#pragma unroll
        for (int j = 0; j < S::kTiles; ++j) o[s][j][0] = o[s][j][1] = 0;
        int64_t token;
        int head, ps;
        const bool real = row_of<S>(p, e, MODE == 0 ? nn & 3 : s * 8 + nn, token, head, ps);
        const int64_t at = real ? token * p.a.q_token_stride + head * p.a.q_head_stride : 0;
        float x[S::kChunks * 16], amax = 0.f;
#pragma unroll
        for (int k = 0; k < S::kChunks * 16; ++k) x[k] = 0.f;
        if (p.q_vec && p.a.q_dtype == SEEDQ_F32) {
#pragma unroll
          for (int k = 0; k < S::kChunks * 4; ++k) {
            const int d = (k >> 2) * 64 + q4 * 16 + (k & 3) * 4;
            if (real && d < D) {
              const float4 f = __ldg((const float4 *)((const float *)p.a.q + at + d));
              x[k * 4] = f.x, x[k * 4 + 1] = f.y, x[k * 4 + 2] = f.z, x[k * 4 + 3] = f.w;
            }
          }
        } else if (p.q_vec) {
          const bool bf = p.a.q_dtype == SEEDQ_BF16;
          uint4 v[S::kChunks * 2];
#pragma unroll
          for (int k = 0; k < S::kChunks * 2; ++k) {
            const int d = (k >> 1) * 64 + q4 * 16 + (k & 1) * 8;
            v[k] = real && d < D ? __ldg((const uint4 *)((const uint16_t *)p.a.q + at + d)) : make_uint4(0, 0, 0, 0);
          }
#pragma unroll
          for (int k = 0; k < S::kChunks * 8; ++k) {
            const uint32_t y = (&v[k >> 2].x)[k & 3];
            const float2 g = bf ? make_float2(__uint_as_float(y << 16), __uint_as_float(y & 0xffff0000u))
                                : __half22float2(*reinterpret_cast<const __half2 *>(&y));
            x[2 * k] = g.x, x[2 * k + 1] = g.y;
          }
        } else if (real) {
          float slow[S::kChunks * 16];  // in local memory: rows that do not allow wide loads
#pragma unroll 1
          for (int k = 0; k < S::kChunks * 16; ++k) {
            const int d = (k >> 4) * 64 + q4 * 16 + (k & 15);
            slow[k] = d < D ? load_elem(p.a.q, p.a.q_dtype, at + d) : 0.f;
          }
#pragma unroll
          for (int k = 0; k < S::kChunks * 16; ++k) x[k] = slow[k];
        }
#pragma unroll
        for (int k = 0; k < S::kChunks * 16; ++k) amax = fmaxf(amax, fabsf(x[k]));
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
        // The row times a power of two, its largest number in [2^13, 2^14).
        int ex = amax > 0.f && amax < CUDART_INF_F ? 13 + 127 - (int)(__float_as_uint(amax) >> 23) : 0;
        ex = min(max(ex, -126), 126);
        const float up = __uint_as_float((uint32_t)(127 + ex) << 23);
        const float f = p.a.scale * kLog2e * __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
        for (int k = 0; k < S::kChunks * 4; ++k)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint32_t a, b;
            split2(x[k * 4 + 2 * y] * up, x[k * 4 + 2 * y + 1] * up, a, b);
            if (MODE == 0) {
              qf[s][0][k][y] = nn < 4 ? a : b;
            } else {
              qf[s][0][k][y] = a;
              if (S::kQHalves == 2) qf[s][S::kQHalves - 1][k][y] = b;
            }
          }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int col = 2 * q4 + k;
          zf[s][k] = __shfl_sync(~0u, f, col * 4);
          m[s][k] = top[s][k] = -CUDART_INF_F;
          l[s][k] = 0.f;
        }
      }
    }

    cp_async_wait<S::kStages - 1>();
    __syncwarp();
    const uint8_t *st = ring + stage * S::kStage;
    stage = stage + 1 == S::kStages ? 0 : stage + 1;
    float ks[S::kGroups], vs[S::kGroups];
    bool all_in = true;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const float *meta = (const float *)(st + S::kMetaAt + g * 16);
      ks[g] = meta[0];
      vs[g] = meta[1];
      all_in = all_in && ((const int *)meta)[2];
    }

    // scores: 16 tokens by 8 columns per set
    float z[S::kSets][S::kGroups][4];  // tokens n, n, n + 8, n + 8 of the columns 2 q4, 2 q4 + 1
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      // Sums of at most 4 products within the tensor cores, which truncate where
      // they add: one for 64 head dims and half.
      uint64_t sum[S::kSets][2];
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        float acc[S::kSets][S::kQHalves][4] = {};
        const uint32_t at = g * (16 * DP) + (kat ^ (c * 64));
        const uint4 x = *(const uint4 *)(st + at), y = *(const uint4 *)(st + at + 8 * DP);  // the tokens n and n + 8
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t a = code_bias<KIND>(xw[k]), b = code_bias<KIND>(yw[k]);
          const uint32_t a0 = widen_lo<KIND>(a), a1 = widen_lo<KIND>(b), a2 = widen_hi<KIND>(a), a3 = widen_hi<KIND>(b);
#pragma unroll
          for (int s = 0; s < S::kSets; ++s)
#pragma unroll
            for (int hf = 0; hf < S::kQHalves; ++hf) mma(acc[s][hf], a0, a1, a2, a3, qf[s][hf][c * 4 + k]);
        }
#pragma unroll
        for (int s = 0; s < S::kSets; ++s)
#pragma unroll
          for (int hf = 0; hf < S::kQHalves; ++hf)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint64_t x = f2_pack(acc[s][hf][2 * k], acc[s][hf][2 * k + 1]);
              sum[s][k] = c + hf == 0 ? x : f2_add(sum[s][k], x);
            }
      }
#pragma unroll
      for (int s = 0; s < S::kSets; ++s)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 pair = f2_unpack(sum[s][k >> 1]);
          float v = k & 1 ? pair.y : pair.x;
          if (MODE == 0) v += __shfl_xor_sync(~0u, v, 2);
          z[s][g][k] = v * (zf[s][k & 1] * ks[g]);
        }
    }

    const bool masked = !all_in || tok + S::kUnit - 1 > see_all || tok <= see_from;
    if (masked) {
      const Desc e = s_desc[w][cdesc];
#pragma unroll
      for (int s = 0; s < S::kSets; ++s)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          int64_t token;
          int head, pos;
          row_of<S>(p, e, MODE == 0 ? (2 * q4 + c) & 3 : s * 8 + 2 * q4 + c, token, head, pos);
          const int to = min(pos, e.hi - 1), from = p.a.window > 0 ? pos - p.a.window : -1;
#pragma unroll
          for (int g = 0; g < S::kGroups; ++g) {
            const bool in = ((const int *)(st + S::kMetaAt + g * 16))[2];
#pragma unroll
            for (int k = c; k < 4; k += 2) {
              const int j = tok + g * 16 + nn + (k >> 1) * 8;
              if (!in || j > to || j <= from) z[s][g][k] = -CUDART_INF_F;
            }
          }
        }
    }

    // the block scales of the values as vf 2^ve, 1 <= |vf| < 2 but for the ends of the range
    float vf[S::kGroups];
    int ve[S::kGroups];
    bool alike = true;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      ve[g] = min((int)(__float_as_uint(vs[g]) >> 23 & 255), 253) - 127;
      vf[g] = vs[g] * __uint_as_float((uint32_t)(127 - ve[g]) << 23);
      alike = alike && ve[g] == ve[0];
    }

    uint32_t pf[S::kSets][S::kHalves][S::kGroups][2];
    uint64_t corr[S::kSets];
#pragma unroll
    for (int s = 0; s < S::kSets; ++s) {
      float cr[2], mu[2], vr[S::kGroups][2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float most[S::kGroups];  // of a group's z
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g) {
          most[g] = fmaxf(z[s][g][k], z[s][g][2 + k]);
          if (g && alike) most[0] = fmaxf(most[0], most[g]);
        }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) most[0] = fmaxf(most[0], __shfl_xor_sync(~0u, most[0], o));
        if (!alike)
#pragma unroll
          for (int g = 1; g < S::kGroups; ++g)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) most[g] = fmaxf(most[g], __shfl_xor_sync(~0u, most[g], o));
        float mx = fmaxf(m[s][k], most[0]);
        if (!alike)
#pragma unroll
          for (int g = 1; g < S::kGroups; ++g) mx = fmaxf(mx, most[g]);
        mu[k] = mx == -CUDART_INF_F ? 0.f : mx;
        const float fall = m[s][k] - mu[k], held = exponent(top[s][k]);
        float high = fmaxf(top[s][k] + fall, most[0] - mu[k] + ve[0]);
        if (!alike)
#pragma unroll
          for (int g = 1; g < S::kGroups; ++g) high = fmaxf(high, most[g] - mu[k] + ve[g]);
        m[s][k] = mx;
        top[s][k] = high;
        const float hold = exponent(high);
        l[s][k] *= exp2_fast(fall);
        cr[k] = exp2_fast(fall + (held - hold));
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g) {
          const int ex = ve[g] + kWeight + 127 - exponent_bits(hold);
          vr[g][k] = vf[g] * __uint_as_float((uint32_t)min(max(ex, 1), 254) << 23);
        }
      }
      corr[s] = f2_pack(cr[0], cr[1]);
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float wt[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float zz = z[s][g][2 * t + k], pr = exp2_fast(zz - mu[k]);
            l[s][k] += pr;
            wt[k] = pr * vr[g][k];
            if (masked && zz == -CUDART_INF_F) wt[k] = 0.f;  // 0, whatever the scale is
          }
          uint32_t a, b;
          split2(wt[0], wt[1], a, b);
          if (MODE == 0) {
            pf[s][0][g][t] = transpose8(q4 < 2 ? a : b);
          } else {
            pf[s][0][g][t] = transpose8(a);
            pf[s][S::kHalves - 1][g][t] = transpose8(b);
          }
        }
    }

#pragma unroll
    for (int part = 0; part < S::kVParts; ++part)
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
        uint32_t vw[4][S::kVB / 4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int row = (t >> 1) * 8 + (t & 1);  // and 2 q4 rows on
          const uint8_t *src = st + S::kValAt + g * (16 * DP) + row * DP + part * 128;
          if constexpr (S::kVB == 16) {
            const uint4 x = *(const uint4 *)(src + (vat ^ (t & 1) * 64));
            vw[t][0] = x.x, vw[t][1] = x.y, vw[t][2] = x.z, vw[t][3] = x.w;
          } else {
            const uint2 x = *(const uint2 *)(src + vat);
            vw[t][0] = x.x, vw[t][1] = x.y;
          }
        }
#pragma unroll
        for (int y = 0; y < S::kVB / 4; ++y) {
          uint32_t a[2][4];  // the bytes (0, 1) and (2, 3) of the words: two tiles
#pragma unroll
          for (int k = 0; k < 2; ++k) {  // the tokens (2r, 2r + 1) and (2r + 8, 2r + 9)
            const uint32_t x = code_bias<KIND>(vw[2 * k][y]), xx = code_bias<KIND>(vw[2 * k + 1][y]);
            const uint32_t lo = __byte_perm(x, xx, 0x5140), up = __byte_perm(x, xx, 0x7362);
            a[0][2 * k] = widen_lo<KIND>(lo);
            a[0][2 * k + 1] = widen_hi<KIND>(lo);
            a[1][2 * k] = widen_lo<KIND>(up);
            a[1][2 * k + 1] = widen_hi<KIND>(up);
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int j = part * (S::kVB / 2) + y * 2 + k;
#pragma unroll
            for (int s = 0; s < S::kSets; ++s) {
              float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
              for (int hf = 0; hf < S::kHalves; ++hf) mma(acc, a[k][0], a[k][1], a[k][2], a[k][3], pf[s][hf][g]);
              const uint64_t a01 = f2_pack(acc[0], acc[1]), a23 = f2_pack(acc[2], acc[3]);
              o[s][j][0] = g == 0 ? f2_fma(o[s][j][0], corr[s], a01) : f2_add(o[s][j][0], a01);
              o[s][j][1] = g == 0 ? f2_fma(o[s][j][1], corr[s], a23) : f2_add(o[s][j][1], a23);
            }
          }
        }
      }
    tok += S::kUnit;
    if (--cleft) continue;

    // ---- the end of this warp's part of an entry
    const int edesc = cdesc;
    const Desc e = s_desc[w][edesc];
    cdesc = cdesc == S::kStages ? 0 : cdesc + 1;
    const bool whole = e.whole, last = !more && it + 1 == copied;
    float inv[S::kSets][2], unit[S::kSets][2];
#pragma unroll
    for (int s = 0; s < S::kSets; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float sum = l[s][k];
        sum += __shfl_xor_sync(~0u, sum, 4);
        sum += __shfl_xor_sync(~0u, sum, 8);
        sum += __shfl_xor_sync(~0u, sum, 16);
        l[s][k] = sum;
        // o / l first: that is small, the block scales may not be
        inv[s][k] = sum == 0.f ? 0.f : __fdiv_rn(1.f / (1 << kWeight), sum);
        const int ex = exponent_bits(exponent(top[s][k]));  // -127 to 126
        unit[s][k] = __uint_as_float(ex == -127 ? 1u << 22 : (uint32_t)(ex + 127) << 23);
      }
    if (!whole) {
      // Its place: the ring if the warp is done, else a slot in the workspace.
      float *part = last ? (float *)ring : ws + (size_t)(kMaxCtas * 2 + blockIdx.x * S::kWarps + w) * S::kSlot;
      if (last) cp_async_wait<0>();
      __syncwarp();
      if (lane < (int)sizeof(Desc) / 4) ((int *)&s_cut[2 * w + last])[lane] = ((const int *)&s_desc[w][edesc])[lane];
#pragma unroll
      for (int s = 0; s < S::kSets; ++s) {
        if (nn == 0) {
          *(float2 *)(part + s * 8 + 2 * q4) = make_float2(m[s][0], m[s][1]);
          *(float2 *)(part + S::kStats / 2 + s * 8 + 2 * q4) = make_float2(l[s][0], l[s][1]);
        }
#pragma unroll
        for (int j = 0; j < S::kTiles; ++j) {
          const float2 x = f2_unpack(o[s][j][0]), y = f2_unpack(o[s][j][1]);
          ((float4 *)(part + S::kStats))[(s * S::kTiles + j) * 32 + lane] =
              make_float4(x.x * inv[s][0] * unit[s][0], x.y * inv[s][1] * unit[s][1], y.x * inv[s][0] * unit[s][0],
                          y.y * inv[s][1] * unit[s][1]);
        }
      }
      continue;
    }
    float4 x[S::kSets * S::kTiles];  // in local memory, so that what follows is a loop and not a page of code
    float2 ml[S::kSets][2];
#pragma unroll
    for (int s = 0; s < S::kSets; ++s) {
#pragma unroll
      for (int j = 0; j < S::kTiles; ++j) {
        const float2 a = f2_unpack(o[s][j][0]), b = f2_unpack(o[s][j][1]);
        x[s * S::kTiles + j] = make_float4(a.x * inv[s][0] * unit[s][0], a.y * inv[s][1] * unit[s][1],
                                              b.x * inv[s][0] * unit[s][0], b.y * inv[s][1] * unit[s][1]);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) ml[s][k] = make_float2(m[s][k], l[s][k]);
    }
#pragma unroll 1
    for (int k = 0; k < 2 * S::kSets; ++k) {
      const int s = k >> 1, row = MODE == 0 ? (2 * q4 + k) & 3 : s * 8 + 2 * q4 + (k & 1);
      int64_t token;
      int head, ps;
      const bool real = row_of<S>(p, e, row, token, head, ps);
      const int64_t at = token * p.a.out_token_stride + head * p.a.out_head_stride;
#pragma unroll 1
      for (int j = 0; j < S::kTiles; j += 2) {
        const float4 a = x[s * S::kTiles + j], b = x[s * S::kTiles + j + 1];
        float y[4] = {k & 1 ? a.y : a.x, k & 1 ? a.w : a.z, k & 1 ? b.y : b.x, k & 1 ? b.w : b.z};
        if (MODE == 0) {
          // the lanes of the high and the low halves then hold the same sums and take turns
#pragma unroll
          for (int t = 0; t < 4; ++t) y[t] += __shfl_xor_sync(~0u, y[t], 2);
          if ((j >> 1 & 1) != (q4 >> 1)) continue;
        }
        const int d = (2 * j / S::kVB) * 128 + nn * S::kVB + 2 * j % S::kVB;
        if (real && d < D) store_row<4>(p.a.out, p.a.out_dtype, at + d, y, p.out_vec);
      }
      if (real && p.a.lse && nn == 0 && (MODE != 0 || q4 < 2)) {
        const float2 v = ml[s][k & 1];
        p.a.lse[token * p.a.n_heads + head] = v.y == 0.f ? -CUDART_INF_F : (v.x + log2f(v.y)) * kLn2;
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();

  // ---- joins: first the entries cut between warps of this CTA, then, if this
  // CTA is the last to arrive, those cut between CTAs
  __shared__ const float *s_from[2 * S::kWarps];
  __shared__ int s_last[2];
  int *counters = (int *)p.a.workspace;
  c0 = s_split.c0, c1 = s_split.c1;
  const int64_t begin = lane < 2 * S::kWarps && s_cut[lane].units ? s_cut[lane].begin : -1;
  const uint32_t parts = __ballot_sync(~0u, begin >= 0);
  if (parts == 0) return;
  // the entries' first parts; an entry's parts are neighbours
  const uint32_t below = parts & ((1u << lane) - 1);
  const int64_t begin_before = __shfl_sync(~0u, begin, below ? 31 - __clz(below) : 0);
  const uint32_t heads = __ballot_sync(~0u, begin >= 0 && (below == 0 || begin_before != begin));
  if (w == 0 && begin >= 0) {
    const int pw = lane >> 1;
    s_from[__popc(below)] = lane & 1 ? (const float *)(smem + ring_at + (size_t)pw * S::kStages * S::kStage)
                                     : ws + (size_t)(kMaxCtas * 2 + blockIdx.x * S::kWarps + pw) * S::kSlot;
  }
  // cut between CTAs: the entry that came from before, the one that goes on
  int cross[2] = {__ffs(parts) - 1, 31 - __clz(parts)};
  if (s_cut[cross[1]].begin < c0 || s_cut[cross[1]].end <= c1) cross[1] = -1;
  if (s_cut[cross[0]].begin >= c0) cross[0] = -1;
  // One or two entries are joined by all warps, tile by tile, more by a warp each.
  const bool shared = __popc(heads) <= 2;
  __syncthreads();
  // the CTAs that hold a cut entry
  auto first_cta = [&](const Desc &x) -> int {
    const int n = s_split.cuts;
    return n ? quotient(x.begin, s_split.length) * n : (int)(x.begin / s_split.share);
  };
  auto cta_count = [&](const Desc &x) -> int {
    return s_split.cuts ? s_split.cuts : (int)((x.end - 1) / s_split.share) - first_cta(x) + 1;
  };
  int turn = 0, side = -1;
  uint32_t todo = heads;
#pragma unroll 1
  while (true) {
    int n, first = w, step = S::kWarps;
    const float *const *list = s_from;
    const float *slots = nullptr;
    float *to = nullptr;
    Desc e;
    if (todo) {
      const int i = __ffs(todo) - 1;
      todo &= todo - 1;
      if (!shared) {
        if (turn++ % S::kWarps != w) continue;
        first = 0, step = 1;
      }
      e = s_cut[i];
      n = __popc(__ballot_sync(~0u, begin == e.begin));
      list += __popc(parts & ((1u << i) - 1));
      if (e.begin < c0) to = cta_slots;
      else if (e.end > c1) to = cta_slots + S::kSlot;
    } else {
      if (side < 0) {  // the parts are written: the last CTA to arrive joins them
        if (cross[0] < 0 && cross[1] < 0) break;
        __syncthreads();
        if (lane == 0 && w < 2 && cross[w] >= 0) {
          const Desc &x = s_cut[cross[w]];
          const int a = first_cta(x), all = cta_count(x);
          // the CTA's parts, seen through the barrier, before the arrival, and the others' after it
          int seen;
          asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(seen) : "l"(counters + a) : "memory");
          s_last[w] = seen == all - 1 ? all : 0;
          if (s_last[w]) counters[a] = 0;
        }
        __syncthreads();
      }
      if (++side == 2) break;
      if (cross[side] < 0 || s_last[side] == 0) continue;
      e = s_cut[cross[side]];
      n = s_last[side];
      // the first CTA's part is its second slot, the others' their first
      list = nullptr;
      slots = ws + (size_t)first_cta(e) * 2 * S::kSlot;
    }
    join<S, MODE>(p, e, n, list, slots, to, first, step);
  }
}

struct Plan {
  int dp, mode, rows;
};
// Tiles of 4 rows where they hold all rows that share a head's keys (a decode
// step of up to 4 query heads per key-value head, half the products of 8 rows:
// 66 us for 64 requests of 2048, 32 heads on 8, else 80), else of 8 (5 to 8 rows in
// tiles of 16: 119 us instead of 80), and of 16 where more than 8 rows would read
// the keys again (16 tokens of 32 heads on 8 over 32768 keys: 93 us, else 111; of 32
// on 32 over a window of 3000 25, else 22); 256 head dims leave no registers for 16.
Plan shape_for(const seedq_kv_cache *c, int32_t n_heads, int32_t max_new) {
  Plan s;
  s.dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
  const int64_t rows = (int64_t)(n_heads / c->n_kv_heads) * max_new;
  s.mode = rows <= 4 ? 0 : rows <= 8 || s.dp == 256 ? 1 : 2;
  s.rows = 4 << s.mode;
  return s;
}
template <int DP, int MODE>
constexpr uint64_t workspace_bytes() {
  using S = Shape<DP, MODE, 2>;
  // arrival counters; per CTA two parts of entries cut between CTAs, per warp one of an entry cut between warps
  return kMaxCtas * 4 + (uint64_t)kMaxCtas * (2 + S::kWarps) * S::kSlot * 4;
}

template <int KIND, int DP, int MODE, int HALVES>
seedq_status launch(Args &p, int dev, cudaStream_t st) {
  using S = Shape<DP, MODE, HALVES>;
  static DeviceOnce once;
  p.chunk = (p.a.n_requests + S::kRequests - 1) / S::kRequests;
  constexpr size_t smem = ((sizeof(Table<S>) + 127) & ~127) + 128 + (size_t)S::kWarps * S::kStages * S::kStage;
  static_assert(smem + 6144 <= kSmemMax, "");
  const int rc = once.run(dev, [] {
    return (int)cudaFuncSetAttribute(k_attend<KIND, DP, MODE, HALVES>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  });
  if (rc) return cuda_fail((cudaError_t)rc);
  k_attend<KIND, DP, MODE, HALVES><<<p.ctas, S::kThreads, smem, st>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}
// f(DP, MODE) for a plan, the two as types.
template <typename F>
auto with_shape(const Plan &s, F f) {
  using std::integral_constant;
  if (s.dp == 64)
    return s.mode == 0   ? f(integral_constant<int, 64>(), integral_constant<int, 0>())
           : s.mode == 1 ? f(integral_constant<int, 64>(), integral_constant<int, 1>())
                         : f(integral_constant<int, 64>(), integral_constant<int, 2>());
  if (s.dp == 128)
    return s.mode == 0   ? f(integral_constant<int, 128>(), integral_constant<int, 0>())
           : s.mode == 1 ? f(integral_constant<int, 128>(), integral_constant<int, 1>())
                         : f(integral_constant<int, 128>(), integral_constant<int, 2>());
  return s.mode == 0 ? f(integral_constant<int, 256>(), integral_constant<int, 0>())
                     : f(integral_constant<int, 256>(), integral_constant<int, 1>());
}

bool aligned(const void *base, int32_t dtype, int64_t ts, int64_t hs) {
  const int64_t per = 16 / dtype_bytes(dtype);
  return (uintptr_t)base % 16 == 0 && ts % per == 0 && hs % per == 0;
}

seedq_status check(const seedq_kv_cache *c, int32_t n_heads, int32_t max_new) {
  const seedq_status st = kv_check(c);
  if (st != SEEDQ_OK) return st;
  if (n_heads < 1 || max_new < 1) return SEEDQ_ERR_INVALID_ARG;
  return n_heads % c->n_kv_heads ? SEEDQ_ERR_UNSUPPORTED : SEEDQ_OK;
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_kv_attend_workspace_bytes(const seedq_kv_cache *cache, int32_t n_heads, int32_t max_new) {
  if (check(cache, n_heads, max_new) != SEEDQ_OK) return 0;
  // The most that any number of new tokens up to max_new takes: tiles of 4 rows,
  // with more warps, take more than tiles of 8.
  uint64_t most = 0;
  Plan s = shape_for(cache, n_heads, 1);
  for (const int last = shape_for(cache, n_heads, max_new).mode; s.mode <= last; ++s.mode)
    most = std::max(most, with_shape(s, [](auto dp, auto mode) { return workspace_bytes<dp.value, mode.value>(); }));
  return most;
}

seedq_status seedq_kv_attend(const seedq_kv_cache *cache, const seedq_attend_args *args, void *cuda_stream) {
  if (!args) return SEEDQ_ERR_INVALID_ARG;
  const seedq_attend_args &a = *args;
  const seedq_status st = check(cache, a.n_heads, a.max_new);
  if (st != SEEDQ_OK) return st;
  if (a.n_requests < 1 || a.n_requests > SEEDQ_MAX_REQUESTS || a.n_tokens < 0 || a.n_tokens > INT32_MAX ||
      !dtype_ok(a.q_dtype) || !dtype_ok(a.out_dtype) || a.table_width < 1 || a.table_width > (1 << 20) ||
      a.table_width > a.table_stride || a.window < 0 || !isfinite(a.scale))
    return SEEDQ_ERR_INVALID_ARG;
  if (a.n_tokens == 0) return SEEDQ_OK;
  if (!a.q || !a.out || !a.seq_lens || !a.starts || !a.block_table || !a.workspace || (uintptr_t)a.workspace % 16 ||
      a.workspace_bytes < seedq_kv_attend_workspace_bytes(cache, a.n_heads, a.max_new))
    return SEEDQ_ERR_INVALID_ARG;
  if (a.n_tokens * (a.n_heads / cache->n_kv_heads) >= INT32_MAX - 31) return SEEDQ_ERR_UNSUPPORTED;  // rows are numbered in 32 bits
  Args p;
  p.c = *cache;
  p.a = a;
  p.group = a.n_heads / cache->n_kv_heads;
  p.group_shift = log2_of(p.group);
  p.gpp_shift = log2_of(cache->page_size / 16);
  p.q_bytes = dtype_bytes(a.q_dtype);
  p.q_vec = aligned(a.q, a.q_dtype, a.q_token_stride, a.q_head_stride);
  p.out_vec = aligned(a.out, a.out_dtype, a.out_token_stride, a.out_head_stride);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e);
  p.ctas = std::min(sms, kMaxCtas);
  p.ctas_inv = ~0ull / (uint64_t)p.ctas + 1;
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  return with_shape(shape_for(cache, a.n_heads, a.max_new), [&](auto dp, auto mode) {
    // One half of a q in 16 bits: 16 tokens of 32 heads on 8 over 32768 keys take 93
    // us, with both halves 102.  Rows of 4 carry both anyway.
    constexpr int kShort = mode.value == 0 ? 2 : 1;
    if (a.q_dtype == SEEDQ_F32)
      return cache->kind == SEEDQ_KV_INT8 ? launch<SEEDQ_KV_INT8, dp.value, mode.value, 2>(p, dev, stream)
                                          : launch<SEEDQ_KV_E4M3, dp.value, mode.value, 2>(p, dev, stream);
    return cache->kind == SEEDQ_KV_INT8 ? launch<SEEDQ_KV_INT8, dp.value, mode.value, kShort>(p, dev, stream)
                                        : launch<SEEDQ_KV_E4M3, dp.value, mode.value, kShort>(p, dev, stream);
  });
}

}  // extern "C"
