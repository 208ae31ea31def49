// Attention of the newest tokens over the 8-bit paged cache (seedq_kv_attend).
//
// Mathematics.  With codes c^k, c^v and block scales s^k, s^v a query row q of
// a head gives
//   z_j = scale * s^k_j (q . c^k_j),  out = sum_j p_j s^v_j c^v_j / sum_j p_j,
//   p_j = 2^(log2(e) z_j - m),  m a running maximum,
// one pass over the keys.  Products run on the tensor cores as m16n8k16 binary16
// products with float32 sums: codes are exact in binary16, and q and the weights
// p_j s^v_j, which are not, are held as a high and a low half (22 bits).  A
// decode step has few rows (query heads that share a key-value head, times new
// tokens), so a tile carries 8 of them twice: the high halves in its rows 0-7,
// the low halves in rows 8-15.  Both lands in the same thread, which adds them;
// the second half costs no instruction.  Weights are taken relative to the
// largest block scale so far and scaled by 2^14, so binary16's range never cuts
// off more than 2^-39 of the largest.  Each step's products start from zero and
// are added to float32 registers, so a long context is not accumulated inside
// the tensor cores, which truncate.
//
// What bounds it: the bytes of the cache, 2 head_dim per key and key-value
// head.  At 8 rows a byte costs 16 operations, far below the balance, but every
// code has to be widened (about 1.4 instructions) and multiplied.
//
// Layout.  For keys, a product's column is a token and its inner index the head
// dim; the order of the inner index is free as long as q uses the same, so each
// lane takes 16 consecutive codes of one token (one 16-byte copy) and q's
// fragments are laid out to match.  For values the inner index is the token and
// a column a head dim, whose order is free again: lane (n, r) takes 16
// consecutive codes of its four tokens.  So every lane copies (cp.async,
// 16 bytes) exactly the codes it will multiply into a ring of its own in shared
// memory: no barrier, no bank conflict, any strides, and what is past a
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

#include "cp_async.cuh"
#include "device_once.h"
#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kMaxCtas = 152;      // one per SM
constexpr int kSmemMax = 227 * 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kWeight = 16384.f;  // weights are held times this

template <int DP, int RT>
struct Shape {
  static constexpr int kUnit = DP <= 128 ? 32 : 16;  // tokens of a unit
  static constexpr int kGroups = kUnit / 16;
  static constexpr int kRows = 8 * RT;
  static constexpr int kChunks = DP / 64;            // 64 head dims: 16 codes of 4 lanes
  static constexpr int kVB = DP >= 128 ? 16 : 8;     // bytes of a lane's value piece
  static constexpr int kVParts = DP / (8 * kVB);
  static constexpr int kTilesN = DP / 8;
  static constexpr int kKeyPieces = kGroups * 2 * kChunks;
  static constexpr int kValPieces = kGroups * 4 * kVParts;
  static constexpr int kValAt = kKeyPieces * 512;
  static constexpr int kMetaAt = kValAt + kValPieces * 32 * kVB;
  static constexpr int kStage = kMetaAt + 16 * kGroups;  // meta: per group both scales and a flag
  static constexpr int kSlot = kRows * (DP + 2);         // floats of a partial result: m, l, o
};

struct Args {
  seedq_kv_cache c;
  seedq_attend_args a;
  int32_t group;       // query heads per key-value head
  int32_t ctas, stages;
  int32_t q_vec, out_vec;  // q / out rows allow 16-byte accesses
};

__device__ __forceinline__ void cp_async16z(uint32_t dst, const void *src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8z(uint32_t dst, const void *src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(in ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_wait_n(int n) {  // at most n groups pending
  switch (n) {
    case 0: cp_async_wait<0>(); break;
    case 1: cp_async_wait<1>(); break;
    case 2: cp_async_wait<2>(); break;
    case 3: cp_async_wait<3>(); break;
    default: cp_async_wait<4>(); break;
  }
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t *>(&h); }

// x = hi + lo in binary16 (pairs).
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 f = __half22float2(h);
  hi = half2_bits(h);
  lo = half2_bits(__floats2half2_rn(x - f.x, y - f.y));
}

// Widen the codes in bytes (0, 1) and (2, 3) of w.  int8: byte + 128 placed
// under the exponent of 1024 is 1152 + code, exact.  E4M3: as code_value, less
// its factor 2^8 (see code_unit).
template <int KIND>
__device__ __forceinline__ uint32_t widen(uint32_t w, uint32_t sel) {
  if (KIND == SEEDQ_KV_INT8) {
    const uint32_t x = __byte_perm(w, 0x64646464u, sel);
    return half2_bits(__hsub2(*reinterpret_cast<const __half2 *>(&x), __float2half2_rn(1152.f)));
  }
  const uint32_t x = __byte_perm(w, 0u, sel);  // bytes to the top of each half
  return ((x >> 1) & 0x3f803f80u) | (x & 0x80008000u);
}
template <int KIND>
__device__ __forceinline__ uint32_t widen_lo(uint32_t w) { return widen<KIND>(w, KIND == SEEDQ_KV_INT8 ? 0x4140u : 0x1404u); }
template <int KIND>
__device__ __forceinline__ uint32_t widen_hi(uint32_t w) { return widen<KIND>(w, KIND == SEEDQ_KV_INT8 ? 0x4342u : 0x3424u); }
template <int KIND>
__device__ __forceinline__ uint32_t code_bias(uint32_t w) { return KIND == SEEDQ_KV_INT8 ? w ^ 0x80808080u : w; }
template <int KIND>
__device__ __forceinline__ constexpr float code_unit() { return KIND == SEEDQ_KV_INT8 ? 1.f : 256.f; }

// A request's share of the work list.
struct Req {
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
  const int64_t cap = (int64_t)p.a.table_width * p.c.page_size;
  r.hi = (int)min((int64_t)max(r.len, 0), cap);
  const int64_t lo = p.a.window > 0 ? (int64_t)r.len - r.fresh + 1 - p.a.window : 0;
  r.lo = (int)min(max(lo, (int64_t)0), (int64_t)r.hi);
  r.tiles = (int)(((int64_t)r.fresh * p.group + S::kRows - 1) / S::kRows);
  r.u0 = r.lo / S::kUnit;
  r.units = max((int)((r.hi + (int64_t)S::kUnit - 1) / S::kUnit) - r.u0, 1);
  return r;
}

// One entry of the work list: (request, key-value head, row tile).
struct Entry {
  Req r;
  int b, h, tile;
  int64_t begin, end;  // its units in the work list
};
template <typename S>
__device__ __forceinline__ Entry entry_at(const Args &p, const int64_t *pre, int64_t u) {
  Entry e;
  int lo = 0, hi = p.a.n_requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= u) lo = mid;
    else hi = mid;
  }
  e.b = lo;
  e.r = request<S>(p, lo);
  const int64_t k = (u - pre[lo]) / e.r.units;
  e.h = (int)(k / e.r.tiles);
  e.tile = (int)(k - (int64_t)e.h * e.r.tiles);
  e.begin = pre[lo] + k * e.r.units;
  e.end = e.begin + e.r.units;
  return e;
}

// Where row `row` of an entry's tile goes; false if it holds no query.
template <typename S>
__device__ __forceinline__ bool row_of(const Args &p, const Entry &e, int row, int64_t &token, int &head, int &pos) {
  const int r = e.tile * S::kRows + row, t = r / p.group;
  token = e.r.first + t;
  head = e.h * p.group + (r - t * p.group);
  pos = e.r.len - e.r.fresh + t;
  return t < e.r.fresh;
}

// Joins n partial results (each m, l per row in units of log2, then the rows'
// averages o) into `to`, or, if to is null, writes the entry's output.  Weights
// are l 2^m; averages, not sums, are kept, so nothing can overflow on the way.
// The parts are from[0..n-1], or, without `from`, the second slot of the CTA
// whose slots begin at from0 and the first slots of the n - 1 CTAs behind it.
template <typename S, int DP, bool GLOBAL>
__device__ void join(const Args &p, const Entry &e, int n, const float *const *from, const float *from0, int64_t step,
                     float *to, float *wts) {
  const int tid = threadIdx.x;
  auto part = [&](int i) -> const float * { return from ? from[i] : i == 0 ? from0 + S::kSlot : from0 + i * step; };
  auto get = [&](const float *x) { return GLOBAL ? __ldcg(x) : *x; };
  float *ms = wts + n * S::kRows, *ls = ms + S::kRows;
  if (tid < S::kRows) {
    float m = -CUDART_INF_F, l = 0.f;
    for (int i = 0; i < n; ++i) m = fmaxf(m, get(part(i) + tid));
    const float mu = m == -CUDART_INF_F ? 0.f : m;
    for (int i = 0; i < n; ++i) {
      const float w = get(part(i) + S::kRows + tid) * exp2_fast(get(part(i) + tid) - mu);
      wts[i * S::kRows + tid] = w;
      l += w;
    }
    ms[tid] = m;
    ls[tid] = l;
  }
  __syncthreads();
  for (int x = tid; x < S::kRows * DP; x += kThreads) {
    const int row = x / DP, d = x - row * DP;
    if (d >= p.c.head_dim) continue;
    float o = 0.f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float w = wts[i * S::kRows + row], v = get(part(i) + 2 * S::kRows + x);
      o += w == 0.f ? 0.f : w * v;
    }
    const float l = ls[row];
    o = l == 0.f ? 0.f : o / l;
    if (to) {
      to[2 * S::kRows + x] = o;
    } else {
      int64_t token;
      int head, pos;
      if (row_of<S>(p, e, row, token, head, pos))
        store_elem(p.a.out, p.a.out_dtype, token * p.a.out_token_stride + head * p.a.out_head_stride + d, o);
    }
  }
  if (tid < S::kRows) {
    if (to) {
      to[tid] = ms[tid];
      to[S::kRows + tid] = ls[tid];
    } else if (p.a.lse) {
      int64_t token;
      int head, pos;
      if (row_of<S>(p, e, tid, token, head, pos)) {
        const float l = ls[tid];
        p.a.lse[token * p.a.n_heads + head] = l == 0.f ? -CUDART_INF_F : (ms[tid] + log2f(l)) * kLn2;
      }
    }
  }
  __syncthreads();
}

template <int KIND, int DP, int RT>
__global__ void __launch_bounds__(kThreads, 1) k_attend(const __grid_constant__ Args p) {
  using S = Shape<DP, RT>;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int nn = lane >> 2, q4 = lane & 3;
  const int B = p.a.n_requests, D = p.c.head_dim;

  // ---- the work list: exclusive sums of the requests' units
  int64_t *pre = (int64_t *)smem;
  __shared__ int64_t s_sums[kWarps];
  {
    int64_t base = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
      const int b = b0 + tid;
      int64_t u = 0;
      if (b < B) {
        const Req r = request<S>(p, b);
        u = r.fresh ? (int64_t)r.units * r.tiles * p.c.n_kv_heads : 0;
      }
      int64_t x = u;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(~0u, x, o);
        if (lane >= o) x += y;
      }
      if (lane == 31) s_sums[w] = x;
      __syncthreads();
      int64_t before = base;
      for (int i = 0; i < kWarps; ++i) {
        if (i < w) before += s_sums[i];
        base += s_sums[i];
      }
      if (b < B) pre[b] = before + x - u;
      __syncthreads();
    }
    if (tid == 0) pre[B] = base;
  }
  __syncthreads();
  const int64_t total = pre[B];
  // Units per CTA: even shares, but at least one unit per warp, so that a short
  // context is joined within few CTAs.
  const int64_t share = max((total + p.ctas - 1) / p.ctas, (int64_t)kWarps);
  const int64_t c0 = min(share * blockIdx.x, total), c1 = min(c0 + share, total);
  if (c0 >= c1) return;
  const int64_t w0 = c0 + (c1 - c0) * w / kWarps, w1 = c0 + (c1 - c0) * (w + 1) / kWarps;

  const int ring_at = ((B + 1) * 8 + 15) & ~15;
  uint8_t *ring = smem + ring_at + (size_t)w * p.stages * S::kStage;
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  float *ws = (float *)((uint8_t *)p.a.workspace + kMaxCtas * 4);
  float *cta_slots = ws + (size_t)blockIdx.x * 2 * S::kSlot;
  float *head_slot = ws + (size_t)kMaxCtas * 2 * S::kSlot + ((size_t)blockIdx.x * kWarps + w) * S::kSlot;
  // Parts of cut entries, in the order of their keys: [2 w] a warp's first
  // entry if more follow, [2 w + 1] its last.
  __shared__ const float *s_part[2 * kWarps];
  __shared__ int64_t s_begin[2 * kWarps];
  if (lane == 0) s_begin[2 * w] = s_begin[2 * w + 1] = -1;

  // ---- copies
  const int gpp = p.c.page_size >> 4;  // groups of 16 tokens per page
  Entry pe;                            // the entry being copied
  int64_t pu = w0;                     // next unit to copy
  int pgb = 0, ids = -1, ids_next = -1, pstage = 0, stage = 0;
  const int32_t *prow = nullptr;
  pe.end = w0;
  auto load_ids = [&](int g) -> int {  // page of group g + lane of the entry being copied
    const int64_t gl = (int64_t)g + lane;
    return gl * 16 < pe.r.hi ? __ldg(prow + gl / gpp) : -1;
  };
  auto issue = [&]() {
    if (pu < w1) {
      if (pu >= pe.end) {
        pe = entry_at<S>(p, pre, pu);
        prow = p.a.block_table + (int64_t)pe.b * p.a.table_stride;
        pgb = (pe.r.u0 + (int)(pu - pe.begin)) * S::kGroups;
        ids = load_ids(pgb);
        ids_next = load_ids(pgb + 32);
      }
      const uint32_t dst = ring_s + pstage * S::kStage;
      pstage = pstage + 1 == p.stages ? 0 : pstage + 1;
      const int g0 = (pe.r.u0 + (int)(pu - pe.begin)) * S::kGroups;
      if (g0 - pgb >= 32) {
        pgb += 32;
        ids = ids_next;
        ids_next = load_ids(pgb + 32);
      }
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
        const int gi = g0 + g, page = __shfl_sync(~0u, ids, gi - pgb);
        const int t0 = gi * 16;
        const bool in = page >= 0 && page < p.c.n_pages && t0 + 16 > pe.r.lo;  // ids is -1 past hi
        const int left = in ? pe.r.hi - t0 : 0;                                // tokens of the group that exist
        const int64_t at = in ? page * p.c.page_stride + pe.h * p.c.head_stride + (int64_t)(gi % gpp) * 16 * p.c.token_stride : 0;
        const uint8_t *kp = (const uint8_t *)p.c.k + at, *vp = (const uint8_t *)p.c.v + at;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int c = 0; c < S::kChunks; ++c) {
            const int j = t * 8 + nn, d = c * 64 + q4 * 16;
            const bool ok = j < left && d < D;
            cp_async16z(dst + ((g * 2 + t) * S::kChunks + c) * 512 + lane * 16, ok ? kp + j * p.c.token_stride + d : (const uint8_t *)p.c.k, ok);
          }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int c = 0; c < S::kVParts; ++c) {
            const int j = (t >> 1) * 8 + q4 * 2 + (t & 1), d = c * 128 + nn * S::kVB;
            const bool ok = j < left && d < D;
            const uint32_t to = dst + S::kValAt + ((g * 4 + t) * S::kVParts + c) * (32 * S::kVB) + lane * S::kVB;
            const uint8_t *src = ok ? vp + j * p.c.token_stride + d : (const uint8_t *)p.c.v;
            if (S::kVB == 16) cp_async16z(to, src, ok);
            else cp_async8z(to, src, ok);
          }
        const uint32_t meta = dst + S::kMetaAt + g * 16;
        if (lane < 2) {
          if (in) {
            const float *sc = (lane ? p.c.v_scale : p.c.k_scale) + (int64_t)page * p.c.n_kv_heads + pe.h;
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(meta + lane * 4), "l"(sc) : "memory");
          } else {
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(meta + lane * 4), "f"(0.f) : "memory");
          }
        } else if (lane == 2) {
          asm volatile("st.shared.s32 [%0], %1;" ::"r"(meta + 8), "r"(in ? 1 : 0) : "memory");
        }
      }
      ++pu;
    }
    cp_async_commit();
  };
  for (int i = 0; i < p.stages - 1; ++i) issue();

  // ---- products
  uint32_t qf[RT][S::kChunks * 4][4];  // q as the products' first operand: high and low halves
  float zf[RT];                        // z in units of log2 per unit of product, but for the key scale
  int pos[RT];                         // the rows' positions
  float o[RT][S::kTilesN][2];
  float m[RT], l[RT], vmax = 0.f;
  Entry e;
  e.end = w0;
  int pos_first = 0, pos_last = 0;

  for (int64_t u = w0; u < w1; ++u) {
    if (u >= e.end) {  // a new entry: its queries
      e = entry_at<S>(p, pre, u);
      vmax = 0.f;
      pos_first = e.r.len - e.r.fresh + (e.tile * S::kRows) / p.group;
      pos_last = min(e.r.len - e.r.fresh + (e.tile * S::kRows + S::kRows - 1) / p.group, e.r.len - 1);
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        m[i] = -CUDART_INF_F;
        l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < S::kTilesN; ++j) o[i][j][0] = o[i][j][1] = 0.f;
        int64_t token;
        int head;
        const bool real = row_of<S>(p, e, i * 8 + nn, token, head, pos[i]);
        const int64_t at = real ? token * p.a.q_token_stride + head * p.a.q_head_stride : 0;
        float x[S::kChunks * 16], amax = 0.f;
#pragma unroll
        for (int c = 0; c < S::kChunks; ++c) {
          const int d = c * 64 + q4 * 16;
          if (!real || d >= D) {
#pragma unroll
            for (int k = 0; k < 16; ++k) x[c * 16 + k] = 0.f;
          } else if (p.q_vec && p.a.q_dtype == SEEDQ_F32) {
            const float4 *src = (const float4 *)((const float *)p.a.q + at + d);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float4 f = __ldg(src + k);
              x[c * 16 + k * 4] = f.x, x[c * 16 + k * 4 + 1] = f.y, x[c * 16 + k * 4 + 2] = f.z, x[c * 16 + k * 4 + 3] = f.w;
            }
          } else if (p.q_vec) {
            const uint4 *src = (const uint4 *)((const uint16_t *)p.a.q + at + d);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint4 f = __ldg(src + k);
              const uint32_t v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                float2 g;
                if (p.a.q_dtype == SEEDQ_BF16) g = make_float2(__uint_as_float(v[y] << 16), __uint_as_float(v[y] & 0xffff0000u));
                else g = __half22float2(*reinterpret_cast<const __half2 *>(&v[y]));
                x[c * 16 + k * 8 + y * 2] = g.x;
                x[c * 16 + k * 8 + y * 2 + 1] = g.y;
              }
            }
          } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) x[c * 16 + k] = load_elem(p.a.q, p.a.q_dtype, at + d + k);
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) amax = fmaxf(amax, fabsf(x[c * 16 + k]));
        }
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
        // The row times a power of two, its largest number in [2^13, 2^14).
        int ex = amax > 0.f && amax < CUDART_INF_F ? 13 + 127 - (int)(__float_as_uint(amax) >> 23) : 0;
        ex = min(max(ex, -126), 126);
        const float up = __uint_as_float((uint32_t)(127 + ex) << 23);
        zf[i] = p.a.scale * kLog2e * code_unit<KIND>() * __uint_as_float((uint32_t)(127 - ex) << 23);
#pragma unroll
        for (int k = 0; k < S::kChunks * 4; ++k) {
          split2(x[k * 4] * up, x[k * 4 + 1] * up, qf[i][k][0], qf[i][k][1]);
          split2(x[k * 4 + 2] * up, x[k * 4 + 3] * up, qf[i][k][2], qf[i][k][3]);
        }
      }
    }

    __syncwarp();  // all lanes are done with the stage that is filled next
    issue();
    cp_async_wait_n(p.stages - 1);
    __syncwarp();
    const uint8_t *st = ring + stage * S::kStage;
    stage = stage + 1 == p.stages ? 0 : stage + 1;
    float ks[S::kGroups], vs[S::kGroups];
    bool all_in = true;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) {
      const float *meta = (const float *)(st + S::kMetaAt + g * 16);
      ks[g] = meta[0];
      vs[g] = meta[1];
      all_in = all_in && ((const int *)meta)[2];
    }

    // scores: a tile of 8 tokens per column block
    float z[RT][S::kGroups * 2][2];
#pragma unroll
    for (int t = 0; t < S::kGroups * 2; ++t) {
      float acc[RT][4];
#pragma unroll
      for (int i = 0; i < RT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
      for (int c = 0; c < S::kChunks; ++c) {
        const uint4 kw = *(const uint4 *)(st + (t * S::kChunks + c) * 512 + lane * 16);
        const uint32_t v[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint32_t cw = code_bias<KIND>(v[y]);
          const uint32_t b0 = widen_lo<KIND>(cw), b1 = widen_hi<KIND>(cw);
#pragma unroll
          for (int i = 0; i < RT; ++i) mma(acc[i], qf[i][c * 4 + y], b0, b1);
        }
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        const float f = zf[i] * ks[t >> 1];
        z[i][t][0] = (acc[i][0] + acc[i][2]) * f;
        z[i][t][1] = (acc[i][1] + acc[i][3]) * f;
      }
    }

    const int j0 = (e.r.u0 + (int)(u - e.begin)) * S::kUnit;
    const bool masked = !all_in || j0 + S::kUnit - 1 > min(pos_first, e.r.hi - 1) || (p.a.window > 0 && j0 <= pos_last - p.a.window);
    if (masked) {
#pragma unroll
      for (int t = 0; t < S::kGroups * 2; ++t) {
        const bool in = ((const int *)(st + S::kMetaAt + (t >> 1) * 16))[2];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int j = j0 + t * 8 + q4 * 2 + k;
            if (!in || j > pos[i] || j >= e.r.hi || (p.a.window > 0 && j <= pos[i] - p.a.window)) z[i][t][k] = -CUDART_INF_F;
          }
      }
    }

    // the block scales of the values, relative to the largest so far
    float vnew = vmax, vr[S::kGroups], vcorr = 1.f;
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g)
      if (fabsf(vs[g]) < CUDART_INF_F) vnew = fmaxf(vnew, fabsf(vs[g]));
#pragma unroll
    for (int g = 0; g < S::kGroups; ++g) vr[g] = vs[g] == vnew ? (vnew > 0.f ? kWeight : 0.f) : __fdiv_rn(vs[g], vnew) * kWeight;
    if (vnew != vmax) vcorr = __fdiv_rn(vmax, vnew);
    vmax = vnew;

    uint32_t pf[RT][S::kGroups][4];
    float corr[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      float mx = m[i];
#pragma unroll
      for (int t = 0; t < S::kGroups * 2; ++t) mx = fmaxf(mx, fmaxf(z[i][t][0], z[i][t][1]));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
      mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
      const float mu = mx == -CUDART_INF_F ? 0.f : mx;
      const float cr = exp2_fast(m[i] - mu);
      m[i] = mx;
      float sum = 0.f;
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g) {
        float wt[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float pr = exp2_fast(z[i][g * 2 + (k >> 1)][k & 1] - mu);
          sum += pr;
          wt[k] = pr * vr[g];
          if (masked && z[i][g * 2 + (k >> 1)][k & 1] == -CUDART_INF_F) wt[k] = 0.f;  // 0, whatever the scale is
        }
        split2(wt[0], wt[1], pf[i][g][0], pf[i][g][1]);
        split2(wt[2], wt[3], pf[i][g][2], pf[i][g][3]);
      }
      l[i] = l[i] * cr + sum;
      corr[i] = cr * vcorr;
    }

#pragma unroll
    for (int part = 0; part < S::kVParts; ++part) {
      uint32_t vw[S::kGroups][4][S::kVB / 4];
#pragma unroll
      for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint8_t *src = st + S::kValAt + ((g * 4 + t) * S::kVParts + part) * (32 * S::kVB) + lane * S::kVB;
          if (S::kVB == 16) {
            const uint4 x = *(const uint4 *)src;
            vw[g][t][0] = x.x, vw[g][t][1] = x.y, vw[g][t][2 % (S::kVB / 4)] = x.z, vw[g][t][3 % (S::kVB / 4)] = x.w;
          } else {
            const uint2 x = *(const uint2 *)src;
            vw[g][t][0] = x.x, vw[g][t][1] = x.y;
          }
        }
#pragma unroll
      for (int y = 0; y < S::kVB / 4; ++y) {
        uint32_t b[S::kGroups][4][2];
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g)
#pragma unroll
          for (int k = 0; k < 2; ++k) {  // the pairs (2r, 2r + 1) and (2r + 8, 2r + 9) of tokens
            const uint32_t x = code_bias<KIND>(vw[g][2 * k][y]), xx = code_bias<KIND>(vw[g][2 * k + 1][y]);
            const uint32_t lo = __byte_perm(x, xx, 0x5140), hi = __byte_perm(x, xx, 0x7362);
            b[g][0][k] = widen_lo<KIND>(lo);
            b[g][1][k] = widen_hi<KIND>(lo);
            b[g][2][k] = widen_lo<KIND>(hi);
            b[g][3][k] = widen_hi<KIND>(hi);
          }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = part * S::kVB + y * 4 + k;
#pragma unroll
          for (int i = 0; i < RT; ++i) {
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int g = 0; g < S::kGroups; ++g) mma(acc, pf[i][g], b[g][k][0], b[g][k][1]);
            o[i][j][0] = fmaf(o[i][j][0], corr[i], acc[0] + acc[2]);
            o[i][j][1] = fmaf(o[i][j][1], corr[i], acc[1] + acc[3]);
          }
        }
      }
    }

    // ---- the end of this warp's part of an entry
    if (u + 1 == e.end || u + 1 == w1) {
      const bool whole = e.begin >= w0 && e.end <= w1;
      const bool last = u + 1 == w1;
      float *part = last ? (float *)ring : head_slot;
      if (!whole) {
        if (last) cp_async_wait<0>();  // nothing of this warp is still on its way into the ring
        __syncwarp();
        if (lane == 0) {
          s_part[2 * w + (last ? 1 : 0)] = part;
          s_begin[2 * w + (last ? 1 : 0)] = e.begin;
        }
      }
#pragma unroll
      for (int i = 0; i < RT; ++i) {
        float sum = l[i];
        sum += __shfl_xor_sync(~0u, sum, 1);
        sum += __shfl_xor_sync(~0u, sum, 2);
        // o / l first: the average code is small, the block scale may not be
        const float inv = sum == 0.f ? 0.f : __fdiv_rn(code_unit<KIND>() / kWeight, sum);
        const int row = i * 8 + nn;
        if (!whole) {
          if (q4 == 0) part[row] = m[i], part[S::kRows + row] = sum;
          float *dst = part + 2 * S::kRows + row * DP;
#pragma unroll
          for (int j = 0; j < S::kTilesN; ++j) {
            const int base = (j / S::kVB) * 128 + j % S::kVB;
            dst[base + (2 * q4) * S::kVB] = o[i][j][0] * inv * vmax;
            dst[base + (2 * q4 + 1) * S::kVB] = o[i][j][1] * inv * vmax;
          }
        } else {
          int64_t token;
          int head, ps;
          if (row_of<S>(p, e, row, token, head, ps)) {
            const int64_t at = token * p.a.out_token_stride + head * p.a.out_head_stride;
#pragma unroll
            for (int j = 0; j < S::kTilesN; ++j) {
              const int d = (j / S::kVB) * 128 + (2 * q4) * S::kVB + j % S::kVB;
              if (d < D) store_elem(p.a.out, p.a.out_dtype, at + d, o[i][j][0] * inv * vmax);
              if (d + S::kVB < D) store_elem(p.a.out, p.a.out_dtype, at + d + S::kVB, o[i][j][1] * inv * vmax);
            }
            if (p.a.lse && q4 == 0)
              p.a.lse[token * p.a.n_heads + head] = sum == 0.f ? -CUDART_INF_F : (m[i] + log2f(sum)) * kLn2;
          }
        }
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();

  // ---- entries cut between warps of this CTA
  __shared__ const float *s_from[2 * kWarps];
  float *wts = (float *)(smem + ring_at + (size_t)kWarps * p.stages * S::kStage);
  int64_t cross[2] = {-1, -1};  // entries cut between CTAs: the one that came from before, the one that goes on
  for (int i = 0; i < 2 * kWarps;) {
    const int64_t begin = s_begin[i];
    if (begin < 0) {
      ++i;
      continue;
    }
    int n = 0;
    __syncthreads();
    for (; i < 2 * kWarps && (s_begin[i] == begin || s_begin[i] < 0); ++i)
      if (s_begin[i] >= 0) {
        if (tid == 0) s_from[n] = s_part[i];
        ++n;
      }
    __syncthreads();
    e = entry_at<S>(p, pre, begin);
    const bool whole = e.begin >= c0 && e.end <= c1;
    const int side = e.begin < c0 ? 0 : 1;
    join<S, DP, false>(p, e, n, s_from, nullptr, 0, whole ? nullptr : cta_slots + side * S::kSlot, wts);
    if (!whole) cross[side] = begin;
  }

  // ---- entries cut between CTAs: the last to arrive joins
  int *counters = (int *)p.a.workspace;
  __shared__ int s_last;
  for (int side = 0; side < 2; ++side) {
    if (cross[side] < 0) continue;
    e = entry_at<S>(p, pre, cross[side]);
    const int first = (int)(e.begin / share), last = (int)((e.end - 1) / share);
    __threadfence();
    __syncthreads();
    if (tid == 0) {
      const int seen = atomicAdd(counters + first, 1);
      s_last = seen == last - first;
      if (s_last) counters[first] = 0;
    }
    __syncthreads();
    if (!s_last) continue;
    __threadfence();
    const int n = last - first + 1;
    // the first CTA's part is its second slot, the others' their first
    const float *from0 = ws + (size_t)first * 2 * S::kSlot;
    join<S, DP, true>(p, e, n, nullptr, from0, 2 * S::kSlot, nullptr, wts);
  }
}

struct Plan {
  int dp, rt, rows;
};
Plan shape_for(const seedq_kv_cache *c, int32_t n_heads, int32_t max_new) {
  Plan s;
  s.dp = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256;
  const int64_t rows = (int64_t)(n_heads / c->n_kv_heads) * max_new;
  s.rt = rows > 8 && s.dp < 256 ? 2 : 1;
  s.rows = 8 * s.rt;
  return s;
}

template <int KIND, int DP, int RT>
seedq_status launch(Args &p, DeviceOnce &once, int dev, cudaStream_t st) {
  using S = Shape<DP, RT>;
  const size_t pre = (((size_t)p.a.n_requests + 1) * 8 + 15) & ~(size_t)15;
  const size_t wts = (size_t)(kMaxCtas + 2) * S::kRows * 4;  // weights of a join of every CTA's part
  const size_t room = kSmemMax - 1024 - pre - wts;
  p.stages = (int)std::min<size_t>(5, room / ((size_t)kWarps * S::kStage));
  if (p.stages < 2) return SEEDQ_ERR_UNSUPPORTED;
  const size_t smem = pre + wts + (size_t)kWarps * p.stages * S::kStage;
  const int rc = once.run(dev, [] {
    return (int)cudaFuncSetAttribute(k_attend<KIND, DP, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax - 1024);
  });
  if (rc) return cuda_fail((cudaError_t)rc);
  k_attend<KIND, DP, RT><<<p.ctas, kThreads, smem, st>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}
template <int KIND>
seedq_status launch_kind(Args &p, const Plan &s, DeviceOnce *once, int dev, cudaStream_t st) {
  if (s.dp == 64) return s.rt == 1 ? launch<KIND, 64, 1>(p, once[0], dev, st) : launch<KIND, 64, 2>(p, once[1], dev, st);
  if (s.dp == 128) return s.rt == 1 ? launch<KIND, 128, 1>(p, once[2], dev, st) : launch<KIND, 128, 2>(p, once[3], dev, st);
  return launch<KIND, 256, 1>(p, once[4], dev, st);
}
DeviceOnce g_once[2][5];

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
  const Plan s = shape_for(cache, n_heads, max_new);
  // arrival counters; per CTA two parts of entries cut between CTAs, per warp one of an entry cut between warps
  return kMaxCtas * 4 + (uint64_t)kMaxCtas * (2 + kWarps) * s.rows * (s.dp + 2) * 4;
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
  Args p;
  p.c = *cache;
  p.a = a;
  p.group = a.n_heads / cache->n_kv_heads;
  p.q_vec = aligned(a.q, a.q_dtype, a.q_token_stride, a.q_head_stride);
  p.out_vec = aligned(a.out, a.out_dtype, a.out_token_stride, a.out_head_stride);
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return cuda_fail(e);
  p.ctas = std::min(sms, kMaxCtas);
  const Plan s = shape_for(cache, a.n_heads, a.max_new);
  const cudaStream_t stream = (cudaStream_t)cuda_stream;
  if (cache->kind == SEEDQ_KV_INT8) return launch_kind<SEEDQ_KV_INT8>(p, s, g_once[0], dev, stream);
  return launch_kind<SEEDQ_KV_E4M3>(p, s, g_once[1], dev, stream);
}

}  // extern "C"
