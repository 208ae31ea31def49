// Page bookkeeping of a step on the device: block tables, slot maps and the
// free stack from request lengths (seedq_batch_plan).
//
// With P tokens a page, request i of length L with n new tokens holds
// ceil(L / P) pages and wants ceil((L + n) / P).  Three exclusive sums over the
// requests give everything: of the new tokens (token offsets), of the pages
// that finished requests return (their places on the stack) and of the pages
// that the others need (the stack entries they pop).  All sums saturate, so
// lengths that make no sense cannot wrap an offset.
//
// A step moves a few kilobytes, so launch latency bounds it, and behind it the
// chain of lengths, two scans, searches and page numbers: 3.6 us for 16 requests
// with a token each, 6.3 us for 600 with up to 512 (2 to 2.5 us are an empty
// launch's).  Every CTA repeats the sums (8 bytes per request, from L2) instead of
// waiting for one that makes them, then takes its share of the tokens, of the
// table rows and of the pages to return; entries of the stack that this call
// itself pushes are found through the sums, not read back from memory another CTA
// may not have written.  512 threads: with 256 the larger case takes 7.9 us, with
// 1024 the smaller 4.2.
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "device_once.h"
#include "serve.cuh"

namespace seedq {
namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kSat = 0x7fffffff;

struct PlanArgs {
  const int32_t *seq_lens, *n_new, *free_count;
  int32_t *table, *free_pages;
  int64_t table_stride;
  int32_t n, page, page_shift, width, capacity, max_tokens;  // page_shift: log2 of page, -1 if it is no power of two
  int64_t *slots;
  int32_t *positions, *requests, *seq_out, *starts, *status, *count_out;
};

__device__ __forceinline__ int sat_add(int a, int b) {  // a, b >= 0
  return (int)min((uint32_t)a + (uint32_t)b, (uint32_t)kSat);
}

// Exclusive sums of v over the CTA (saturating), N at once, and the totals.
template <int N>
__device__ __forceinline__ void cta_scan(int (&v)[N], int (*warp_sums)[N], int (&total)[N]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int y = __shfl_up_sync(~0u, v[k], o);
      if (lane >= o) v[k] = sat_add(v[k], y);
    }
  if (lane == 31)
#pragma unroll
    for (int k = 0; k < N; ++k) warp_sums[w][k] = v[k];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    int x = lane < kWarps ? warp_sums[lane][k] : 0;  // every warp sums the warps' again: one latency
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
      const int y = __shfl_up_sync(~0u, x, o);
      if (lane >= o) x = sat_add(x, y);
    }
    total[k] = __shfl_sync(~0u, x, kWarps - 1);
    const int before = __shfl_sync(~0u, x, max(w - 1, 0)), excl = __shfl_up_sync(~0u, v[k], 1);
    v[k] = sat_add(w ? before : 0, lane ? excl : 0);
  }
  __syncthreads();
}

// For tokens >= 0; the sum is below 2^32.
__device__ __forceinline__ int pages_of(int tokens, const PlanArgs &a) {
  const uint32_t x = (uint32_t)tokens + (uint32_t)a.page - 1;
  return (int)(a.page_shift >= 0 ? x >> a.page_shift : x / (uint32_t)a.page);
}

// Last i in [0, n) with v[i] <= x (v ascending, v[0] <= x).
__device__ __forceinline__ int find_last(const int *v, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (v[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kThreads) k_batch_plan(const __grid_constant__ PlanArgs a) {
  extern __shared__ int sm[];
  int *start = sm;              // n + 1: token offsets
  int *back = sm + a.n + 1;     // n + 1: stack places of returned pages
  int *need = back + a.n + 1;   // n + 1: stack entries popped before
  int *state = need + a.n + 1;  // n: status, or -1 for a finished request
  __shared__ int warp_sums[kWarps][2], warp_need[kWarps][1];
  const int page = a.page;
  const int count = min(max(*a.free_count, 0), a.capacity);
  const int room = a.capacity - count;

  int tok0 = 0, back0 = 0;
  for (int base = 0; base < a.n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    int L = 0, m = 0, st = SEEDQ_REQ_OK, ret = 0;
    if (i < a.n) {
      L = a.seq_lens[i];
      m = a.n_new[i];
      const int64_t len = (int64_t)L + max(m, 0);
      if (m < -1 || L < 0 || len > kSat || pages_of((int)len, a) > a.width) st = SEEDQ_REQ_BAD;
      else if (m == -1) st = -1, ret = pages_of(L, a);
    }
    int sums[2] = {max(m, 0), ret}, total[2];
    cta_scan(sums, warp_sums, total);
    const int t = sat_add(tok0, sums[0]), b = sat_add(back0, sums[1]);
    tok0 = sat_add(tok0, total[0]);
    back0 = sat_add(back0, total[1]);
    if (i < a.n) {
      if (st == SEEDQ_REQ_OK && sat_add(t, max(m, 0)) > a.max_tokens) st = SEEDQ_REQ_NO_ROOM;
      if (st == -1 && sat_add(b, ret) > room) st = SEEDQ_REQ_NO_ROOM;
      start[i] = min(t, a.max_tokens);
      back[i] = min(b, room);
      state[i] = st;
    }
  }
  if (threadIdx.x == 0) start[a.n] = min(tok0, a.max_tokens), back[a.n] = min(back0, room);
  __syncthreads();
  // Pages on the stack after the returns: a prefix of the finished requests
  // fits, so what fits ends where the first that does not begins.
  __shared__ int s_returned, s_taken;
  if (threadIdx.x == 0) s_returned = back0 <= room ? back0 : 0, s_taken = 0;
  __syncthreads();
  if (back0 > room)
    for (int i = threadIdx.x; i < a.n; i += blockDim.x)
      if (state[i] == -1) atomicMax(&s_returned, back[i] + pages_of(a.seq_lens[i], a));
  __syncthreads();
  const int avail = count + s_returned;

  int need0 = 0;
  for (int base = 0; base < a.n; base += blockDim.x) {
    const int i = base + threadIdx.x;
    int want = 0;
    if (i < a.n && state[i] == SEEDQ_REQ_OK) {
      const int L = a.seq_lens[i];
      want = pages_of(L + a.n_new[i], a) - pages_of(L, a);
    }
    int sums[1] = {want}, total[1];
    cta_scan(sums, warp_need, total);
    const int t = sat_add(need0, sums[0]);
    need0 = sat_add(need0, total[0]);
    if (i < a.n) {
      need[i] = t;
      if (want > 0) {
        if (sat_add(t, want) > avail) state[i] = SEEDQ_REQ_NO_PAGES;
        else atomicMax(&s_taken, t + want);
      }
    }
  }
  __syncthreads();

  // A stack entry: below count it was there, above it this call returned it.
  auto stack = [&](int s) -> int {
    if (s < count) return a.free_pages[s];
    int r = find_last(back, a.n, s - count);
    while (r >= 0 && state[r] != -1) --r;  // zero-width entries between
    return r < 0 ? -1 : a.table[(int64_t)r * a.table_stride + (s - count - back[r])];
  };

  const int stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
  for (int i = first; i < a.n; i += stride) {
    const int L = a.seq_lens[i], m = a.n_new[i], st = state[i];
    a.starts[i] = start[i];
    a.status[i] = max(st, 0);
    a.seq_out[i] = st == -1 ? 0 : st == SEEDQ_REQ_OK ? L + m : L;
  }
  if (first == 0) {
    a.starts[a.n] = start[a.n];
    *a.count_out = avail - s_taken;
  }
  // Table rows and returned pages: a warp per request.
  const int lane = threadIdx.x & 31;
  for (int i = first >> 5; i < a.n; i += stride >> 5) {
    const int L = a.seq_lens[i], st = state[i];
    int32_t *row = a.table + (int64_t)i * a.table_stride;
    const int held = pages_of(max(L, 0), a);
    if (st == -1) {
      for (int c = lane; c < held; c += 32) a.free_pages[count + back[i] + c] = row[c];
    } else if (st == SEEDQ_REQ_OK) {
      const int want = pages_of(L + a.n_new[i], a) - held;
      for (int c = lane; c < want; c += 32) row[held + c] = stack(avail - 1 - need[i] - c);
    }
  }
  const int used = start[a.n];
  for (int t = first; t < a.max_tokens; t += stride) {
    int64_t slot = -1;
    int pos = 0, req = -1;
    if (t < used) {
      req = find_last(start, a.n, t);
      const int L = a.seq_lens[req], d = t - start[req];
      pos = (int)min((int64_t)L + d, (int64_t)kSat);
      if (state[req] == SEEDQ_REQ_OK) {
        const int pg = a.page_shift >= 0 ? pos >> a.page_shift : pos / page, held = pages_of(L, a);
        const int id = pg < held ? a.table[(int64_t)req * a.table_stride + pg] : stack(avail - 1 - need[req] - (pg - held));
        slot = (int64_t)id * page + (pos - pg * page);
      }
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
    a.requests[t] = req;
  }
}

DeviceOnce g_plan_smem;

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" seedq_status seedq_batch_plan(int32_t n_requests, const int32_t *seq_lens, const int32_t *n_new,
                                         int32_t page_size, int32_t *block_table, int64_t table_stride,
                                         int32_t table_width, int32_t *free_pages, int32_t free_capacity,
                                         const int32_t *free_count, int32_t max_tokens, int64_t *slots,
                                         int32_t *positions, int32_t *requests, int32_t *seq_lens_out,
                                         int32_t *starts, int32_t *status, int32_t *free_count_out,
                                         void *cuda_stream) {
  if (!seq_lens || !n_new || !block_table || !free_pages || !free_count || !slots || !positions || !requests ||
      !seq_lens_out || !starts || !status || !free_count_out)
    return SEEDQ_ERR_INVALID_ARG;
  if (n_requests < 1 || n_requests > SEEDQ_MAX_REQUESTS || max_tokens < 1 || max_tokens == INT32_MAX || page_size < 1 ||
      table_width < 1 || table_width > (1 << 20) || table_width > table_stride || free_capacity < 0 ||
      free_capacity == INT32_MAX)
    return SEEDQ_ERR_INVALID_ARG;
  // Other CTAs still read the inputs while the first ones write.
  for (const int32_t *o : {positions, requests, seq_lens_out, starts, status, free_count_out})
    if (o == seq_lens || o == n_new || o == free_count) return SEEDQ_ERR_INVALID_ARG;
  PlanArgs a{seq_lens, n_new, free_count, block_table, free_pages, table_stride, n_requests, page_size, log2_of(page_size), table_width,
             free_capacity, max_tokens, slots, positions, requests, seq_lens_out, starts, status, free_count_out};
  const size_t smem = sizeof(int) * (4 * (size_t)n_requests + 3);
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  const int rc = g_plan_smem.run(dev, [] {
    return (int)cudaFuncSetAttribute(k_batch_plan, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (int)(sizeof(int) * (4 * SEEDQ_MAX_REQUESTS + 3)));
  });
  if (rc) return cuda_fail((cudaError_t)rc);
  const int ctas = std::min(152, std::max((max_tokens + kThreads - 1) / kThreads, (n_requests * 32 + 4095) / 4096));
  k_batch_plan<<<ctas, kThreads, smem, (cudaStream_t)cuda_stream>>>(a);
  e = cudaGetLastError();
  return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
}
