// The pages of chosen beams (seedq_beam_reorder): a beam that goes on from another
// takes over its list of pages, full pages are shared, and the partly filled last
// one is copied for every child but the first.
//
// What the beams of a request share lies at the same place of their lists, so no
// page needs a count of its holders: page p at column c is kept if a beam that has
// children holds it there, and goes back to the stack once if none does.  Work is
// cut into tiles of 32 columns of a request, a warp each, a lane per column.  The
// first pass counts the pages that go back, a sum over the tiles gives each its
// place on the stack, and the second writes lists and stack; a row's old entries
// are read by the warp that writes the new ones, so lists may be changed in place.
//
// The copies are units of one head and tensor of one layer and page, dealt to all
// warps: of a second launch, or, where they are small, of the first.
//
// Measured: 4 requests of 4 beams of 600 tokens, 32 layers of 8 heads of 128, 8.4 us
// (the lists 6: launch, six dependent trips to memory and two barriers of the
// cluster); 32 requests of 8 beams, 8 layers, 22 us, of which the copies (67 MB) take
// 11 to 12 (5.8 TB/s).
#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "device_once.h"
#include "overlap.h"
#include "serve.cuh"

namespace cg = cooperative_groups;

namespace seedq {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32;
constexpr int kMaxBeams = SEEDQ_MAX_BEAMS;
constexpr int kMaxCluster = 8;  // one CTA takes 27.5 us instead of 21.8 for 32 requests of 8 beams
constexpr int kAtOnce = 8;      // rows of a tile under way
constexpr int kLayersAtOnce = 64;  // whose pointers go in a launch's parameters
// What may have to be copied, up to which the first launch does it: a fork of 2 small
// layers takes as long on the GPU (8 us) and 3 us less of the caller's time.
constexpr int64_t kFewBytes = 1 << 20;

// One copy: tokens [0, used) of page src to page dst.
struct alignas(16) Copy {
  int32_t src, dst, used, none;
};
struct Workspace {
  int32_t n, pad[3];
  Copy copy[1];  // one per row
};

struct PagesArgs {
  int32_t groups, beams, page, page_shift, width, capacity;
  int64_t table_stride, out_stride;
  const int32_t *parents, *seq_lens, *table, *free_count;
  int32_t *table_out, *free_pages, *seq_out, *status, *count_out;
  Workspace *work;
};

__device__ __forceinline__ int pages_of(int tokens, const PagesArgs &a) {  // tokens >= 0
  const uint32_t x = (uint32_t)tokens + (uint32_t)a.page - 1;
  return (int)(a.page_shift >= 0 ? x >> a.page_shift : x / (uint32_t)a.page);
}

struct CopyArgs {
  const Workspace *work;
  int32_t layers, heads, pieces;  // pieces of 16 codes of a token
  int64_t pages, page_stride, head_stride, token_stride;
  uint8_t *codes[kLayersAtOnce][2];
  float *scales[kLayersAtOnce][2];
};
constexpr int kCopyAhead = 8;  // loads of 16 bytes that a lane has under way (4: 23.7 us instead of 21.8, 16: 34)

// What warp `me` of `warps` copies of the first n entries of the list.
__device__ __forceinline__ void copy_pages(const CopyArgs &a, int n, int64_t me, int64_t warps) {
  const int lane = threadIdx.x & 31;
  const int of_copy = a.layers * 2 * a.heads;
  const int step = 32 / a.pieces, first = lane / a.pieces;  // tokens of a warp's step; the lane's
  const int64_t lane_at = first * a.token_stride + (lane - first * a.pieces) * 16, step_at = step * a.token_stride;
  const int64_t units = (int64_t)n * of_copy;
  for (int64_t u = me; u < units; u += warps) {
    const int c = (int)(u / of_copy), rest = (int)(u - (int64_t)c * of_copy), lt = rest / a.heads, h = rest - lt * a.heads;
    const int4 entry = __ldcg((const int4 *)(a.work->copy + c));
    const Copy y{entry.x, entry.y, entry.z, 0};
    if (y.src < 0 || y.src >= a.pages || y.dst < 0 || y.dst >= a.pages) continue;
    uint8_t *base = a.codes[lt >> 1][lt & 1] + h * a.head_stride + lane_at;
    const uint8_t *src = base + y.src * a.page_stride;
    uint8_t *dst = base + y.dst * a.page_stride;
    float *s = a.scales[lt >> 1][lt & 1];
    const float scale = lane == 0 ? s[(int64_t)y.src * a.heads + h] : 0.f;
    const int used = first < step ? y.used : 0;  // lanes that are left over copy nothing
    for (int t = first; t < used; t += kCopyAhead * step, src += kCopyAhead * step_at, dst += kCopyAhead * step_at) {
      uint4 v[kCopyAhead];
#pragma unroll
      for (int k = 0; k < kCopyAhead; ++k)
        if (t + k * step < used) v[k] = *(const uint4 *)(src + k * step_at);
#pragma unroll
      for (int k = 0; k < kCopyAhead; ++k)
        if (t + k * step < used) *(uint4 *)(dst + k * step_at) = v[k];
    }
    if (lane == 0) s[(int64_t)y.dst * a.heads + h] = scale;
  }
}

// Exclusive sums of v over the CTA, two at once, and the totals.
__device__ __forceinline__ int2 cta_sum(int2 v, int2 *warp_sums, int2 &total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int2 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(~0u, x.x, o), z = __shfl_up_sync(~0u, x.y, o);
    if (lane >= o) x.x += y, x.y += z;
  }
  if (lane == 31) warp_sums[w] = x;
  __syncthreads();
  int2 before = make_int2(0, 0);
  total = make_int2(0, 0);
#pragma unroll
  for (int k = 0; k < kWarps; ++k) {
    const int2 y = warp_sums[k];
    if (k < w) before.x += y.x, before.y += y.y;
    total.x += y.x, total.y += y.y;
  }
  __syncthreads();
  return make_int2(before.x + x.x - v.x, before.y + x.y - v.y);
}

// What the kernel keeps of a row: the row of its group that it goes on from (-1:
// none), its new length (-1: refused), its pages before, its place among the rows
// that want a copy (-1: none).
struct Rows {
  int *from, *len, *held, *nth, *first_tile;  // first_tile: per group, and their number
};

// COPY: the copies as well.
template <bool COPY>
__global__ void __launch_bounds__(kThreads) k_beam_pages(const __grid_constant__ PagesArgs a, const __grid_constant__ std::conditional_t<COPY, CopyArgs, char> y) {
  extern __shared__ int sm[];
  const int n = a.groups * a.beams, B = a.beams;
  const Rows r{sm, sm + n, sm + 2 * n, sm + 3 * n, sm + 4 * n};
  int *tiles = sm + 4 * n + a.groups + 1 + (threadIdx.x >> 5) * B * 32;  // the warp's tile
  __shared__ int2 s_warp[kWarps];
  __shared__ int s_back[kWarps], s_cta_back;
  const cg::cluster_group cluster = cg::this_cluster();
  const int rank = (int)cluster.block_rank(), ranks = (int)cluster.num_blocks();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  auto meet = [&]() {  // all CTAs of the cluster
    if (ranks == 1) __syncthreads();
    else cluster.sync();
  };
  if (!COPY) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int count = min(max(*a.free_count, 0), a.capacity);

  // rows: every CTA makes the same tables.  First as they are given.
  for (int i = threadIdx.x; i < n; i += kThreads) r.from[i] = a.parents[i], r.nth[i] = a.seq_lens[i];
  __syncthreads();
  auto pages_held = [&](int len) { return len < 0 || pages_of(len, a) > a.width ? -1 : pages_of(len, a); };  // -1: makes no sense
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int g0 = i / B * B, p = r.from[i], old = pages_held(r.nth[i]);
    const int from = p >= 0 && p < B ? r.nth[g0 + p] : 0;
    r.held[i] = max(old, 0);
    r.len[i] = p < -1 || p >= B || pages_held(from) < 0 ? -1 : p < 0 ? 0 : from;
  }
  __syncthreads();
  // The rows that want a copy: those with an earlier sibling and a partly filled page.
  // Tiles: as many of a group as its longest list has.
  int copies = 0, n_tiles = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    int2 mine = make_int2(0, 0), total;
    if (i < n) {
      const int g0 = i / B * B, p = r.from[i], len = r.len[i];
      if (len > 0 && len % a.page)
#pragma unroll 4
        for (int q = g0; q < i; ++q) mine.x |= r.from[q] == p;
      if (i < a.groups) {
        int most = 0;
#pragma unroll 4
        for (int b = 0; b < B; ++b) most = max(most, r.held[i * B + b]);
        mine.y = (most + 31) / 32;
      }
    }
    const int2 at = cta_sum(mine, s_warp, total);
    if (i < n) {
      r.nth[i] = mine.x ? copies + at.x : -1;
      if (i < a.groups) r.first_tile[i] = n_tiles + at.y;
    }
    copies += total.x, n_tiles += total.y;
  }
  for (int i = threadIdx.x; i < n; i += kThreads)
    if (r.len[i] < 0) r.from[i] = -1;  // refused: goes on from none
  if (threadIdx.x == 0) r.first_tile[a.groups] = n_tiles;
  __syncthreads();

  // The entry that the thread's row gets if no page comes back, on its way.
  const int my_row = rank * kThreads + threadIdx.x, my_nth = my_row < n ? r.nth[my_row] : -1;
  const int top = my_nth >= 0 && my_nth < count ? a.free_pages[count - 1 - my_nth] : -1;

  const int64_t workers = (int64_t)ranks * kWarps, me = (int64_t)rank * kWarps + w;
  const int t0 = (int)(n_tiles * me / workers), t1 = (int)(n_tiles * (me + 1) / workers);
  int g0 = 0;
  if (t0 < t1) {
    int lo = 0, hi = a.groups;  // last group with first_tile <= t0
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (r.first_tile[mid] <= t0) lo = mid;
      else hi = mid;
    }
    g0 = lo;
  }
  // Reads a tile; bit b of the result: row b's page at the lane's column goes back here.
  auto read_tile = [&](int g, int col) -> uint32_t {
    uint32_t held = 0, live = 0;
    int id[kAtOnce];
    for (int b0 = 0; b0 < B; b0 += kAtOnce) {
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int i = g * B + b0 + k;
        id[k] = b0 + k < B && col < r.held[i] ? a.table[(int64_t)i * a.table_stride + col] : -1;
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
        if (b0 + k < B) {
          tiles[(b0 + k) * 32 + lane] = id[k];
          if (id[k] >= 0) held |= 1u << (b0 + k);
          const int p = r.from[g * B + b0 + k];
          if (p >= 0) live |= 1u << p;
        }
    }
    uint32_t back = 0;
    if (B <= kAtOnce) {  // all in registers
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        uint32_t same = 0;
#pragma unroll
        for (int b = 0; b < kAtOnce; ++b) same |= (uint32_t)(id[b] == id[q]) << b;
        const bool stays = same & held & (live | ((1u << q) - 1));
        back |= (uint32_t)!stays << q;
      }
      return back & held & ~live;
    }
    for (uint32_t dead = held & ~live; dead; dead &= dead - 1) {
      const int q = __ffs(dead) - 1, id = tiles[q * 32 + lane];
      bool stays = false;
      for (uint32_t other = held & (live | ((1u << q) - 1)); other && !stays; other &= other - 1)
        stays = tiles[(__ffs(other) - 1) * 32 + lane] == id;
      if (!stays) back |= 1u << q;
    }
    return back;
  };

  int mine = 0;
  uint32_t back = 0;  // of the tile that was read last
  for (int t = t0, g = g0; t < t1; ++t) {
    while (t >= r.first_tile[g + 1]) ++g;
    back = read_tile(g, (t - r.first_tile[g]) * 32 + lane);
    mine += __popc(back);
  }
  mine = __reduce_add_sync(~0u, mine);
  if (lane == 0) s_back[w] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    int x = 0;
    for (int k = 0; k < kWarps; ++k) x += s_back[k];
    s_cta_back = x;
  }
  meet();
  const int of_rank = lane < ranks ? *cluster.map_shared_rank(&s_cta_back, lane) : 0;
  const int all = __reduce_add_sync(~0u, of_rank);
  const int before = __reduce_add_sync(~0u, (lane < rank ? of_rank : 0) + (lane < w ? s_back[lane] : 0));
  const int total = (int)min((int64_t)count + all, (int64_t)a.capacity);

  int place = count + before;
  for (int t = t0, g = g0; t < t1; ++t) {
    while (t >= r.first_tile[g + 1]) ++g;
    const int col = (t - r.first_tile[g]) * 32 + lane;
    if (t1 - t0 > 1) back = read_tile(g, col);
    int x = __popc(back);
    const int c = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(~0u, x, o);
      if (lane >= o) x += y;
    }
    int at = place + x - c;
    for (uint32_t rest = back; rest; rest &= rest - 1, ++at)
      if (at < a.capacity) a.free_pages[at] = tiles[(__ffs(rest) - 1) * 32 + lane];
    place += __shfl_sync(~0u, x, 31);
    for (int b = 0; b < B; ++b) {
      const int i = g * B + b, len = r.len[i], nth = r.nth[i];
      if (len <= 0 || nth >= total || col >= pages_of(len, a)) continue;
      const int id = tiles[r.from[i] * 32 + lane];
      if (nth >= 0 && col == pages_of(len, a) - 1) a.work->copy[nth].src = id;  // gets a page of its own
      else a.table_out[(int64_t)i * a.out_stride + col] = id;
    }
  }
  meet();  // the stack is whole, and no CTA's counts are read any more

  for (int i = rank * kThreads + threadIdx.x; i < n; i += ranks * kThreads) {
    const int len = r.len[i], nth = r.nth[i];
    const bool fits = nth < total;
    a.seq_out[i] = len > 0 && fits ? len : 0;
    a.status[i] = len < 0 ? SEEDQ_REQ_BAD : fits ? SEEDQ_REQ_OK : SEEDQ_REQ_NO_PAGES;
    if (nth >= 0 && fits) {
      const int dst = total == count && i == my_row ? top : __ldcg(a.free_pages + (total - 1 - nth));
      a.table_out[(int64_t)i * a.out_stride + pages_of(len, a) - 1] = dst;
      a.work->copy[nth].dst = dst;
      a.work->copy[nth].used = len % a.page;
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    a.work->n = min(copies, total);
    *a.count_out = total - min(copies, total);
  }
  if constexpr (COPY) {
    meet();  // the list is whole
    copy_pages(y, min(copies, total), me, workers);
  }
}

constexpr int kCopyThreads = 256, kCopyCtas = 4;  // per SM

__global__ void __launch_bounds__(kCopyThreads, kCopyCtas) k_beam_copy(const __grid_constant__ CopyArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // for the list of copies
  copy_pages(a, a.work->n, (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5), (int64_t)gridDim.x * (kCopyThreads / 32));
}

DeviceOnce g_pages_smem;

size_t pages_smem(int groups, int beams) {
  return sizeof(int) * ((size_t)4 * groups * beams + groups + 1 + (size_t)kWarps * beams * 32);
}

}  // namespace
}  // namespace seedq

using namespace seedq;

extern "C" {

uint64_t seedq_beam_reorder_workspace_bytes(int32_t n_groups, int32_t n_beams) {
  if (n_groups < 1 || n_beams < 1 || n_beams > kMaxBeams || (int64_t)n_groups * n_beams > SEEDQ_MAX_REQUESTS) return 0;
  return sizeof(Workspace) + (uint64_t)n_groups * n_beams * sizeof(Copy);
}

seedq_status seedq_beam_reorder(const seedq_kv_cache *caches, int32_t n_caches, const seedq_beam_reorder_args *args, void *cuda_stream) {
  if (!caches || !args || n_caches < 1 || n_caches > SEEDQ_BEAM_MAX_CACHES) return SEEDQ_ERR_INVALID_ARG;
  const seedq_kv_cache &c = caches[0];
  for (int i = 0; i < n_caches; ++i) {
    const seedq_kv_cache &x = caches[i];
    const seedq_status st = kv_check(&x);
    if (st != SEEDQ_OK) return st;
    if (x.n_kv_heads != c.n_kv_heads || x.head_dim != c.head_dim || x.page_size != c.page_size || x.n_pages != c.n_pages ||
        x.page_stride != c.page_stride || x.head_stride != c.head_stride || x.token_stride != c.token_stride)
      return SEEDQ_ERR_INVALID_ARG;
  }
  const seedq_beam_reorder_args &p = *args;
  const uint64_t bytes = seedq_beam_reorder_workspace_bytes(p.n_groups, p.n_beams);
  if (bytes == 0 || !p.parents || !p.seq_lens || !p.block_table || !p.table_out || !p.free_pages || !p.free_count || !p.seq_lens_out ||
      !p.status || !p.free_count_out || !p.workspace || (uintptr_t)p.workspace % 16 || p.workspace_bytes < bytes)
    return SEEDQ_ERR_INVALID_ARG;
  if (p.table_width < 1 || p.table_width > (1 << 20) || p.table_width > p.table_stride || p.table_width > p.out_stride ||
      p.free_capacity < c.n_pages || p.free_capacity == INT32_MAX)
    return SEEDQ_ERR_INVALID_ARG;
  if (p.table_out == p.block_table && p.out_stride != p.table_stride) return SEEDQ_ERR_INVALID_ARG;
  // What is read and what is written lie apart, but where one is the other: lengths, count and
  // a row's entries are read before they are written.
  const Wide n = (Wide)p.n_groups * p.n_beams;
  auto table = [&](const int32_t *t, int64_t stride) { return byte_rows(t, (Wide)p.table_width * 4, n, (Wide)stride * 4); };
  const ByteRows out[] = {byte_rows(p.seq_lens_out, n * 4), byte_rows(p.free_count_out, 4), table(p.table_out, p.out_stride),
                          byte_rows(p.status, n * 4), byte_rows(p.free_pages, (Wide)p.free_capacity * 4)};
  const ByteRows in[] = {byte_rows(p.seq_lens, n * 4), byte_rows(p.free_count, 4), table(p.block_table, p.table_stride), byte_rows(p.parents, n * 4)};
  for (int i = 0; i < 5; ++i) {
    for (int k = 0; k < 4; ++k)
      if (!(i == k && k < 3 && out[i].at == in[k].at) && overlap(out[i], in[k])) return SEEDQ_ERR_INVALID_ARG;
    for (int k = 0; k < i; ++k)
      if (overlap(out[i], out[k])) return SEEDQ_ERR_INVALID_ARG;
  }
  PagesArgs a{p.n_groups, p.n_beams, c.page_size, log2_of(c.page_size), p.table_width, p.free_capacity, p.table_stride, p.out_stride,
              p.parents, p.seq_lens, p.block_table, p.free_count, p.table_out, p.free_pages, p.seq_lens_out, p.status, p.free_count_out,
              (Workspace *)p.workspace};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  const int rc = g_pages_smem.run(dev, [] {
    const int most = (int)std::max(pages_smem(SEEDQ_MAX_REQUESTS, 1), pages_smem(SEEDQ_MAX_REQUESTS / kMaxBeams, kMaxBeams));
    const cudaError_t e = cudaFuncSetAttribute(k_beam_pages<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return (int)(e == cudaSuccess ? cudaFuncSetAttribute(k_beam_pages<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) : e);
  });
  if (rc) return cuda_fail((cudaError_t)rc);
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  const int64_t tiles = (int64_t)p.n_groups * ((p.table_width + 31) / 32);
  int ranks = 1;
  while (ranks < kMaxCluster && tiles > ranks * kWarps) ranks *= 2;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ranks, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  CopyArgs y{};
  y.work = a.work, y.heads = c.n_kv_heads, y.pieces = c.head_dim / 16, y.pages = c.n_pages;
  y.page_stride = c.page_stride, y.head_stride = c.head_stride, y.token_stride = c.token_stride;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ranks), cfg.blockDim = dim3(kThreads), cfg.dynamicSmemBytes = pages_smem(p.n_groups, p.n_beams);
  cfg.stream = st, cfg.attrs = &attr, cfg.numAttrs = ranks > 1;
  auto layers = [&](int first) {
    y.layers = std::min(n_caches - first, kLayersAtOnce);
    for (int i = 0; i < y.layers; ++i) {
      const seedq_kv_cache &x = caches[first + i];
      y.codes[i][0] = (uint8_t *)x.k, y.codes[i][1] = (uint8_t *)x.v;
      y.scales[i][0] = x.k_scale, y.scales[i][1] = x.v_scale;
    }
  };
  layers(0);
  const int64_t tensors = (int64_t)p.n_groups * p.n_beams * n_caches * 2 * y.heads;
  if (tensors * (c.page_size - 1) * c.head_dim <= kFewBytes && n_caches <= kLayersAtOnce) {
    e = cudaLaunchKernelEx(&cfg, k_beam_pages<true>, a, y);
    return e == cudaSuccess ? SEEDQ_OK : cuda_fail(e);
  }
  e = cudaLaunchKernelEx(&cfg, k_beam_pages<false>, a, char(0));
  if (e != cudaSuccess) return cuda_fail(e);
  for (int first = 0; first < n_caches; first += kLayersAtOnce) {
    if (first) layers(first);
    const int64_t most = (int64_t)p.n_groups * p.n_beams * y.layers * 2 * y.heads, per = kCopyThreads / 32;
    // Its CTAs may start while the pages are being handed out; they wait for that before they read.
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t copy{};
    copy.gridDim = dim3((unsigned)std::min<int64_t>((most + per - 1) / per, 152 * kCopyCtas));
    copy.blockDim = dim3(kCopyThreads), copy.stream = st, copy.attrs = &early, copy.numAttrs = 1;
    e = cudaLaunchKernelEx(&copy, k_beam_copy, y);
    if (e != cudaSuccess) return cuda_fail(e);
  }
  return SEEDQ_OK;
}

}  // extern "C"
