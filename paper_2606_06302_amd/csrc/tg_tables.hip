// Block tables and slot maps on the device: tg_reserve (Eq. 4, Sections 4.1 and
// 4.2.3 of arXiv 2606.06302) from lengths that are on the device, and the pool
// rows of one layer's entries.
//
// tg_reserve_device is three launches on one stream:
//   lengths  one thread per (request, layer, group) table: kv_len = ceil(r * N)
//            (one fp64 multiply, as on the host) of the group's heads, their
//            maximum, the table's pages; a sum and the errors of every workgroup
//   pages    the needed front of the free list copied and its ids checked, by
//            all workgroups alike: a table's pages are its share of that front,
//            whatever its length
//   offsets  every workgroup adds up the workgroups' sums before its own, then
//            scans its tables; or, after an error anywhere, writes zeros
// Every value is written by one workgroup and read only by later launches: no
// atomics, no order that the result could depend on.
#include <hip/hip_runtime.h>

#include "tg_internal.h"

namespace {

constexpr int kBlock = 256;
constexpr int kWaves = kBlock / 64;
constexpr int kCopyBlocks = 1024;    // most workgroups of the pages launch
constexpr int kCopyPerBlock = 4096;  // ids a workgroup copies before another one joins

struct TableParams {
  const int32_t* ctx_len;
  const int32_t* headroom;
  const double* ratio;
  const double* budget;
  const int32_t* group_of;
  const int32_t* free_pages;
  int64_t num_free, pool_pages, pt_capacity;
  int32_t* kv_len;
  int32_t* group_len;
  int64_t* pt_offsets;
  int32_t* pt_pages;
  int64_t* pages_needed;
  int32_t* status;
  int64_t* sums;        // [blocks] pages of a workgroup's tables
  int32_t* bad;         // [blocks] a workgroup met an invalid length, ratio or group
  int32_t* bad_page;    // [copy_blocks]
  int64_t tables;       // batch * L * G
  int32_t blocks, copy_blocks;
  int32_t L, H, G, P;
};

// Sum over a workgroup; every thread receives it.
__device__ int64_t block_sum(int64_t x, int64_t* sm) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor((long long)x, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x += sm[w];
  return x;
}

__device__ __forceinline__ int64_t table_pages(const TableParams& p, int64_t t, int32_t group_len) {
  const int b = (int)(t / ((int64_t)p.L * p.G));
  const int room = p.headroom ? max(p.headroom[b], 0) : 0;
  return ((int64_t)group_len + room + p.P - 1) / p.P;
}

__global__ void __launch_bounds__(kBlock) tg_table_lengths_kernel(TableParams p) {
  __shared__ int64_t sm[kWaves];
  const int64_t t = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  int64_t pages = 0;
  bool bad = false;
  if (t < p.tables) {
    const int g = (int)(t % p.G);
    const int64_t bl = t / p.G;
    const int l = (int)(bl % p.L), b = (int)(bl / p.L);
    const int n = p.ctx_len[b];
    bad = n < 1 || (p.headroom && p.headroom[b] < 0);
    int32_t longest = 0;
    for (int h = 0; h < p.H; ++h) {
      const int of = p.group_of[(int64_t)l * p.H + h];
      if (of < 0 || of >= p.G) bad = true;
      if (of != g) continue;
      const double r = p.ratio ? p.ratio[bl * p.H + h] : p.budget[(int64_t)l * p.H + h];
      const bool ok = r > 0.0 && r <= 1.0;   // false for NaN
      if (!ok) bad = true;
      const int32_t len = ok && n >= 1 ? (int32_t)ceil(r * (double)n) : 0;
      p.kv_len[bl * p.H + h] = len;
      longest = max(longest, len);
    }
    p.group_len[t] = longest;
    pages = table_pages(p, t, longest);
  }
  pages = block_sum(pages, sm);
  const int64_t any = block_sum(bad, sm);
  if (threadIdx.x == 0) {
    p.sums[blockIdx.x] = pages;
    p.bad[blockIdx.x] = any > 0;
  }
}

// What the lengths launch found: the sum of every workgroup's pages (and of
// those before `block`), whether any input was invalid.
struct Found {
  int64_t needed, before;
  bool bad;
};
__device__ Found found(const TableParams& p, int block, int64_t* sm) {
  int64_t all = 0, before = 0, bad = 0;
  for (int i = threadIdx.x; i < p.blocks; i += kBlock) {
    const int64_t s = p.sums[i];
    all += s;
    before += i < block ? s : 0;
    bad += p.bad[i];
  }
  Found f;
  f.needed = block_sum(all, sm);
  f.before = block_sum(before, sm);
  f.bad = block_sum(bad, sm) > 0;
  return f;
}

__global__ void __launch_bounds__(kBlock) tg_table_pages_kernel(TableParams p) {
  __shared__ int64_t sm[kWaves];
  const Found f = found(p, 0, sm);
  int64_t bad = 0;
  if (!f.bad && f.needed <= p.num_free && f.needed <= p.pt_capacity) {
    for (int64_t k = (int64_t)blockIdx.x * kBlock + threadIdx.x; k < f.needed; k += (int64_t)gridDim.x * kBlock) {
      const int32_t id = p.free_pages[k];
      if (id < 0 || id >= p.pool_pages) bad = 1;
      p.pt_pages[k] = id;
    }
  }
  bad = block_sum(bad, sm);
  if (threadIdx.x == 0) p.bad_page[blockIdx.x] = bad > 0;
}

__global__ void __launch_bounds__(kBlock) tg_table_offsets_kernel(TableParams p) {
  __shared__ int64_t sm[kWaves];
  const Found f = found(p, blockIdx.x, sm);
  int64_t bad_page = 0;
  for (int i = threadIdx.x; i < p.copy_blocks; i += kBlock) bad_page += p.bad_page[i];
  bad_page = block_sum(bad_page, sm);
  int32_t status = TG_OK;
  if (f.bad)
    status = TG_ERR_INVALID_ARG;
  else if (f.needed > p.num_free)
    status = TG_ERR_OUT_OF_PAGES;
  else if (f.needed > p.pt_capacity)
    status = TG_ERR_BUFFER_TOO_SMALL;
  else if (bad_page)
    status = TG_ERR_INVALID_ARG;
  const int64_t t = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  const int64_t pages = t < p.tables ? table_pages(p, t, p.group_len[t]) : 0;
  // inclusive sum over the workgroup
  int64_t x = pages;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)x, o);
    if ((int)(threadIdx.x & 63) >= o) x += y;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sm[threadIdx.x >> 6] = x;
  __syncthreads();
  x += f.before;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) x += sm[w];
  if (t < p.tables) p.pt_offsets[t] = status == TG_OK ? x - pages : 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.pt_offsets[p.tables] = status == TG_OK ? f.needed : 0;
    *p.pages_needed = f.needed;
    *p.status = status;
  }
}

struct MapParams {
  const int64_t* pt_offsets;
  const int32_t* pt_pages;
  const int32_t* group_of;
  const int32_t* slot_of;
  const int32_t* begin;
  const int32_t* len;
  int64_t* map;
  int32_t n, layer, L, H, G, Hp, P;
};

// Grid (ceil(n / kMapPerBlock), units): kMapPerBlock entries of one head.
constexpr int kMapPerBlock = 4 * kBlock;

__global__ void __launch_bounds__(kBlock) tg_slot_map_kernel(MapParams p) {
  const int64_t unit = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
  const int h = (int)(unit % p.H);
  const int64_t b = unit / p.H;
  const int64_t at = (b * p.L + p.layer) * p.H + h;
  const int64_t lh = (int64_t)p.layer * p.H + h;
  const int64_t t = (b * p.L + p.layer) * p.G + p.group_of[lh];
  const int64_t base = p.pt_offsets[t];
  const int64_t cap = (p.pt_offsets[t + 1] - base) * p.P;
  const int64_t first = p.begin ? p.begin[at] : 0;
  const int64_t end = p.len ? min<int64_t>(p.len[at], cap) : cap;
  const int slot = p.slot_of[lh];
  for (int q = 0; q < 4; ++q) {
    const int j = (int)blockIdx.x * kMapPerBlock + q * kBlock + threadIdx.x;
    if (j >= p.n) return;
    const int64_t e = first + j;
    int64_t row = -1;
    if (e >= 0 && e < end) {
      const int64_t page = p.pt_pages[base + e / p.P];
      row = (page * 2 * p.Hp + slot) * p.P + e % p.P;
    }
    p.map[unit * p.n + j] = row;
  }
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
  int64_t tables, blocks;
  size_t sums, bad, total;
};

Layout layout_of(const tg_geometry& g, int batch) {
  Layout l;
  l.tables = (int64_t)batch * g.num_layers * (g.num_kv_heads / g.heads_per_group);
  l.blocks = (l.tables + kBlock - 1) / kBlock;
  l.sums = align256((size_t)l.blocks * sizeof(int64_t));
  l.bad = align256((size_t)l.blocks * sizeof(int32_t));
  l.total = l.sums + l.bad + align256(kCopyBlocks * sizeof(int32_t));
  return l;
}

}  // namespace

extern "C" {

size_t tg_reserve_device_workspace_bytes(const tg_geometry* geom, int32_t batch) {
  if (tg::check_geometry(geom) != TG_OK || batch < 1) return 0;
  return layout_of(*geom, batch).total;
}

int32_t tg_reserve_device(const tg_reserve_device_args* a, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = tg::check_geometry(&g)) return rc;
  if (a->batch < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch must be >= 1");
  if (!a->ctx_len || !a->group_of || !a->kv_len || !a->group_len || !a->pt_offsets || !a->pages_needed || !a->status)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  if (!a->ratio && !a->budget) return tg::fail(TG_ERR_INVALID_ARG, "ratio and budget are both NULL");
  if (a->num_free < 0 || a->pool_pages < 0 || a->pt_capacity < 0) return tg::fail(TG_ERR_INVALID_ARG, "negative pool size");
  if (a->num_free > 0 && !a->free_pages) return tg::fail(TG_ERR_INVALID_ARG, "free_pages is NULL");
  if (a->pt_capacity > 0 && !a->pt_pages) return tg::fail(TG_ERR_INVALID_ARG, "pt_pages is NULL");
  const Layout l = layout_of(g, a->batch);
  if (l.blocks > INT32_MAX) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
  if (!a->workspace || a->workspace_bytes < l.total)
    return tg::fail(TG_ERR_BUFFER_TOO_SMALL, "workspace holds %zu bytes, need %zu", a->workspace_bytes, l.total);
  if (!tg::aligned16({a->workspace})) return tg::fail(TG_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
  TableParams p;
  p.ctx_len = a->ctx_len;
  p.headroom = a->headroom;
  p.ratio = a->ratio;
  p.budget = a->budget;
  p.group_of = a->group_of;
  p.free_pages = a->free_pages;
  p.num_free = a->num_free;
  p.pool_pages = a->pool_pages;
  p.pt_capacity = a->pt_capacity;
  p.kv_len = a->kv_len;
  p.group_len = a->group_len;
  p.pt_offsets = a->pt_offsets;
  p.pt_pages = a->pt_pages;
  p.pages_needed = a->pages_needed;
  p.status = a->status;
  char* ws = static_cast<char*>(a->workspace);
  p.sums = reinterpret_cast<int64_t*>(ws);
  p.bad = reinterpret_cast<int32_t*>(ws + l.sums);
  p.bad_page = reinterpret_cast<int32_t*>(ws + l.sums + l.bad);
  p.tables = l.tables;
  p.blocks = (int32_t)l.blocks;
  p.L = g.num_layers;
  p.H = g.num_kv_heads;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.P = g.page_size;
  const int64_t most = a->num_free < a->pt_capacity ? a->num_free : a->pt_capacity;   // ids that can be taken
  const int64_t copy = (most + kCopyPerBlock - 1) / kCopyPerBlock;
  p.copy_blocks = (int32_t)(copy < 1 ? 1 : copy > kCopyBlocks ? kCopyBlocks : copy);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  hipLaunchKernelGGL(tg_table_lengths_kernel, dim3((unsigned)l.blocks), dim3(kBlock), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "reserve launch failed: %s", hipGetErrorString(e));
  hipLaunchKernelGGL(tg_table_pages_kernel, dim3(p.copy_blocks), dim3(kBlock), 0, st, p);
  e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "reserve launch failed: %s", hipGetErrorString(e));
  hipLaunchKernelGGL(tg_table_offsets_kernel, dim3((unsigned)l.blocks), dim3(kBlock), 0, st, p);
  e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "reserve launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}

int32_t tg_slot_map(const tg_slot_map_args* a, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = tg::check_geometry(&g)) return rc;
  if (a->batch < 1 || a->n < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch and n must be >= 1");
  if (a->layer < 0 || a->layer >= g.num_layers) return tg::fail(TG_ERR_INVALID_ARG, "layer %d out of range", a->layer);
  if (!a->pt_offsets || !a->pt_pages || !a->group_of || !a->slot_of || !a->map)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  MapParams p;
  p.pt_offsets = a->pt_offsets;
  p.pt_pages = a->pt_pages;
  p.group_of = a->group_of;
  p.slot_of = a->slot_of;
  p.begin = a->begin;
  p.len = a->len;
  p.map = a->map;
  p.n = a->n;
  p.layer = a->layer;
  p.L = g.num_layers;
  p.H = g.num_kv_heads;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.Hp = g.heads_per_group;
  p.P = g.page_size;
  const int64_t across = ((int64_t)a->n + kMapPerBlock - 1) / kMapPerBlock;
  if (a->batch > 65535) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
  if (g.num_kv_heads > 65535) return tg::fail(TG_ERR_INVALID_ARG, "too many heads");
  hipLaunchKernelGGL(tg_slot_map_kernel, dim3((unsigned)across, (unsigned)g.num_kv_heads, (unsigned)a->batch), dim3(kBlock),
                     0, static_cast<hipStream_t>(hip_stream), p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "slot map launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}

}  // extern "C"
