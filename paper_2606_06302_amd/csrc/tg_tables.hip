// Block tables and slot maps on the device: tg_reserve (Eq. 4, Sections 4.1 and
// 4.2.3 of arXiv 2606.06302) from lengths that are on the device, and the pool
// rows of one layer's entries.
//
// tg_reserve_device is two launches on one stream:
//   lengths  a workgroup per kBlock heads: kv_len = ceil(r * N) (one fp64
//            multiply, as on the host), the groups' maxima in LDS, their pages; a
//            sum and the errors of every workgroup.  Beside them, workgroups that
//            look through as much of the free list as could be taken for the
//            first id outside the pool: what is needed is not known yet
//   tables   every workgroup adds up the sums before its own and scans its
//            tables' pages, and all copy the needed front of the free list (a
//            table's pages are its share of that front, whatever its length);
//            after an error anywhere the offsets are zeros and nothing is copied
// Bound by the bytes of the page ids for large admissions (64 requests, 64 layers, 8
// heads, 5.2 million ids: 5.2 + 7.4 us for 42 MB, the first half from HBM, the other
// from the caches) and by latency for small ones: one launch of one workgroup does
// all of it.
// Every value is written by one workgroup and read only by a later launch: no
// atomics on global memory, no order that the result could depend on.
#include <hip/hip_runtime.h>

#include "tg_device.h"
#include "tg_internal.h"

namespace {

constexpr int kBlock = 256;
constexpr int kSmallBlock = 1024;
constexpr int kCopyBlocks = 1024;    // most workgroups that check or copy page ids
constexpr int kCopyPerBlock = 4096;  // ids of a workgroup before another one joins
// One workgroup does it all up to so many tables, heads and page ids.  Against the
// two launches, with a slot map behind, on the GPU's clock / with the host's
// launches: 4 tables and 74 ids 8.3 / 11.1 us against 8.9 / 14.0; 256 tables, 5700
// ids 8.9 / 10.8 against 9.5 / 13.6; 1024 tables, 7400 ids 10.3 / 11.0 against 10.1 /
// 13.7.
constexpr int kSmallTables = kSmallBlock, kSmallHeads = 4 * kSmallBlock, kSmallIds = 12 * kSmallBlock;

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
  int64_t* sums;        // [blocks] pages of a workgroup's tables; the complement after an invalid length, ratio or group
  int64_t* bad_id;      // [copy_blocks] first place in the free list with an id outside the pool
  int64_t rows;         // batch * L
  int64_t most;         // ids that could be taken: min(num_free, pt_capacity)
  int32_t blocks, copy_blocks, rows_per_block;
  int32_t L, H, G, P;
  bool vec;             // the page id arrays allow 16-byte accesses
};

// A reduction of the workgroup's values; every thread receives it.
template <int N, typename T, typename Op>
__device__ T block_reduce(T x, T* sm, Op op) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = op(x, (T)__shfl_xor((long long)x, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = x;
  __syncthreads();
  x = sm[0];
#pragma unroll
  for (int w = 1; w < N / 64; ++w) x = op(x, sm[w]);
  return x;
}
struct Sum {
  __device__ int64_t operator()(int64_t a, int64_t b) const { return a + b; }
};
struct Min {
  __device__ int64_t operator()(int64_t a, int64_t b) const { return a < b ? a : b; }
};

// Sum of the values of the threads up to and with this one.
template <int N>
__device__ int64_t block_inclusive_sum(int64_t x, int64_t* sm) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = __shfl_up((long long)x, o);
    if ((int)(threadIdx.x & 63) >= o) x += y;
  }
  __syncthreads();
  if ((threadIdx.x & 63) == 63) sm[threadIdx.x >> 6] = x;
  __syncthreads();
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) x += sm[w];
  return x;
}

// The retained lengths of the heads of rows [row0, row0 + n) (a row: one
// request's layer), their groups' maxima in longest[n * G].  Whether a value was
// invalid (its length counts as 0).
template <int N>
__device__ bool lengths(const TableParams& p, int64_t row0, int n, int32_t* longest) {
  for (int i = threadIdx.x; i < n * p.G; i += N) longest[i] = 0;
  __syncthreads();
  bool bad = false;
  for (int i = threadIdx.x; i < n * p.H; i += N) {
    const int64_t row = row0 + i / p.H;
    const int h = i % p.H, l = (int)(row % p.L), b = (int)(row / p.L);
    const int64_t at = row0 * p.H + i;   // of (b, l, h)
    const int ctx = p.ctx_len[b], of = p.group_of[(int64_t)l * p.H + h];
    const double r = p.ratio ? p.ratio[at] : p.budget[(int64_t)l * p.H + h];
    const bool ok = ctx >= 1 && r > 0.0 && r <= 1.0;   // false for NaN
    const int32_t len = ok ? (int32_t)ceil(r * (double)ctx) : 0;
    p.kv_len[at] = len;
    const bool in = of >= 0 && of < p.G;
    if (in) atomicMax(&longest[i / p.H * p.G + of], len);   // LDS
    if (!ok || !in || (p.headroom && p.headroom[b] < 0)) bad = true;
  }
  __syncthreads();
  return bad;
}

__device__ __forceinline__ int64_t table_pages(const TableParams& p, int64_t table, int32_t longest) {
  const int b = (int)(table / ((int64_t)p.L * p.G));
  const int room = p.headroom ? max(p.headroom[b], 0) : 0;
  return ((int64_t)longest + room + p.P - 1) / p.P;
}

__device__ __forceinline__ int32_t status_of(const TableParams& p, bool bad, int64_t needed, int64_t bad_id) {
  if (bad) return TG_ERR_INVALID_ARG;
  if (needed > p.num_free) return TG_ERR_OUT_OF_PAGES;
  if (needed > p.pt_capacity) return TG_ERR_BUFFER_TOO_SMALL;
  return bad_id < needed ? TG_ERR_INVALID_ARG : TG_OK;
}

// fn(place, id) over this workgroup's share of the free list's first n ids
template <int N, typename F>
__device__ __forceinline__ void for_ids(const TableParams& p, int64_t n, int block, int blocks, F fn) {
  const int64_t vecs = p.vec ? n / 4 : 0;
#pragma unroll 4
  for (int64_t i = (int64_t)block * N + threadIdx.x; i < vecs; i += (int64_t)blocks * N) fn(4 * i, reinterpret_cast<const int4*>(p.free_pages)[i]);
  for (int64_t i = 4 * vecs + (int64_t)block * N + threadIdx.x; i < n; i += (int64_t)blocks * N) fn(i, p.free_pages[i]);
}

// The first place with an id outside the pool.
struct FirstBad {
  const TableParams& p;
  int64_t at = INT64_MAX;
  __device__ void operator()(int64_t i, int32_t id) {
    if (id < 0 || id >= p.pool_pages) at = min(at, i);
  }
  __device__ void operator()(int64_t i, const int4& v) {
    (*this)(i, v.x);
    (*this)(i + 1, v.y);
    (*this)(i + 2, v.z);
    (*this)(i + 3, v.w);
  }
};
struct Copy {
  const TableParams& p;
  __device__ void operator()(int64_t i, int32_t id) { p.pt_pages[i] = id; }
  __device__ void operator()(int64_t i, const int4& v) {
    // past the caches, which still hold what the first launch read: 17.2 -> 16.5 us for
    // 5.2 million ids
    typedef int i4 __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(i4{v.x, v.y, v.z, v.w}, reinterpret_cast<i4*>(p.pt_pages + i));
  }
};

__global__ void __launch_bounds__(kBlock) tg_table_lengths_kernel(TableParams p) {
  __shared__ int64_t sm[kBlock / 64];
  __shared__ int32_t longest[kBlock];
  if ((int)blockIdx.x >= p.blocks) {
    const int block = blockIdx.x - p.blocks;
    FirstBad bad{p};
    for_ids<kBlock>(p, p.most, block, p.copy_blocks, [&](int64_t i, auto v) { bad(i, v); });
    const int64_t at = block_reduce<kBlock>(bad.at, sm, Min());
    if (threadIdx.x == 0) p.bad_id[block] = at;
    return;
  }
  const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
  const int n = (int)min<int64_t>(p.rows_per_block, p.rows - row0);
  const bool bad = lengths<kBlock>(p, row0, n, longest);
  int64_t pages = 0;
  if ((int)threadIdx.x < n * p.G) {   // at most kBlock tables
    const int64_t table = row0 * p.G + threadIdx.x;
    p.group_len[table] = longest[threadIdx.x];
    pages = table_pages(p, table, longest[threadIdx.x]);
  }
  // pages in the upper bits, whether anything was invalid in the lowest 16 (at most kBlock of them)
  const int64_t sum = block_reduce<kBlock>(pages * 65536 + bad, sm, Sum());
  if (threadIdx.x == 0) p.sums[blockIdx.x] = sum % 65536 != 0 ? ~(sum / 65536) : sum / 65536;
}

__global__ void __launch_bounds__(kBlock) tg_table_fill_kernel(TableParams p) {
  __shared__ int64_t sm[kBlock / 64], sm_before[kBlock / 64], sm_bad[kBlock / 64];
  int64_t all = 0, before = 0, bad_id = INT64_MAX;
  bool bad = false;
  static_assert(kCopyBlocks == 4 * kBlock, "all of bad_id is asked for at once");
#pragma unroll
  for (int q = 0; q < 4; ++q) bad_id = min(bad_id, p.bad_id[min((int)threadIdx.x + q * kBlock, p.copy_blocks - 1)]);
  for (int i = threadIdx.x; i < p.blocks; i += kBlock) {
    const int64_t s = p.sums[i];
    const int64_t pages = s < 0 ? ~s : s;
    all += pages;
    before += i < (int)blockIdx.x ? pages : 0;
    bad |= s < 0;
  }
  // the three sums at once; an invalid length is a bad id before the first
  if (bad) bad_id = -1;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    all += __shfl_xor((long long)all, o);
    before += __shfl_xor((long long)before, o);
    bad_id = min(bad_id, (int64_t)__shfl_xor((long long)bad_id, o));
  }
  if ((threadIdx.x & 63) == 0) {
    sm[threadIdx.x >> 6] = all;
    sm_before[threadIdx.x >> 6] = before;
    sm_bad[threadIdx.x >> 6] = bad_id;
  }
  __syncthreads();
  all = before = 0;
#pragma unroll
  for (int w = 0; w < kBlock / 64; ++w) {
    all += sm[w];
    before += sm_before[w];
    bad_id = min(bad_id, sm_bad[w]);
  }
  const int64_t needed = all;
  const int32_t status = status_of(p, bad_id < 0, needed, bad_id);
  if (status == TG_OK && (int)blockIdx.x < p.copy_blocks) {
    Copy copy{p};
    for_ids<kBlock>(p, needed, blockIdx.x, p.copy_blocks, [&](int64_t i, auto v) { copy(i, v); });
  }
  if ((int)blockIdx.x < p.blocks) {
    const int64_t row0 = (int64_t)blockIdx.x * p.rows_per_block;
    const int n = (int)min<int64_t>(p.rows_per_block, p.rows - row0) * p.G;
    const int64_t table = row0 * p.G + threadIdx.x;
    const bool mine = (int)threadIdx.x < n;
    const int64_t pages = mine ? table_pages(p, table, p.group_len[table]) : 0;
    const int64_t end = before + block_inclusive_sum<kBlock>(pages, sm);
    if (mine) p.pt_offsets[table] = status == TG_OK ? end - pages : 0;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.pt_offsets[p.rows * p.G] = status == TG_OK ? needed : 0;
    *p.pages_needed = needed;
    *p.status = status;
  }
}

__global__ void __launch_bounds__(kSmallBlock) tg_table_small_kernel(TableParams p) {
  __shared__ int64_t sm[kSmallBlock / 64];
  __shared__ int32_t longest[kSmallTables];
  const bool invalid = lengths<kSmallBlock>(p, 0, (int)p.rows, longest);
  const int tables = (int)p.rows * p.G;
  const bool mine = (int)threadIdx.x < tables;
  const int64_t pages = mine ? table_pages(p, threadIdx.x, longest[threadIdx.x]) : 0;
  if (mine) p.group_len[threadIdx.x] = longest[threadIdx.x];
  const int64_t end = block_inclusive_sum<kSmallBlock>(pages, sm);
  __syncthreads();
  if (threadIdx.x == kSmallBlock - 1) sm[0] = end;
  __syncthreads();
  const int64_t needed = sm[0];
  FirstBad first{p};
  for_ids<kSmallBlock>(p, min(needed, p.most), 0, 1, [&](int64_t i, auto v) { first(i, v); });
  const int64_t bad_id = block_reduce<kSmallBlock>(invalid ? -1 : first.at, sm, Min());
  const int32_t status = status_of(p, bad_id < 0, needed, bad_id);
  if (status == TG_OK) {
    Copy copy{p};
    for_ids<kSmallBlock>(p, needed, 0, 1, [&](int64_t i, auto v) { copy(i, v); });
  }
  if (mine) p.pt_offsets[threadIdx.x] = status == TG_OK ? end - pages : 0;
  if (threadIdx.x == 0) {
    p.pt_offsets[tables] = status == TG_OK ? needed : 0;
    *p.pages_needed = needed;
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

// Grid (ceil(n / kMapPerBlock), heads, requests): kMapPerBlock entries of one head.
constexpr int kMapPerBlock = 4 * kBlock;

__global__ void __launch_bounds__(kBlock) tg_slot_map_kernel(MapParams p) {
  const int h = blockIdx.y;
  const int64_t b = blockIdx.z, unit = b * p.H + h;
  const int64_t at = (b * p.L + p.layer) * p.H + h;
  const int64_t lh = (int64_t)p.layer * p.H + h;
  const tgd::TablePages table = tgd::table_of(p.pt_offsets, (b * p.L + p.layer) * p.G, p.group_of[lh], p.G);
  const int64_t cap = table.pages * p.P;
  const int64_t first = p.begin ? p.begin[at] : 0;
  const int64_t end = p.len ? min<int64_t>(p.len[at], cap) : cap;
  const int slot = p.slot_of[lh];
  for (int q = 0; q < 4; ++q) {
    const int64_t j = (int64_t)blockIdx.x * kMapPerBlock + q * kBlock + threadIdx.x;
    if (j >= p.n) return;
    const int64_t e = first + j;
    int64_t row = -1;
    if (e >= 0 && e < end) {
      const int64_t page = p.pt_pages[table.base + e / p.P];
      row = (page * 2 * p.Hp + slot) * p.P + e % p.P;
    }
    p.map[unit * p.n + j] = row;
  }
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {
  int64_t rows, blocks;
  int rows_per_block;
  size_t sums, bad_id, total;
};

Layout layout_of(const tg_geometry& g, int batch) {
  Layout l;
  l.rows = (int64_t)batch * g.num_layers;
  l.rows_per_block = kBlock / g.num_kv_heads;
  if (l.rows_per_block < 1) l.rows_per_block = 1;
  l.blocks = (l.rows + l.rows_per_block - 1) / l.rows_per_block;
  l.sums = align256((size_t)l.blocks * sizeof(int64_t));
  l.bad_id = align256(kCopyBlocks * sizeof(int64_t));
  l.total = l.sums + l.bad_id;
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
  if (g.num_kv_heads > kBlock)
    return tg::fail(TG_ERR_UNSUPPORTED, "reserve on the device supports up to %d KV heads (got %d)", kBlock, g.num_kv_heads);
  const Layout l = layout_of(g, a->batch);
  if (l.blocks > INT32_MAX - kCopyBlocks) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
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
  p.bad_id = reinterpret_cast<int64_t*>(ws + l.sums);
  p.rows = l.rows;
  p.blocks = (int32_t)l.blocks;
  p.rows_per_block = l.rows_per_block;
  p.L = g.num_layers;
  p.H = g.num_kv_heads;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.P = g.page_size;
  p.vec = tg::aligned16({a->free_pages, a->pt_pages});
  p.most = a->num_free < a->pt_capacity ? a->num_free : a->pt_capacity;
  const int64_t copy = (p.most + kCopyPerBlock - 1) / kCopyPerBlock;
  p.copy_blocks = (int32_t)(copy < 1 ? 1 : copy > kCopyBlocks ? kCopyBlocks : copy);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  if (l.rows * p.G <= kSmallTables && l.rows * p.H <= kSmallHeads && p.most <= kSmallIds) {
    hipLaunchKernelGGL(tg_table_small_kernel, dim3(1), dim3(kSmallBlock), 0, st, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "reserve launch failed: %s", hipGetErrorString(e));
    return TG_OK;
  }
  hipLaunchKernelGGL(tg_table_lengths_kernel, dim3(p.blocks + p.copy_blocks), dim3(kBlock), 0, st, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "reserve launch failed: %s", hipGetErrorString(e));
  hipLaunchKernelGGL(tg_table_fill_kernel, dim3(p.blocks > p.copy_blocks ? p.blocks : p.copy_blocks), dim3(kBlock), 0, st, p);
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
