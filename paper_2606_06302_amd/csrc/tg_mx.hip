// Writing one token per request into a quantised cache (tg_append_mx), and reading
// a layer's entries back as rows of bf16 or fp32 (tg_unpack_mx).
#include <hip/hip_runtime.h>

#include "tg_mx.h"

namespace {

using namespace tgd;

constexpr int kThreads = 256;

struct AppendParams {
  const u4* k_tok;
  const u4* v_tok;
  uint8_t* pool;
  const int32_t* pt_pages;
  const int64_t* pt_offsets;
  const int32_t* group_of;
  const int32_t* slot_of;
  int32_t* live_len;
  int32_t* full;
  int32_t batch, L, H, G, Hp, layer;
  int32_t d, kb, vb;
};

// A lane holds 16 bytes of a head's K row and of its V row, as in tg_append: 8
// elements of bf16 (four lanes share a scale) or 4 of fp32 (eight do).  Bound by
// its chain of loads (length, table, page id): 64 requests of 8 heads take 4.6 us
// with the copy that puts their lengths back, tg_append 4.7.
template <typename T>
__global__ __launch_bounds__(kThreads) void tg_append_mx_kernel(AppendParams p) {
  constexpr int E = Row16<T>::kElems;
  const int lpr = p.d / E;
  const int units_per_wg = kThreads / lpr;
  const int64_t unit = (int64_t)blockIdx.x * units_per_wg + threadIdx.x / lpr;
  const int sub = threadIdx.x % lpr;
  if (unit >= (int64_t)p.batch * p.H) return;
  const u4 kv = p.k_tok[unit * lpr + sub], vv = p.v_tok[unit * lpr + sub];
  const int b = (int)(unit / p.H), h = (int)(unit % p.H);
  const int64_t lh = (int64_t)p.layer * p.H + h;
  int32_t* live = p.live_len + ((int64_t)b * p.L + p.layer) * p.H + h;
  const int n = *live;
  const TablePages table = table_of(p.pt_offsets, ((int64_t)b * p.L + p.layer) * p.G, p.group_of[lh], p.G);
  if (n < 0 || n >= table.pages * kMxPage) {
    if (p.full && sub == 0) *p.full = 1;
    return;
  }
  const int64_t page = p.pt_pages[table.base + n / kMxPage];
  uint8_t* slab = p.pool + (page * p.Hp + p.slot_of[lh]) * mx_slab_bytes(p.d, p.kb, p.vb);
  const MxParts at = mx_parts(p.d, p.kb, p.vb);
  uint32_t scale;
  u2 c = mx_quantise<T>(kv, p.kb, &scale);
  mx_store<E>(slab, slab + at.k_scales, n % kMxPage, sub * E, p.d, p.kb, false, c, scale);
  c = mx_quantise<T>(vv, p.vb, &scale);
  mx_store<E>(slab + at.v_codes, slab + at.v_scales, n % kMxPage, sub * E, p.d, p.vb, true, c, scale);
  // every lane of the unit has read n (same wave, same load)
  if (sub == 0) *live = n + 1;
}

struct UnpackParams {
  const uint8_t* pool;
  u4* rows;
  const int32_t* pt_pages;
  const int32_t* dst_pages;   // = pt_pages where there are none
  const int64_t* pt_offsets;
  const int32_t* group_of;
  const int32_t* slot_of;
  const int32_t* begin;   // [B][L][H] or NULL
  const int32_t* len;     // [B][L][H]
  int32_t L, H, G, Hp, layer;
  int64_t units;
};

// 16 bytes of a row from its codes
template <typename T, int BITS>
__device__ __forceinline__ u4 row16(const u2& c, float s) {
  if constexpr (sizeof(T) == 2) {
    if constexpr (BITS == 4)
      return u4{mx_pair4<0>(c.x, s), mx_pair4<1>(c.x, s), mx_pair4<2>(c.x, s), mx_pair4<3>(c.x, s)};
    else
      return u4{mx_pair8<0>(c.x, s), mx_pair8<1>(c.x, s), mx_pair8<0>(c.y, s), mx_pair8<1>(c.y, s)};
  } else {
    const uint32_t a = BITS == 4 ? mx_pair4<0>(c.x, s) : mx_pair8<0>(c.x, s);
    const uint32_t b = BITS == 4 ? mx_pair4<1>(c.x, s) : mx_pair8<1>(c.x, s);
    return u4{a << 16, a & 0xffff0000u, b << 16, b & 0xffff0000u};
  }
}

constexpr int kUnits = 1024;    // (request, head) units shared out at once
constexpr int kUnpackWgs = 256; // the CUs of an MI355X; any number is right

// The lengths are on the device and differ a lot between heads, so the pages are
// shared out here: every workgroup lays the units' pages end to end (a sum over
// the units in LDS) and every wave takes an equal range of them, up to 64 pages at
// a time, one a lane for what is looked up per page.  A lane reads and writes 16
// bytes of a row, so that the stores, most of the bytes, are whole rows in order;
// a page's codes are requested before the page before it is stored.
//
// Bound by memory: 8 requests of up to 16384 tokens (4-bit rows to bf16, 214 MB)
// 37 us, 5.8 TB/s (three such calls in turn, more than the last-level cache holds,
// 37.3); a few pages 4.6 us, the chain from tables to codes.  A
// workgroup a unit with plain stores took 92 us there, stores past the caches 52,
// equal ranges of pages 38.  One workgroup a CU: with two, three or four the same
// 37.6, 37.9 and 39.3, small calls 5.2 / 5.3 / 5.5 / 6.0, of 14 others two
// are faster with two a CU, by 2 and 6 %.
template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(kThreads) void tg_unpack_mx_kernel(UnpackParams p) {
  constexpr int E = Row16<T>::kElems;
  constexpr int LPR = D / E;                 // lanes per row
  constexpr int RPP = 64 / LPR;              // rows at once
  constexpr int NR = kMxPage / RPP;
  constexpr int kSlab = mx_slab_bytes(D, KB, VB);
  constexpr int kPer = kUnits / kThreads;    // units of a thread
  constexpr MxParts at = mx_parts(D, KB, VB);
  __shared__ int64_t sm_end[kUnits];         // pages up to and with the unit's
  __shared__ int64_t sm_first[kUnits];       // of the unit's page ids, from its first entry read
  __shared__ int32_t sm_lo[kUnits], sm_hi[kUnits];
  __shared__ int64_t sm_wave[kThreads / 64];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + wave, waves = (int64_t)gridDim.x * (kThreads / 64);
  const int sub = lane % LPR, r0 = lane / LPR;

  for (int64_t u0 = 0; u0 < p.units; u0 += kUnits) {
    const int n = (int)min((int64_t)kUnits, p.units - u0);
    int64_t mine[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int k = threadIdx.x * kPer + i;
      int64_t pages = 0;
      if (k < n) {
        const int64_t b = (uint32_t)(u0 + k) / (uint32_t)p.H;
        const int h = (int)((uint32_t)(u0 + k) % (uint32_t)p.H);
        const int64_t blh = (b * p.L + p.layer) * p.H + h;
        const TablePages table =
            table_of(p.pt_offsets, (b * p.L + p.layer) * p.G, p.group_of[(int64_t)p.layer * p.H + h], p.G);
        const int32_t lo = p.begin ? max(p.begin[blh], 0) : 0;
        const int32_t hi = (int32_t)min((int64_t)p.len[blh], table.pages * kMxPage);
        sm_lo[k] = lo;
        sm_hi[k] = hi;
        sm_first[k] = table.base + lo / kMxPage;
        pages = hi > lo ? (hi - 1) / kMxPage - lo / kMxPage + 1 : 0;
      }
      sum += pages;
      mine[i] = sum;
    }
    int64_t before = sum;   // of the threads up to and with this one, in its wave
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const int64_t x = __shfl_up(before, s);
      before += lane >= s ? x : 0;
    }
    if (lane == 63) sm_wave[wave] = before;
    __syncthreads();
    before -= sum;
    for (int i = 0; i < wave; ++i) before += sm_wave[i];
#pragma unroll
    for (int i = 0; i < kPer; ++i) sm_end[threadIdx.x * kPer + i] = before + mine[i];
    __syncthreads();

    const int64_t total = sm_end[kUnits - 1];
    const int64_t f1 = total * (w + 1) / waves;
    for (int64_t f = total * w / waves; f < f1; f += 64) {
      const int count = (int)min((int64_t)64, f1 - f);
      // of page f + lane: its slab, its rows in the other pool, the rows to write
      int64_t src = 0, dst = 0;
      int32_t from = 0, to = 0;
      if (lane < count) {
        int u = 0;
#pragma unroll
        for (int s = kUnits / 2; s > 0; s /= 2) u += sm_end[u + s - 1] <= f + lane ? s : 0;
        const int64_t at_page = f + lane - (u > 0 ? sm_end[u - 1] : 0);
        const int h = (int)((uint32_t)(u0 + u) % (uint32_t)p.H);
        const int slot = p.slot_of[(int64_t)p.layer * p.H + h];
        const int64_t id = sm_first[u] + at_page;
        const int32_t row = (int32_t)(sm_lo[u] / kMxPage + at_page) * kMxPage;
        src = ((int64_t)p.pt_pages[id] * p.Hp + slot) * kSlab;
        dst = ((int64_t)p.dst_pages[id] * 2 * p.Hp + slot) * kMxPage;
        from = sm_lo[u] - row;
        to = sm_hi[u] - row;
      }
      auto of64 = [](int64_t x, int j) {
        return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int32_t)(x >> 32), j) << 32) |
                         (uint32_t)__builtin_amdgcn_readlane((int32_t)x, j));
      };
      struct Page {
        u2 kc[NR], vc[NR];
        uint32_t ks[NR], vs[NR];
      };
      auto load = [&](Page& g, int j) {
        const uint8_t* slab = p.pool + of64(src, j);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const int t = i * RPP + r0;
          g.kc[i] = mx_load<E>(slab, t, sub * E, D, KB, false);
          g.vc[i] = mx_load<E>(slab + at.v_codes, t, sub * E, D, VB, true);
          g.ks[i] = slab[at.k_scales + mx_scale_at(t, sub * E / kMxGroup, D, false)];
          g.vs[i] = slab[at.v_scales + mx_scale_at(t, sub * E / kMxGroup, D, true)];
        }
      };
      auto store = [&](const Page& g, int j) {
        u4* kr = p.rows + of64(dst, j) * LPR + lane;
        u4* vr = kr + (int64_t)p.Hp * kMxPage * LPR;
        const int lo = __builtin_amdgcn_readlane(from, j), hi = __builtin_amdgcn_readlane(to, j);
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const int t = i * RPP + r0;
          if (t >= lo && t < hi) {
            __builtin_nontemporal_store(row16<T, KB>(g.kc[i], mx_scale(g.ks[i])), kr + i * 64);
            __builtin_nontemporal_store(row16<T, VB>(g.vc[i], mx_scale(g.vs[i])), vr + i * 64);
          }
        }
      };
      Page a, b;
      load(a, 0);
      for (int j = 0; j < count; j += 2) {
        if (j + 1 < count) load(b, j + 1);
        store(a, j);
        if (j + 1 >= count) break;
        if (j + 2 < count) load(a, j + 2);
        store(b, j + 1);
      }
    }
    if (u0 + kUnits < p.units) __syncthreads();   // the sums may be written again
  }
}

using UnpackFn = void (*)(UnpackParams);

template <typename T, int D>
UnpackFn pick_unpack(int kb, int vb) {
  if (kb == 4) return vb == 4 ? &tg_unpack_mx_kernel<T, D, 4, 4> : &tg_unpack_mx_kernel<T, D, 4, 8>;
  return vb == 4 ? &tg_unpack_mx_kernel<T, D, 8, 4> : &tg_unpack_mx_kernel<T, D, 8, 8>;
}

}  // namespace

extern "C" {

size_t tg_mx_page_bytes(const tg_geometry* geom, const tg_mx_format* format) {
  if (tg::check_mx(geom, format)) return 0;
  return (size_t)geom->heads_per_group *
         mx_slab_bytes(geom->head_dim, tg::mx_bits(format->k_format), tg::mx_bits(format->v_format));
}

int32_t tg_append_mx(const tg_append_args* a, const tg_mx_format* format, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = tg::check_mx(&g, format)) return rc;
  if (a->dtype != TG_F32 && a->dtype != TG_BF16) return tg::fail(TG_ERR_UNSUPPORTED, "dtype must be f32 or bf16");
  if (a->batch < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch must be >= 1");
  if (a->layer < 0 || a->layer >= g.num_layers) return tg::fail(TG_ERR_INVALID_ARG, "layer %d out of range", a->layer);
  if (!a->k_tok || !a->v_tok || !a->kv_pool || !a->pt_pages || !a->pt_offsets || !a->group_of || !a->slot_of ||
      !a->live_len)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  if (!tg::aligned16({a->k_tok, a->v_tok, a->kv_pool}))
    return tg::fail(TG_ERR_INVALID_ARG, "device buffers must be 16-byte aligned");
  AppendParams p;
  p.k_tok = static_cast<const u4*>(a->k_tok);
  p.v_tok = static_cast<const u4*>(a->v_tok);
  p.pool = static_cast<uint8_t*>(a->kv_pool);
  p.pt_pages = a->pt_pages;
  p.pt_offsets = a->pt_offsets;
  p.group_of = a->group_of;
  p.slot_of = a->slot_of;
  p.live_len = a->live_len;
  p.full = a->full;
  p.batch = a->batch;
  p.L = g.num_layers;
  p.H = g.num_kv_heads;
  p.Hp = g.heads_per_group;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.layer = a->layer;
  p.d = g.head_dim;
  p.kb = tg::mx_bits(format->k_format);
  p.vb = tg::mx_bits(format->v_format);
  const int64_t per_wg = kThreads * (a->dtype == TG_F32 ? 4 : 8) / g.head_dim;
  const int64_t blocks = tg::ceil_div((int64_t)a->batch * g.num_kv_heads, per_wg);
  if (blocks > INT32_MAX) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
  hipLaunchKernelGGL(a->dtype == TG_F32 ? tg_append_mx_kernel<float> : tg_append_mx_kernel<uint16_t>,
                     dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "append launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}

int32_t tg_unpack_mx(const tg_unpack_mx_args* a, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = tg::check_mx(&g, &a->format)) return rc;
  if (a->dtype != TG_F32 && a->dtype != TG_BF16) return tg::fail(TG_ERR_UNSUPPORTED, "dtype must be f32 or bf16");
  if (a->batch < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch must be >= 1");
  if (a->layer < 0 || a->layer >= g.num_layers) return tg::fail(TG_ERR_INVALID_ARG, "layer %d out of range", a->layer);
  if (!a->mx_pool || !a->kv_pool || !a->pt_pages || !a->pt_offsets || !a->group_of || !a->slot_of || !a->len)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  if (!tg::aligned16({a->mx_pool, a->kv_pool}))
    return tg::fail(TG_ERR_INVALID_ARG, "device buffers must be 16-byte aligned");
  UnpackParams p;
  p.pool = static_cast<const uint8_t*>(a->mx_pool);
  p.rows = static_cast<u4*>(a->kv_pool);
  p.pt_pages = a->pt_pages;
  p.dst_pages = a->dst_pages ? a->dst_pages : a->pt_pages;
  p.pt_offsets = a->pt_offsets;
  p.group_of = a->group_of;
  p.slot_of = a->slot_of;
  p.begin = a->begin;
  p.len = a->len;
  p.L = g.num_layers;
  p.H = g.num_kv_heads;
  p.Hp = g.heads_per_group;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.layer = a->layer;
  p.units = (int64_t)a->batch * g.num_kv_heads;
  if (p.units > INT32_MAX) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
  const int kb = tg::mx_bits(a->format.k_format), vb = tg::mx_bits(a->format.v_format);
  UnpackFn fn = a->dtype == TG_F32 ? (g.head_dim == 64 ? pick_unpack<float, 64>(kb, vb) : pick_unpack<float, 128>(kb, vb))
                                   : (g.head_dim == 64 ? pick_unpack<uint16_t, 64>(kb, vb) : pick_unpack<uint16_t, 128>(kb, vb));
  hipLaunchKernelGGL(fn, dim3(kUnpackWgs), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "unpack launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}

}  // extern "C"
