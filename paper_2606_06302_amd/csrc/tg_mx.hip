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
// elements of bf16 (four lanes share a scale) or 4 of fp32 (eight do).
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
  float x[E];
  uint32_t scale;
  Row16<T>::unpack(kv, x);
  u2 c = mx_quantise<E>(x, p.kb, &scale);
  mx_store<E>(slab, slab + at.k_scales, n % kMxPage, sub * E, p.d, p.kb, false, c, scale);
  Row16<T>::unpack(vv, x);
  c = mx_quantise<E>(x, p.vb, &scale);
  mx_store<E>(slab + at.v_codes, slab + at.v_scales, n % kMxPage, sub * E, p.d, p.vb, true, c, scale);
  // every lane of the unit has read n (same wave, same load)
  if (sub == 0) *live = n + 1;
}

struct UnpackParams {
  const uint8_t* pool;
  u4* rows;
  const int32_t* pt_pages;
  const int32_t* dst_pages;
  const int64_t* pt_offsets;
  const int32_t* group_of;
  const int32_t* slot_of;
  const int32_t* begin;   // [B][L][H] or NULL
  const int32_t* len;     // [B][L][H]
  int32_t L, H, G, Hp, layer;
  int32_t waves;          // waves that share a unit
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

// A wave takes a page of one head at a time: every lane 16 bytes of a row, so that
// the stores, most of the bytes, are whole rows in order.
template <typename T, int D, int KB, int VB>
__global__ __launch_bounds__(kThreads) void tg_unpack_mx_kernel(UnpackParams p) {
  constexpr int E = Row16<T>::kElems;
  constexpr int LPR = D / E;                 // lanes per row
  constexpr int RPP = 64 / LPR;              // rows at once
  constexpr int NR = kMxPage / RPP;
  constexpr MxParts at = mx_parts(D, KB, VB);
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = w / p.waves;
  const int first = (int)(w % p.waves);
  const int64_t b = unit / p.H;
  const int h = (int)(unit % p.H);
  const int64_t lh = (int64_t)p.layer * p.H + h, blh = (b * p.L + p.layer) * p.H + h;
  const TablePages table = table_of(p.pt_offsets, (b * p.L + p.layer) * p.G, p.group_of[lh], p.G);
  const int64_t cap = table.pages * kMxPage;
  const int64_t lo = p.begin ? max(p.begin[blh], 0) : 0, hi = min((int64_t)p.len[blh], cap);
  const int slot = p.slot_of[lh];
  const int sub = lane % LPR, r0 = lane / LPR;
  for (int64_t pg = lo / kMxPage + first; pg * kMxPage < hi; pg += p.waves) {
    const uint8_t* slab = p.pool + ((int64_t)p.pt_pages[table.base + pg] * p.Hp + slot) * mx_slab_bytes(D, KB, VB);
    u2 kc[NR], vc[NR];
    uint32_t ks[NR], vs[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int t = i * RPP + r0;
      kc[i] = mx_load<E>(slab, t, sub * E, D, KB, false);
      vc[i] = mx_load<E>(slab + at.v_codes, t, sub * E, D, VB, true);
      ks[i] = slab[at.k_scales + mx_scale_at(t, sub * E / kMxGroup, D, false)];
      vs[i] = slab[at.v_scales + mx_scale_at(t, sub * E / kMxGroup, D, true)];
    }
    const int64_t dst = (p.dst_pages ? p.dst_pages : p.pt_pages)[table.base + pg];
    u4* kr = p.rows + ((dst * 2 * p.Hp + slot) * kMxPage) * LPR + lane;
    u4* vr = kr + (int64_t)p.Hp * kMxPage * LPR;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int64_t entry = pg * kMxPage + i * RPP + r0;
      if (entry >= lo && entry < hi) {
        kr[i * 64] = row16<T, KB>(kc[i], mx_scale(ks[i]));
        vr[i * 64] = row16<T, VB>(vc[i], mx_scale(vs[i]));
      }
    }
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
  p.dst_pages = a->dst_pages;
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
  const int64_t units = (int64_t)a->batch * g.num_kv_heads;
  // the lengths are on the device: every unit gets the same number of waves
  p.waves = (int32_t)(4 * tg::ceil_div(2048, units) < 16 ? 16 : 4 * tg::ceil_div(2048, units));
  const int64_t blocks = units * p.waves / 4;
  if (blocks > INT32_MAX) return tg::fail(TG_ERR_INVALID_ARG, "batch too large");
  const int kb = tg::mx_bits(a->format.k_format), vb = tg::mx_bits(a->format.v_format);
  UnpackFn fn = a->dtype == TG_F32 ? (g.head_dim == 64 ? pick_unpack<float, 64>(kb, vb) : pick_unpack<float, 128>(kb, vb))
                                   : (g.head_dim == 64 ? pick_unpack<uint16_t, 64>(kb, vb) : pick_unpack<uint16_t, 128>(kb, vb));
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream), p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "unpack launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}

}  // extern "C"
