// Ragged paged split-KV decode attention over a quantised cache (tg_decode_mx).
//
// The plans, work items, partials and merge are tg_decode's; a bin is run by a
// workgroup, whose waves take the item's pages KP at a time in turn, each with an
// online-softmax state of its own, merged through LDS at the item's end.
//
// The slab of a page (tg_mx.h) lies as the lanes of a wave take it, so a page is
// four loads a lane straight into registers: K codes, V codes and a scale word of
// each.  gfx950 turns two codes into two bf16 numbers with their power-of-two
// scale in one full-rate instruction, exactly, and the products run on them with
// the query heads of the KV head as the 16 columns (columns past G repeat a real
// head and are never stored):
//   * S^T[16 tok][16 heads] = K q^T, D/32 x v_mfma_f32_16x16x32_bf16.  The lanes
//     of quarter j hold dims j D/4 .. of a row, so the k index runs through the
//     dims in that order, in K and in q alike.
//   * online softmax over the step's 16 KP tokens; the 4 lanes of a column are
//     combined with the permlane swaps, and the maximum is raised only when a step
//     exceeds it by more than 2^8 in weight.
//   * O^T[16 dims][16 heads] += V^T P^T, D/16 products 32 tokens deep: tokens
//     4j .. 4j + 3 of two pages for lane group j, which is where S^T leaves them.
//     The V operand pairs tokens, its codes pair dims: one byte permute each.
// With fp32 queries, q and P go in as three bf16 parts that hold their 24 bits.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "tg_mx.h"

namespace {

using namespace tgd;

constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;
constexpr int KP = 2;          // pages of a step
constexpr int kMaxGqa = 16;
constexpr int kPad = 4;        // floats between the heads' accumulators in LDS

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

#define TG_CONST __attribute__((address_space(4)))

struct MxDecodeParams {
  const void* q;
  uint8_t* pool;
  int64_t page_bytes;
  int32_t slab_bytes;
  int32_t num_q_heads, num_kv_heads, n_bins, gqa;
  const int32_t* unit_splits;
  const int32_t* unit_partial_base;
  void* out;
  float* lse;
  float* part_o;               // [num_partials][gqa][d]
  float* part_lse;             // [num_partials][gqa]
  uint64_t* timestamps;
  int32_t* live;               // live lengths of this layer, or NULL
  int32_t live_stride;
  int32_t* merge_counters;     // of the in-launch merge, or NULL
  const u4* append_k;
  const u4* append_v;
  int32_t* append_full;
  float scale;                 // sm_scale, over softcap with a cap
  float cap;                   // softcap, or 0
};

__device__ __forceinline__ f32x4 mfma(const u4& a, const u4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// Codes 2i and 2i + 1 of a lane as a pair of bf16.
template <int BITS>
__device__ __forceinline__ uint32_t pair(const uint32_t* w, int i, float s) {
  if constexpr (BITS == 4) {
    switch (i & 3) {
      case 0: return mx_pair4<0>(w[i >> 2], s);
      case 1: return mx_pair4<1>(w[i >> 2], s);
      case 2: return mx_pair4<2>(w[i >> 2], s);
      default: return mx_pair4<3>(w[i >> 2], s);
    }
  } else {
    return (i & 1) ? mx_pair8<1>(w[i >> 1], s) : mx_pair8<0>(w[i >> 1], s);
  }
}

// The W words of a lane's codes.
template <int W>
__device__ __forceinline__ void load_codes(const uint8_t* codes, int lane, uint32_t* w) {
  if constexpr (W == 2) {
    const u2 x = *reinterpret_cast<const u2*>(codes + lane * 8);
    w[0] = x.x;
    w[1] = x.y;
  } else {
#pragma unroll
    for (int c = 0; c < W / 4; ++c) {
      const u4 x = *reinterpret_cast<const u4*>(codes + c * 1024 + lane * 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[4 * c + i] = x[i];
    }
  }
}

// fp32 as three bf16 parts, cut and not rounded: their sum is x.  An infinity is
// its first part.
__device__ __forceinline__ void split3(float x, uint32_t* part) {
  const uint32_t hi = __float_as_uint(x) & 0xffff0000u;
  const float r1 = __builtin_isinf(x) ? 0.f : x - __uint_as_float(hi);
  const uint32_t mid = __float_as_uint(r1) & 0xffff0000u;
  part[0] = hi;
  part[1] = mid;
  part[2] = __float_as_uint(r1 - __uint_as_float(mid)) & 0xffff0000u;
}
__device__ __forceinline__ uint32_t join16(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

template <typename T>
__device__ __forceinline__ void store4(T* dst, const f32x4& v);
template <>
__device__ __forceinline__ void store4<float>(float* dst, const f32x4& v) { *reinterpret_cast<f32x4*>(dst) = v; }
template <>
__device__ __forceinline__ void store4<uint16_t>(uint16_t* dst, const f32x4& v) {
  *reinterpret_cast<u2*>(dst) = u2{uint32_t(f32_to_bf16(v[0])) | (uint32_t(f32_to_bf16(v[1])) << 16),
                                   uint32_t(f32_to_bf16(v[2])) | (uint32_t(f32_to_bf16(v[3])) << 16)};
}

__device__ __forceinline__ tg_work_item load_item(const TG_CONST tg_work_item* src) {
  tg_work_item r;
  r.pt_base = src->pt_base;
  r.b = src->b;
  r.kv_head = src->kv_head;
  r.slot = src->slot;
  r.tok_begin = src->tok_begin;
  r.tok_end = src->tok_end;
  r.out_idx = src->out_idx;
  return r;
}

constexpr size_t lds_floats(int gqa, int d) { return (size_t)kWaves * gqa * (d + kPad + 2) + 4; }

template <typename T, int D, int KB, int VB>
__global__ void __launch_bounds__(kBlock)
    tg_decode_mx_kernel(MxDecodeParams p, const tg_work_item* __restrict__ items_g, const int32_t* __restrict__ pt_g,
                        const int32_t* __restrict__ bin_offsets_g) {
  constexpr int E = Row16<T>::kElems;
  constexpr int NPART = sizeof(T) == 4 ? 3 : 1;   // bf16 parts of q and P
  constexpr int KW = D * KB / 128, VW = D * VB / 128;
  constexpr int NQ = D / 32, NV = D / 16;
  constexpr MxParts at = mx_parts(D, KB, VB);
  constexpr float kSlack = 8.0f;
  extern __shared__ float lds[];

  const TG_CONST tg_work_item* const items = (const TG_CONST tg_work_item*)items_g;
  const TG_CONST int32_t* const pt = (const TG_CONST int32_t*)pt_g;
  const TG_CONST int32_t* const bin_offsets = (const TG_CONST int32_t*)bin_offsets_g;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, rb = lane >> 4;
  const int G = p.gqa;
  const int hq = col < G ? col : col % G;
  float* const sm_acc = lds;                                  // [wave][head][D + kPad]
  float* const sm_m = lds + kWaves * G * (D + kPad);          // [wave][head]
  float* const sm_l = sm_m + kWaves * G;
  int* const sm_flag = reinterpret_cast<int*>(sm_l + kWaves * G);
  const uint64_t t_start = __builtin_amdgcn_s_memrealtime();
  const int it_begin = bin_offsets[blockIdx.x], it_end = bin_offsets[blockIdx.x + 1];
  const float cs = p.cap > 0.f ? kLog2e : p.scale * kLog2e;   // log2 units per unit of (capped) score

  for (int it = it_begin; it < it_end; ++it) {
    tg_work_item item = load_item(items + it);
    int arow = -1;
    if (item.tok_end < 0) {
      const int n = p.live ? p.live[(int64_t)item.b * p.live_stride + item.kv_head] : -item.tok_end;
      item.tok_end = __builtin_amdgcn_readfirstlane(
          resolve_open(item.tok_begin, item.tok_end, n, p.append_k != nullptr, &arow));
      arow = __builtin_amdgcn_readfirstlane(arow);
    }
    const int ntok = item.tok_end - item.tok_begin;
    const int np = (ntok + kMxPage - 1) / kMxPage;
    const TG_CONST int32_t* const ids = pt + item.pt_base + item.tok_begin / kMxPage;
    const uint8_t* const slabs = p.pool + (int64_t)item.slot * p.slab_bytes;
    const int ns = (np - wave * KP + kWaves * KP - 1) / (kWaves * KP);   // this wave's steps; may be 0

    // the wave that attends to the new token quantises and stores it first, and
    // reads it back with its page
    if (arow >= 0 && (np - 1) / KP % kWaves == wave) {
      constexpr int LPR = D / E;
      const int t = arow % kMxPage;
      uint8_t* slab = p.pool + (int64_t)ids[np - 1] * p.page_bytes + (int64_t)item.slot * p.slab_bytes;
      const int64_t row = ((int64_t)item.b * p.num_kv_heads + item.kv_head) * LPR + lane % LPR;
      if (lane < 2 * LPR) {
        const bool is_v = lane >= LPR;
        float x[E];
        uint32_t scale;
        Row16<T>::unpack(is_v ? p.append_v[row] : p.append_k[row], x);
        if (is_v) {
          const u2 c = mx_quantise<E>(x, VB, &scale);
          mx_store<E>(slab + at.v_codes, slab + at.v_scales, t, lane % LPR * E, D, VB, true, c, scale);
        } else {
          const u2 c = mx_quantise<E>(x, KB, &scale);
          mx_store<E>(slab, slab + at.k_scales, t, lane * E, D, KB, false, c, scale);
        }
      }
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this wave's loads of the page come behind the stores
    }

    u4 qv[NPART][NQ];
    {
      const T* q = static_cast<const T*>(p.q) +
                   ((int64_t)item.b * p.num_q_heads + item.kv_head * G + hq) * D + rb * (D / 4);
#pragma unroll
      for (int m = 0; m < NQ; ++m) {
        if constexpr (NPART == 1) {
          qv[0][m] = *reinterpret_cast<const u4*>(q + 8 * m);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t a[3], b[3];
            split3(q[8 * m + 2 * i], a);
            split3(q[8 * m + 2 * i + 1], b);
#pragma unroll
            for (int s = 0; s < 3; ++s) qv[s][m][i] = join16(a[s], b[s]);
          }
        }
      }
    }

    struct Tile {
      uint32_t k[KP][KW], v[KP][VW], ks[KP], vs[KP];
    };
    auto load = [&](Tile& t, int step) {
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        const int page = min((step * kWaves + wave) * KP + k, np - 1);
        const uint8_t* slab = slabs + (int64_t)ids[page] * p.page_bytes;
        load_codes<KW>(slab, lane, t.k[k]);
        load_codes<VW>(slab + at.v_codes, lane, t.v[k]);
        t.ks[k] = slab[at.k_scales + (D == 128 ? rb : rb >> 1) * kMxPage + col];
        t.vs[k] = *reinterpret_cast<const uint32_t*>(slab + at.v_scales + rb * (D / 8) + col / (512 / D) * 4);
      }
    };

    float m = -INFINITY, l = 0.f;
    f32x4 acc[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto compute = [&](Tile& t, int step) {
      const int left = ntok - (step * kWaves + wave) * KP * kMxPage;   // tokens from the step's first on
      float sv[4 * KP];
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        const float ks = mx_scale(t.ks[k]);
#pragma unroll
        for (int c = 0; c < NQ; ++c) {
          const u4 a = {pair<KB>(t.k[k], 4 * c, ks), pair<KB>(t.k[k], 4 * c + 1, ks), pair<KB>(t.k[k], 4 * c + 2, ks),
                        pair<KB>(t.k[k], 4 * c + 3, ks)};
#pragma unroll
          for (int part = 0; part < NPART; ++part) s = mfma(a, qv[part][c], s);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = s[i];
          if (p.cap > 0.f) x = p.cap * tanh_f32(x * p.scale);
          sv[4 * k + i] = k * kMxPage + 4 * rb + i < left ? x : -INFINITY;
        }
      }
      float mx = sv[0];
#pragma unroll
      for (int i = 1; i < 4 * KP; ++i) mx = fmaxf(mx, sv[i]);
      mx = swap32_max(swap16_max(mx));
      const bool raise = (mx - m) * cs > kSlack;
      if (__any(raise)) {
        const float m_new = raise ? mx : m;
        const float alpha = fast_exp2((m - m_new) * cs);   // 0 when m was -inf
        l = raise ? l * alpha : l;
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[n][r] = raise ? acc[n][r] * alpha : acc[n][r];
        m = m_new;
      }
      const float mref = m > -INFINITY ? m : 0.f;   // every score -inf so far: weights 0
      u4 pb[NPART];
#pragma unroll
      for (int i = 0; i < 4 * KP; ++i) sv[i] = fast_exp2((sv[i] - mref) * cs);
      l += ((sv[0] + sv[1]) + (sv[2] + sv[3])) + ((sv[4] + sv[5]) + (sv[6] + sv[7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (NPART == 1) {
          // bf16 outputs: P rounded to bf16, half a step of the output's own
          pb[0][i] = uint32_t(f32_to_bf16(sv[2 * i])) | (uint32_t(f32_to_bf16(sv[2 * i + 1])) << 16);
        } else {
          uint32_t a[3], b[3];
          split3(sv[2 * i], a);
          split3(sv[2 * i + 1], b);
#pragma unroll
          for (int s = 0; s < 3; ++s) pb[s][i] = join16(a[s], b[s]);
        }
      }
      if (left < KP * kMxPage) {   // rows past the retained length may hold anything: codes 0, scale 1
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          const int keep = min(max(left - k * kMxPage - 4 * rb, 0), 4);   // of the lane's 4 tokens
          const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
          t.vs[k] = (t.vs[k] & mask) | (0x7f7f7f7fu & ~mask);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            if (r < keep) continue;
            if constexpr (VW == 2) {
              t.v[k][r / 2] &= r % 2 ? 0x0000ffffu : 0xffff0000u;
            } else {
#pragma unroll
              for (int w = 0; w < VW / 4; ++w) t.v[k][r * (VW / 4) + w] = 0u;
            }
          }
        }
      }
      float vs[KP][4];
#pragma unroll
      for (int k = 0; k < KP; ++k)
#pragma unroll
        for (int r = 0; r < 4; ++r) vs[k][r] = mx_scale((t.vs[k] >> (8 * r)) & 0xffu);
#pragma unroll
      for (int i = 0; i < NV / 2; ++i) {   // dims 2i and 2i + 1 of the lane's sixteenth
        u4 a, b;
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          uint32_t w[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) w[r] = pair<VB>(t.v[k], r * (D / 32) + i, vs[k][r]);
          a[2 * k] = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u);
          a[2 * k + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u);
          b[2 * k] = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
          b[2 * k + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
        }
#pragma unroll
        for (int part = 0; part < NPART; ++part) {
          acc[2 * i] = mfma(a, pb[part], acc[2 * i]);
          acc[2 * i + 1] = mfma(b, pb[part], acc[2 * i + 1]);
        }
      }
    };

    Tile t0, t1;
    if (ns > 0) load(t0, 0);
    if (ns > 1) load(t1, 1);
    for (int s = 0; s < ns; s += 2) {
      compute(t0, s);
      if (s + 2 < ns) load(t0, s + 2);
      if (s + 1 < ns) {
        compute(t1, s + 1);
        if (s + 3 < ns) load(t1, s + 3);
      }
    }

    // the waves' states through LDS (a wave without a step has m = -inf and weight 0)
    l = swap32_sum(swap16_sum(l));
    if (col < G) {
      float* dst = sm_acc + (wave * G + col) * (D + kPad) + rb * (D / 4);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int n = 0; n < NV; n += 4)
          *reinterpret_cast<f32x4*>(dst + r * NV + n) = f32x4{acc[n][r], acc[n + 1][r], acc[n + 2][r], acc[n + 3][r]};
      if (rb == 0) {
        sm_m[wave * G + col] = m;
        sm_l[wave * G + col] = l;
      }
    }
    __syncthreads();   // every wave has read the live length too
    if (threadIdx.x == 0) {
      if (arow >= 0) p.live[(int64_t)item.b * p.live_stride + item.kv_head] = arow + 1;
      if (arow == -2 && p.append_full) *p.append_full = 1;
    }
    const bool merges = item.out_idx >= 0 && p.merge_counters;
    for (int o = threadIdx.x; o < G * (D / 4); o += kBlock) {
      const int g = o / (D / 4), c = o % (D / 4);
      float M = sm_m[g];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sm_m[w * G + g]);
      float L = 0.f;
      f32x4 A = {0.f, 0.f, 0.f, 0.f};
      const float mref = M > -INFINITY ? M : 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = fast_exp2((sm_m[w * G + g] - mref) * cs);
        L = fmaf(sm_l[w * G + g], f, L);
        const f32x4 x = *reinterpret_cast<const f32x4*>(sm_acc + (w * G + g) * (D + kPad) + 4 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) A[i] = fmaf(x[i], f, A[i]);
      }
      // no score above -inf: zeros, and an lse that loses against any other piece's
      const float div = L == 0.f ? 1.f : L;
      const f32x4 O = {A[0] / div, A[1] / div, A[2] / div, A[3] / div};
      const float lse = L == 0.f ? -FLT_MAX : M * (cs * kLn2) + logf(L);
      if (item.out_idx < 0) {
        const int64_t row = (int64_t)item.b * p.num_q_heads + item.kv_head * G + g;
        store4<T>(static_cast<T*>(p.out) + row * D + 4 * c, O);
        if (p.lse && c == 0) p.lse[row] = lse;
      } else {
        const int64_t row = (int64_t)item.out_idx * G + g;
        float* dst = p.part_o + row * D + 4 * c;
        if (merges) {
          // read in this launch by the workgroup that merges the unit, maybe on another XCD
          uint64_t* d64 = reinterpret_cast<uint64_t*>(dst);
          const auto word = [](float lo, float hi) {
            return (uint64_t)__float_as_uint(lo) | ((uint64_t)__float_as_uint(hi) << 32);
          };
          __hip_atomic_store(d64, word(O[0], O[1]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          __hip_atomic_store(d64 + 1, word(O[2], O[3]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (c == 0) __hip_atomic_store(p.part_lse + row, lse, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else {
          *reinterpret_cast<f32x4*>(dst) = O;
          if (c == 0) p.part_lse[row] = lse;
        }
      }
    }
    if (merges) {
      // The piece that arrives last merges its unit, with the recurrence and in the
      // order of the merge launch.  The partials were written with device-scope
      // stores and are complete (the wait) before the arrival is counted; they are
      // read with device-scope loads issued after the count came back.
      const int u = item.b * p.num_kv_heads + item.kv_head;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      const int splits = p.unit_splits[u];
      if (threadIdx.x == 0)
        *sm_flag = __hip_atomic_fetch_add(p.merge_counters + u, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __syncthreads();
      if (*sm_flag == splits - 1) {
        const int base = p.unit_partial_base[u];
        for (int o = threadIdx.x; o < G * (D / 4); o += kBlock) {
          const int g = o / (D / 4), c = o % (D / 4);
          float M = -INFINITY, L = 0.f;
          f32x4 A = {0.f, 0.f, 0.f, 0.f};
          constexpr int kBatch = 4;
          for (int i0 = 0; i0 < splits; i0 += kBatch) {
            float lv[kBatch];
            f32x4 ov[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
              const int64_t row = (int64_t)(base + min(i0 + j, splits - 1)) * G + g;
              lv[j] = __hip_atomic_load(p.part_lse + row, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
              const uint64_t* src = reinterpret_cast<const uint64_t*>(p.part_o + row * D + 4 * c);
              const uint64_t lo = __hip_atomic_load(src, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
              const uint64_t hi = __hip_atomic_load(src + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
              ov[j] = f32x4{__uint_as_float((uint32_t)lo), __uint_as_float((uint32_t)(lo >> 32)),
                            __uint_as_float((uint32_t)hi), __uint_as_float((uint32_t)(hi >> 32))};
            }
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
              const bool use = i0 + j < splits;
              const float mn = fmaxf(M, lv[j]);
              const float a = __expf(M - mn), w = __expf(lv[j] - mn);
              const float Ln = fmaf(L, a, w);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float An = fmaf(A[i], a, w * ov[j][i]);
                A[i] = use ? An : A[i];
              }
              L = use ? Ln : L;
              M = use ? mn : M;
            }
          }
          const int64_t row = (int64_t)item.b * p.num_q_heads + item.kv_head * G + g;
          store4<T>(static_cast<T*>(p.out) + row * D + 4 * c, f32x4{A[0] / L, A[1] / L, A[2] / L, A[3] / L});
          if (p.lse && c == 0) p.lse[row] = M + logf(L);
        }
        if (threadIdx.x == 0) __hip_atomic_store(p.merge_counters + u, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
    }
    __syncthreads();   // the states may be overwritten
  }
  if (p.timestamps && threadIdx.x == 0) {
    p.timestamps[2 * blockIdx.x] = t_start;
    p.timestamps[2 * blockIdx.x + 1] = it_begin < it_end ? __builtin_amdgcn_s_memrealtime() : t_start;
  }
}

using MxDecodeFn = void (*)(MxDecodeParams, const tg_work_item*, const int32_t*, const int32_t*);

template <typename T, int D>
MxDecodeFn pick_bits(int kb, int vb) {
  if (kb == 4) return vb == 4 ? &tg_decode_mx_kernel<T, D, 4, 4> : &tg_decode_mx_kernel<T, D, 4, 8>;
  return vb == 4 ? &tg_decode_mx_kernel<T, D, 8, 4> : &tg_decode_mx_kernel<T, D, 8, 8>;
}

MxDecodeFn pick_decode_mx(int dtype, int d, const tg_mx_format& f) {
  const int kb = tg::mx_bits(f.k_format), vb = tg::mx_bits(f.v_format);
  if (dtype == TG_F32) return d == 64 ? pick_bits<float, 64>(kb, vb) : pick_bits<float, 128>(kb, vb);
  return d == 64 ? pick_bits<uint16_t, 64>(kb, vb) : pick_bits<uint16_t, 128>(kb, vb);
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

}  // namespace

extern "C" {

int32_t tg_decode_mx_bins(const tg_geometry* geom, int32_t dtype, const tg_mx_format* format, int32_t device,
                          int32_t batch, int32_t layer, const int32_t* kv_len, int32_t* n_bins) {
  if (!n_bins) return tg::fail(TG_ERR_INVALID_ARG, "n_bins is NULL");
  if (int32_t rc = tg::check_mx(geom, format)) return rc;
  if (int32_t rc = tg::check_decode_shape(geom, dtype)) return rc;
  int64_t pages = 0;
  if (kv_len) {
    if (batch < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch must be >= 1");
    if (layer < 0 || layer >= geom->num_layers) return tg::fail(TG_ERR_INVALID_ARG, "layer %d out of range", layer);
    for (int64_t b = 0; b < batch; ++b)
      for (int h = 0; h < geom->num_kv_heads; ++h) {
        const int32_t n = kv_len[(b * geom->num_layers + layer) * geom->num_kv_heads + h];
        if (n < 1) return tg::fail(TG_ERR_INVALID_ARG, "kv_len %d of request %lld, head %d", n, (long long)b, h);
        pages += tg::ceil_div(n, kMxPage);
      }
  }
  const int gqa = geom->num_q_heads / geom->num_kv_heads;
  MxDecodeFn fn = pick_decode_mx(dtype, geom->head_dim, *format);
  int cus = 0, per_cu = 0, prev = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess)
    return tg::fail(TG_ERR_HIP, "hipDeviceGetAttribute failed for device %d", device);
  if (hipGetDevice(&prev) != hipSuccess) return tg::fail(TG_ERR_HIP, "hipGetDevice failed");
  if (prev != device && hipSetDevice(device) != hipSuccess) return tg::fail(TG_ERR_HIP, "hipSetDevice failed");
  const hipError_t e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, reinterpret_cast<const void*>(fn), kBlock,
                                                                    lds_floats(gqa, geom->head_dim) * sizeof(float));
  if (prev != device) (void)hipSetDevice(prev);
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "occupancy query failed: %s", hipGetErrorString(e));
  const int64_t most = (int64_t)per_cu * cus;
  const int64_t want = kv_len ? tg::ceil_div(pages, kWaves * KP) : most;
  *n_bins = (int32_t)(want < most ? want : most);
  return TG_OK;
}

int32_t tg_decode_mx(const tg_decode_args* a, const tg_mx_format* format, float softcap, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  if (int32_t rc = tg::check_mx(&a->geom, format)) return rc;
  if (int32_t rc = tg::check_decode_args(a, a->workspace, a->workspace_bytes)) return rc;
  if (softcap != 0.f) {
    if (int32_t rc = tg::check_softcap(softcap, a->sm_scale)) return rc;
  } else if (!(a->sm_scale >= 0.f) || !std::isfinite(a->sm_scale)) {
    return tg::fail(TG_ERR_INVALID_ARG, "sm_scale must be finite and >= 0");
  }
  const tg_geometry& g = a->geom;
  const int gqa = g.num_q_heads / g.num_kv_heads, d = g.head_dim;
  char* ws = static_cast<char*>(a->workspace);
  MxDecodeParams p;
  p.q = a->q;
  p.pool = static_cast<uint8_t*>(a->kv_pool);
  p.slab_bytes = mx_slab_bytes(d, tg::mx_bits(format->k_format), tg::mx_bits(format->v_format));
  p.page_bytes = (int64_t)g.heads_per_group * p.slab_bytes;
  p.num_q_heads = g.num_q_heads;
  p.num_kv_heads = g.num_kv_heads;
  p.n_bins = a->n_bins;
  p.gqa = gqa;
  p.unit_splits = a->unit_splits;
  p.unit_partial_base = a->unit_partial_base;
  p.out = a->out;
  p.lse = a->lse;
  p.part_o = reinterpret_cast<float*>(ws);
  p.part_lse = ws ? reinterpret_cast<float*>(ws + align256((size_t)a->num_partials * gqa * d * 4)) : nullptr;
  p.timestamps = a->timestamps;
  p.live = a->live_len ? a->live_len + (int64_t)a->layer * g.num_kv_heads : nullptr;
  p.live_stride = g.num_layers * g.num_kv_heads;
  p.append_k = static_cast<const u4*>(a->append_k);
  p.append_v = static_cast<const u4*>(a->append_v);
  p.append_full = a->append_full;
  p.cap = softcap;
  p.scale = a->sm_scale != 0.f ? a->sm_scale : 1.0f / std::sqrt((float)d);
  if (softcap > 0.f) p.scale /= softcap;
  const bool merges = a->merge_counters && a->num_partials > 0 && tg::decode_merges_in_one_chain(a);
  p.merge_counters = merges ? a->merge_counters : nullptr;
  if (a->num_items == 0) return TG_OK;
  hipLaunchKernelGGL(pick_decode_mx(a->dtype, d, *format), dim3(a->n_bins), dim3(kBlock),
                     lds_floats(gqa, d) * sizeof(float), static_cast<hipStream_t>(hip_stream), p, a->items, a->pt_pages,
                     a->bin_offsets);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  if (a->num_partials > 0 && !merges) return tg::launch_decode_merge(a, p.part_o, p.part_lse, hip_stream);
  return TG_OK;
}

}  // extern "C"
