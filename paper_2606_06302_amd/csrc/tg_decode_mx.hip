// Ragged paged split-KV decode attention over a quantised cache (tg_decode_mx).
//
// The plans, work items, partials and merge launch are tg_decode's; a bin is run by
// a workgroup of four waves.  The pages of its items, laid end to end, are cut into
// four equal ranges, and every wave runs its range by itself with an online softmax
// of its own; the waves meet once, at the end, where the up to three items that a
// cut goes through are joined through LDS.  What an item says (length, head, place of
// its page ids) is held a lane an item.  Page ids are a scalar load per step, made a
// step ahead; an item's queries are loaded when it starts.
//
// Data movement.  A page's slab (tg_mx.h) goes as it lies into a stage of the
// wave's ring in LDS with gfx950's global_load_lds (no registers, one wait counted
// by hand); one step is in flight while the one before is computed.
//
// Arithmetic.  gfx950 turns two codes into two bf16 numbers with their power-of-two
// scale in one full-rate instruction, exactly, and the products run on them with
// the query heads of the KV head as the 16 columns (columns past G repeat a real
// head and are never stored):
//   * S^T[16 tok][16 heads] = K q^T, D/32 x v_mfma_f32_16x16x32_bf16.  The lanes
//     of quarter j hold dims j D/4 .. of a row, so the k index runs through the
//     dims in that order, in K and in q alike.
//   * online softmax over the step's tokens; the 4 lanes of a column are combined
//     with the permlane swaps, and the maximum is raised only when a step exceeds
//     it by more than 2^8 in weight.
//   * O^T[16 dims][16 heads] += V^T P^T, D/16 products 32 (or 16) tokens deep:
//     tokens 4j .. 4j + 3 of a page for lane group j, which is where S^T leaves
//     them.  The codes pair dims, the operand pairs tokens: one byte permute each.
// With fp32 queries, q and P go in as three bf16 parts that hold their 24 bits.  With
// bf16 queries P goes in as two, 16 bits: rounded to bf16 alone it is the larger part
// of the result's error (32 requests of 8192 tokens in 4 bits, as a share of the
// result: 0.0022, in two parts 0.0017, the result's own rounding), and all of a small
// result where values cancel.  The second part costs 1 to 4 % of a call (there 24.2
// and 25.1 us); where a step is one page, both go into one product of twice the depth.
//
// Bound by memory where there is enough of it: 32 requests, gqa 4, 166568 pages in 8
// bits (704 MB) 116 us, 6.1 TB/s.  In 4 bits (362 MB) 69 us, 5.3 TB/s: there the
// compute is as near.  A step of two 4-bit pages of 128 dims (about 210 vector
// instructions and 24 matrix products) takes a SIMD with two waves on it 1640 cycles
// where the slabs stay in the caches, 6.5 TB/s over the chip; one 8-bit page 1025,
// 10 TB/s.  A wave waits 0.3 us for its bin, 0.8 for the items, 0.5 to 0.8 for the
// first page ids, 0.9 to 2.6 for the first slab; its results and the join take 0.5 to
// 1.3; the merge launch 2.5 to 5: 32 requests, 43233 pages (94 MB) 25 us.
// A step is two pages (one, of 8 + 8 bits and 128 dims) also where a wave has one: the
// second is then the first again, thrown away by the mask.  In bins of three pages wave
// 0 has none.
// Registers: 135 to 168 vector registers in bf16 (183 for 4 + 8 bits at 128 dims, two
// waves a SIMD), 155 to 168 in fp32 at 64 dims, 183 to 207 at 128; 27 to 36 scalar ones
// are kept in vector registers, none in memory.
// Measured on the way there, with P in one part: two barriers an item and headers
// loaded item by item 28 us, the waves' ranges 25.7, every read of a step ahead of its
// products 24.6; a merge inside the launch (counters, device-scope stores) 2 to 5 us
// more than the merge launch; 8 waves a workgroup and half the bins 27.  The
// block-scaled product on the 4-bit codes themselves adds up to only 12 bits of the
// largest term.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "tg_mx.h"

namespace {

using namespace tgd;

constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;
constexpr int kMaxGqa = 16;
constexpr int kPad = 4;        // floats between the heads' accumulators in LDS

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

#define TG_CONST __attribute__((address_space(4)))

struct MxDecodeParams {
  const void* q;
  uint8_t* pool;
  int64_t page_bytes;
  int32_t num_q_heads, num_kv_heads, gqa;
  void* out;
  float* lse;
  float* part_o;               // [num_partials][gqa][d]
  float* part_lse;             // [num_partials][gqa]
  uint64_t* timestamps;
  int32_t* live;               // live lengths of this layer, or NULL
  int32_t live_stride;
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

typedef short s16x4 __attribute__((ext_vector_type(4)));
// A product over the tokens of one page (2 words of 4 tokens' pairs) or two.
template <int PAGES>
__device__ __forceinline__ f32x4 mfma_pv(const uint32_t* a, const uint32_t* b, const f32x4& c) {
  if constexpr (PAGES == 2)
    return mfma(u4{a[0], a[1], a[2], a[3]}, u4{b[0], b[1], b[2], b[3]}, c);
  else
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, u2{a[0], a[1]}),
                                                     __builtin_bit_cast(s16x4, u2{b[0], b[1]}), c, 0, 0, 0);
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

// Two fp32 values as bf16, to the nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}
// Byte R of a word of scales as the scale, in one instruction.
template <int R>
__device__ __forceinline__ float byte_scale(uint32_t w) {
  uint32_t s;
  const uint32_t shift = 23;
  if constexpr (R == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(s) : "v"(shift), "v"(w));
  else if constexpr (R == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(s) : "v"(shift), "v"(w));
  else if constexpr (R == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(s) : "v"(shift), "v"(w));
  else
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(s) : "v"(shift), "v"(w));
  return __uint_as_float(s);
}

template <typename T>
__device__ __forceinline__ void store4(T* dst, const f32x4& v);
template <>
__device__ __forceinline__ void store4<float>(float* dst, const f32x4& v) { *reinterpret_cast<f32x4*>(dst) = v; }
template <>
__device__ __forceinline__ void store4<uint16_t>(uint16_t* dst, const f32x4& v) {
  *reinterpret_cast<u2*>(dst) = u2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// A wave's ring in LDS, by format: two steps of two pages, of one where two would
// take a CU's third workgroup (8-bit rows of 128 dims).  Two / three / four steps: 32
// requests in 4 bits 25.1 / 25.3 / 25.8 us, one long request of 64 dims 15.5 / 15.5 /
// 15.8; 64 requests in 8 bits, where three do not fit with three workgroups, 60.5 / 70.
template <int D, int KB, int VB>
struct Shape {
  static constexpr int kPages = KB + VB == 16 && D == 128 ? 1 : 2;   // of a step
  static constexpr int kSlab = mx_slab_bytes(D, KB, VB);
  // a slab comes in whole kilobytes of 16 bytes a lane and a rest of 4 or 16
  static constexpr int kFull = kSlab / 1024, kRest = kSlab % 1024;
  static constexpr bool kWideRest = kRest > 256;
  static constexpr int kStage = kPages * kSlab;
  static constexpr int kDma = kPages * (kFull + 1);                  // loads of a step
  static constexpr int kRing = 2;                                    // steps
  static constexpr int kRow = (D + kPad) * 4;                        // a head's accumulator in LDS
  // A wave's state of an item that it shares: accumulators, then (m, l) of every
  // head.  The last one takes the place of the ring; waves 1 to 3 may park one on
  // the way.
  __host__ __device__ static constexpr int state_bytes(int gqa) { return (gqa * (kRow + 8) + 15) / 16 * 16; }
  __host__ __device__ static constexpr int wave_bytes(int gqa) {
    return kRing * kStage > state_bytes(gqa) ? kRing * kStage : state_bytes(gqa);
  }
  static constexpr size_t lds_bytes(int gqa) { return kWaves * wave_bytes(gqa) + (kWaves - 1) * state_bytes(gqa); }
};

// 16 or 4 bytes a lane from base + offset into LDS at lds + 16 (4) * lane, past the
// caches' keeping: a step reads every byte of the cache once.  M0 is read one wait
// state after its write at the earliest, which neither the hardware nor, in inline
// assembly, the compiler sees to: hence the s_nop.
__device__ __forceinline__ void dma16(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt sc1" ::"v"(offset), "s"(base), "{m0}"(lds) : "memory");
}
__device__ __forceinline__ void dma4(const void* base, uint32_t offset, uint32_t lds) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dword %0, %1 nt sc1" ::"v"(offset), "s"(base), "{m0}"(lds) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* ptr) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)ptr));
}

__device__ __forceinline__ int lane_of(int x, int j) { return __builtin_amdgcn_readlane(x, j); }
__device__ __forceinline__ int64_t lane_of64(int64_t x, int j) {
  return (int64_t)(((uint64_t)(uint32_t)lane_of((int32_t)(x >> 32), j) << 32) | (uint32_t)lane_of((int32_t)x, j));
}

template <typename T, int D, int KB, int VB>
__global__ void __launch_bounds__(kBlock, sizeof(T) == 2 && !(D == 128 && KB == 4 && VB == 8) ? 3 : 2)
    tg_decode_mx_kernel(MxDecodeParams p, const tg_work_item* __restrict__ items_g, const int32_t* __restrict__ pt_g,
                        const int32_t* __restrict__ bin_offsets_g) {
  using S = Shape<D, KB, VB>;
  constexpr int E = Row16<T>::kElems;
  constexpr int NPART = sizeof(T) == 4 ? 3 : 1;   // bf16 parts of q
  constexpr int PPART = sizeof(T) == 4 ? 3 : 2;   // of P
  constexpr int KP = S::kPages;
  constexpr int KW = D * KB / 128, VW = D * VB / 128;
  constexpr int NQ = D / 32, NV = D / 16;
  constexpr int QC = D / 4 / E;                   // 16-byte chunks of q a lane
  constexpr int LPR = D / E;                      // 16-byte chunks of a row of T
  constexpr int R = S::kRing;
  constexpr MxParts at = mx_parts(D, KB, VB);
  // V's operands are made beside the products of q.k, where registers allow it
  constexpr bool kEarly = NPART == 1;
  constexpr float kSlack = 8.0f;
  extern __shared__ __align__(16) uint8_t lds[];

  const TG_CONST int32_t* const pt = (const TG_CONST int32_t*)pt_g;
  const TG_CONST int32_t* const bin_offsets = (const TG_CONST int32_t*)bin_offsets_g;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, rb = lane >> 4;
  const int G = p.gqa;
  const int hq = col < G ? col : col % G;
  const int park_bytes = S::state_bytes(G), wave_bytes = S::wave_bytes(G);
  uint8_t* const ring = lds + wave * wave_bytes;
  uint8_t* const parks = lds + kWaves * wave_bytes;
  const uint32_t ring_lds = lds_address(ring);
  const uint64_t t_start = __builtin_amdgcn_s_memrealtime();
  const int it_begin = bin_offsets[blockIdx.x], it_end = bin_offsets[blockIdx.x + 1];
  if (it_begin >= it_end) {
    if (p.timestamps && threadIdx.x == 0) p.timestamps[2 * blockIdx.x] = p.timestamps[2 * blockIdx.x + 1] = t_start;
    return;
  }
  const float cs = p.cap > 0.f ? kLog2e : p.scale * kLog2e;   // log2 units per unit of (capped) score

  // four dims of a head's result of an item: the output, or this piece's partial
  auto write4 = [&](int b, int h, int out_idx, int g, int e, const f32x4& O, float lse) {
    if (out_idx < 0) {
      const int64_t row = (int64_t)b * p.num_q_heads + h * G + g;
      store4<T>(static_cast<T*>(p.out) + row * D + e, O);
      if (p.lse && e == 0) p.lse[row] = lse;
      return;
    }
    const int64_t row = (int64_t)out_idx * G + g;
    float* dst = p.part_o + row * D + e;
    *reinterpret_cast<f32x4*>(dst) = O;
    if (e == 0) p.part_lse[row] = lse;
  };
  // no score above -inf: zeros, and an lse that loses against any other piece's
  auto lse_of = [&](float m, float l) { return l == 0.f ? -FLT_MAX : fmaf(m, cs * kLn2, __builtin_amdgcn_logf(l) * kLn2); };

  // the items of the bin, up to 64 at a time, one a lane
  for (int chunk = it_begin; chunk < it_end; chunk += 64) {
    const int n_items = min(64, it_end - chunk);
    int64_t h_first;         // of the item's page ids
    int h_ntok, h_slot, h_b, h_head, h_out, h_arow = -1, h_end;   // arow: the entry that takes the new token, or < 0
    {
      const tg_work_item im = items_g[chunk + min(lane, n_items - 1)];
      int end = im.tok_end;
      if (end < 0) {
        const int n = p.live ? p.live[(int64_t)im.b * p.live_stride + im.kv_head] : -end;
        end = resolve_open(im.tok_begin, im.tok_end, n, p.append_k != nullptr, &h_arow);
      }
      h_first = im.pt_base + im.tok_begin / kMxPage;
      h_ntok = end - im.tok_begin;
      h_slot = im.slot;
      h_b = im.b;
      h_head = im.kv_head;
      h_out = im.out_idx;
      h_end = lane < n_items ? (h_ntok + kMxPage - 1) / kMxPage : 0;   // pages, then where they end
      h_end = wave_inclusive_sum(h_end);
    }
    const int pages = lane_of(h_end, 63);
    auto cut = [&](int w) { return (int)((int64_t)pages * w >> 2); };
    const int f0 = cut(wave), f1 = cut(wave + 1);
    auto begin_of = [&](int it) { return it > 0 ? lane_of(h_end, it - 1) : 0; };
    const int it0 = __builtin_ctzll(__ballot(h_end > f0) | (1ull << 63));   // the item of page f0

    // the loads run ahead of the products, over all items
    int d_it = it0, d_page = f0 - begin_of(it0), d_left = f1 - f0;   // d_left: pages to request
    int d_np = lane_of(h_end, it0) - begin_of(it0);
    int64_t d_first = lane_of64(h_first, it0);
    const uint8_t* d_slabs = p.pool + (int64_t)lane_of(h_slot, it0) * S::kSlab;
    struct Ids {
      int32_t v[KP];
    } d_id = {};
    auto page_ids = [&] {
      const int last = min(d_np, d_page + d_left) - 1;
#pragma unroll
      for (int k = 0; k < KP; ++k) d_id.v[k] = pt[d_first + min(d_page + k, last)];
    };
    auto issue = [&](int to) {   // one step, and on to the next
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        const uint8_t* slab = d_slabs + (int64_t)d_id.v[k] * p.page_bytes;
        const uint32_t dst = ring_lds + to * S::kStage + k * S::kSlab;
#pragma unroll
        for (int j = 0; j < S::kFull; ++j) dma16(slab + j * 1024, lane * 16, dst + j * 1024);
        if constexpr (S::kWideRest) {
          if (lane < S::kRest / 16) dma16(slab + S::kFull * 1024, lane * 16, dst + S::kFull * 1024);
        } else {
          if (lane < S::kRest / 4) dma4(slab + S::kFull * 1024, lane * 4, dst + S::kFull * 1024);
        }
      }
      const int took = min(KP, min(d_np - d_page, d_left));
      d_page += took;
      d_left -= took;
      if (d_left <= 0) return;
      if (d_page >= d_np) {
        ++d_it;
        d_page = 0;
        d_np = lane_of(h_end, d_it) - lane_of(h_end, d_it - 1);
        d_first = lane_of64(h_first, d_it);
        d_slabs = p.pool + (int64_t)lane_of(h_slot, d_it) * S::kSlab;
      }
      page_ids();
    };
    int it = it0, slot = 0;   // slot: of the ring, of the step computed next
    float m = -INFINITY, l = 0.f;
    f32x4 acc[NV];
    if (f0 < f1) {
      page_ids();
#pragma unroll
      for (int r = 0; r < R - 1; ++r)
        if (d_left > 0) issue(r);
    }
    for (int at_page = f0; at_page < f1; ++it) {
      const int first_page = at_page - begin_of(it);   // of the item
      const int np = lane_of(h_end, it) - begin_of(it);
      const int stop = min(np, first_page + f1 - at_page);
      const int ntok = lane_of(h_ntok, it), arow = lane_of(h_arow, it);

      // waiting for the queries waits for the step in flight too, which is needed next
      // (queries fetched an item ahead, through LDS, took the same time)
      u4 qv[NPART][NQ], tok = {};
      {
        const int b = lane_of(h_b, it), h = lane_of(h_head, it);
        const u4* q = static_cast<const u4*>(p.q) + ((int64_t)b * p.num_q_heads + h * G + hq) * LPR + rb * QC;
        u4 x[QC];
#pragma unroll
        for (int i = 0; i < QC; ++i) x[i] = q[i];
        if (arow >= 0 && lane < 2 * LPR) {
          const int64_t row = ((int64_t)b * p.num_kv_heads + h) * LPR;
          tok = lane < LPR ? p.append_k[row + lane] : p.append_v[row + lane - LPR];
        }
#pragma unroll
        for (int c = 0; c < NQ; ++c) {
          if constexpr (NPART == 1) {
            qv[0][c] = x[c];
          } else {
            float y[8];
            Row16<float>::unpack(x[2 * c], y);
            Row16<float>::unpack(x[2 * c + 1], y + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t a[3], b[3];
              split3(y[2 * i], a);
              split3(y[2 * i + 1], b);
#pragma unroll
              for (int s = 0; s < 3; ++s) qv[s][c][i] = join16(a[s], b[s]);
            }
          }
        }
      }
      m = -INFINITY;
      l = 0.f;
#pragma unroll
      for (int n = 0; n < NV; ++n) acc[n] = f32x4{0.f, 0.f, 0.f, 0.f};

      for (int page = first_page; page < stop; page += KP, slot = slot + 1 < R ? slot + 1 : 0) {
        if (d_left > 0) {   // R - 1 steps stay in flight
          issue(slot > 0 ? slot - 1 : R - 1);
          wait_vmcnt<S::kDma * (R - 1)>();
        } else {
          wait_vmcnt<0>();
        }
        uint8_t* const stage = ring + slot * S::kStage;
        const int left = min(ntok - page * kMxPage, (stop - page) * kMxPage);   // tokens from the step's first on

        // the new token, the item's last entry: quantised into its place in the pool, and in the stage
        if (arow >= 0 && stop == np && page + KP >= np) {
          const int t = arow % kMxPage, k = np - 1 - page;
          uint8_t* slab = p.pool + (int64_t)pt[lane_of64(h_first, it) + np - 1] * p.page_bytes +
                          (int64_t)lane_of(h_slot, it) * S::kSlab;
          if (lane < 2 * LPR) {
            const bool is_v = lane >= LPR;
            const int e = lane % LPR * E;
            uint32_t scale;
            uint8_t* const mine = stage + k * S::kSlab;
            if (is_v) {
              const u2 c = mx_quantise<T>(tok, VB, &scale);
              mx_store<E>(slab + at.v_codes, slab + at.v_scales, t, e, D, VB, true, c, scale);
              mx_store<E>(mine + at.v_codes, mine + at.v_scales, t, e, D, VB, true, c, scale);
            } else {
              const u2 c = mx_quantise<T>(tok, KB, &scale);
              mx_store<E>(slab, slab + at.k_scales, t, e, D, KB, false, c, scale);
              mx_store<E>(mine, mine + at.k_scales, t, e, D, KB, false, c, scale);
            }
          }
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
          __builtin_amdgcn_wave_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }

        // every read of the step goes out before its first product
        uint32_t kc[KP][KW], vc[KP][VW], vw[KP];
        float ks[KP];
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          const uint8_t* slab = stage + k * S::kSlab;
          load_codes<KW>(slab, lane, kc[k]);
          ks[k] = mx_scale(slab[at.k_scales + (D == 128 ? rb : rb >> 1) * kMxPage + col]);
        }
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          const uint8_t* slab = stage + k * S::kSlab;
          load_codes<VW>(slab + at.v_codes, lane, vc[k]);
          vw[k] = *reinterpret_cast<const uint32_t*>(slab + at.v_scales + rb * (D / 8) + col / (512 / D) * 4);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (left < KP * kMxPage) {   // rows past the retained length may hold anything: codes 0, scale 1
#pragma unroll
          for (int k = 0; k < KP; ++k) {
            const int keep = min(max(left - k * kMxPage - 4 * rb, 0), 4);   // of the lane's 4 tokens
            const uint32_t mask = keep == 4 ? ~0u : (1u << (8 * keep)) - 1u;
            vw[k] = (vw[k] & mask) | (0x7f7f7f7fu & ~mask);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const bool drop = r >= keep;
              if constexpr (VW == 2) {
                vc[k][r / 2] &= drop ? (r % 2 ? 0x0000ffffu : 0xffff0000u) : ~0u;
              } else {
#pragma unroll
                for (int w = 0; w < VW / 4; ++w) vc[k][r * (VW / 4) + w] = drop ? 0u : vc[k][r * (VW / 4) + w];
              }
            }
          }
        }

        f32x4 s[KP];
#pragma unroll
        for (int k = 0; k < KP; ++k) s[k] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NQ; ++c)
#pragma unroll
          for (int k = 0; k < KP; ++k) {
            const u4 a = {pair<KB>(kc[k], 4 * c, ks[k]), pair<KB>(kc[k], 4 * c + 1, ks[k]),
                          pair<KB>(kc[k], 4 * c + 2, ks[k]), pair<KB>(kc[k], 4 * c + 3, ks[k])};
#pragma unroll
            for (int part = 0; part < NPART; ++part) s[k] = mfma(a, qv[part][c], s[k]);
          }

        // V's operands: dims 2i and 2i + 1 of the lane's sixteenth, pairs of tokens
        float vs[KP][4];
#pragma unroll
        for (int k = 0; k < KP; ++k) {
          vs[k][0] = byte_scale<0>(vw[k]);
          vs[k][1] = byte_scale<1>(vw[k]);
          vs[k][2] = byte_scale<2>(vw[k]);
          vs[k][3] = byte_scale<3>(vw[k]);
        }
        auto v_operands = [&](int i, uint32_t* a, uint32_t* b) {
#pragma unroll
          for (int k = 0; k < KP; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) w[r] = pair<VB>(vc[k], r * (D / 32) + i, vs[k][r]);
            a[2 * k] = __builtin_amdgcn_perm(w[1], w[0], 0x05040100u);
            a[2 * k + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x05040100u);
            b[2 * k] = __builtin_amdgcn_perm(w[1], w[0], 0x07060302u);
            b[2 * k + 1] = __builtin_amdgcn_perm(w[3], w[2], 0x07060302u);
          }
        };
        uint32_t va[NV / 2][2 * KP], vb[NV / 2][2 * KP];
        if constexpr (kEarly) {
#pragma unroll
          for (int i = 0; i < NV / 2; ++i) {
            v_operands(i, va[i], vb[i]);
#pragma unroll
            for (int j = 0; j < 2 * KP; ++j) asm volatile("" : "+v"(va[i][j]), "+v"(vb[i][j]));   // here, not behind the branches
          }
        }
        float sv[4 * KP];
#pragma unroll
        for (int i = 0; i < 4 * KP; ++i) sv[i] = s[i / 4][i % 4];
        if (p.cap > 0.f) {
#pragma unroll
          for (int i = 0; i < 4 * KP; ++i) sv[i] = p.cap * tanh_f32(sv[i] * p.scale);
        }
        if (left < KP * kMxPage) {
#pragma unroll
          for (int i = 0; i < 4 * KP; ++i) sv[i] = i / 4 * kMxPage + 4 * rb + i % 4 < left ? sv[i] : -INFINITY;
        }
        float mx = sv[0];
#pragma unroll
        for (int i = 1; i < 4 * KP; ++i) mx = fmaxf(mx, sv[i]);
        mx = swap32_max(swap16_max(mx));
        const bool raise = (mx - m) * cs > kSlack;
        if (__any(raise)) {
          const float m_new = raise ? mx : m;
          const float alpha = raise ? fast_exp2((m - m_new) * cs) : 1.f;   // 0 when m was -inf
          l *= alpha;
          m = m_new;
#pragma unroll
          for (int n = 0; n < NV; ++n) acc[n] *= alpha;
        }
        const float mref = m > -INFINITY ? m : 0.f;   // every score -inf so far: weights 0
#pragma unroll
        for (int i = 0; i < 4 * KP; ++i) {
          // fp32: relative to m itself and not to a rounded m cs, as the states are weighted by m
          if constexpr (NPART == 1) sv[i] = fast_exp2(fmaf(sv[i], cs, -mref * cs));
          else sv[i] = fast_exp2((sv[i] - mref) * cs);
        }
        float sum = (sv[0] + sv[1]) + (sv[2] + sv[3]);
        if constexpr (KP == 2) sum += (sv[4] + sv[5]) + (sv[6] + sv[7]);
        l += sum;
        uint32_t pb[PPART][2 * KP];
#pragma unroll
        for (int i = 0; i < 2 * KP; ++i) {
          if constexpr (PPART == 2) {
            // the first part cut, 2^-7 of P left at most, the second rounded: off by 2^-16 of P
            const uint32_t x0 = __float_as_uint(sv[2 * i]), x1 = __float_as_uint(sv[2 * i + 1]);
            pb[0][i] = join16(x0, x1);
            pb[1][i] = pack_bf16(sv[2 * i] - __uint_as_float(x0 & 0xffff0000u), sv[2 * i + 1] - __uint_as_float(x1 & 0xffff0000u));
          } else {
            uint32_t a[3], b[3];
            split3(sv[2 * i], a);
            split3(sv[2 * i + 1], b);
#pragma unroll
            for (int s = 0; s < 3; ++s) pb[s][i] = join16(a[s], b[s]);
          }
        }
#pragma unroll
        for (int i = 0; i < NV / 2; ++i) {
          uint32_t a[2 * KP], b[2 * KP];
          if constexpr (!kEarly) v_operands(i, a, b);
#pragma unroll
          for (int part = 0; part < PPART; ++part) {
            if constexpr (KP == 1 && PPART == 2) {   // both parts in one product of twice the depth
              if (part > 0) break;
              const uint32_t a2[4] = {va[i][0], va[i][1], va[i][0], va[i][1]};
              const uint32_t b2[4] = {vb[i][0], vb[i][1], vb[i][0], vb[i][1]};
              const uint32_t w[4] = {pb[0][0], pb[0][1], pb[1][0], pb[1][1]};
              acc[2 * i] = mfma_pv<2>(a2, w, acc[2 * i]);
              acc[2 * i + 1] = mfma_pv<2>(b2, w, acc[2 * i + 1]);
            } else {
              acc[2 * i] = mfma_pv<KP>(kEarly ? va[i] : a, pb[part], acc[2 * i]);
              acc[2 * i + 1] = mfma_pv<KP>(kEarly ? vb[i] : b, pb[part], acc[2 * i + 1]);
            }
          }
        }
      }
      at_page += stop - first_page;

      l = swap32_sum(swap16_sum(l));
      const bool whole = first_page == 0 && stop == np;
      if (whole) {
        if (col < G) {
          const float inv = __builtin_amdgcn_rcpf(l == 0.f ? 1.f : l);
          const float lse = lse_of(m, l);
          const int b = lane_of(h_b, it), h = lane_of(h_head, it), out_idx = lane_of(h_out, it);
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int n = 0; n < NV; n += 4)
              write4(b, h, out_idx, col, rb * (D / 4) + r * NV + n,
                     f32x4{acc[n][r] * inv, acc[n + 1][r] * inv, acc[n + 2][r] * inv, acc[n + 3][r] * inv}, lse);
        }
      } else if (col < G) {
        // a shared item's state: parked if the wave goes on (its first item then, so it is
        // not wave 0), else where its ring was (no load is in flight then)
        uint8_t* state = at_page < f1 ? parks + (wave - 1) * park_bytes : ring;
        float* dst = reinterpret_cast<float*>(state) + col * (D + kPad) + rb * (D / 4);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int n = 0; n < NV; n += 4)
            *reinterpret_cast<f32x4*>(dst + r * NV + n) = f32x4{acc[n][r], acc[n + 1][r], acc[n + 2][r], acc[n + 3][r]};
        if (rb == 0) {
          float* ml = reinterpret_cast<float*>(state + G * S::kRow) + 2 * col;
          ml[0] = m;
          ml[1] = l;
        }
      }
    }
    __syncthreads();

    // items that a cut goes through
#pragma unroll 1
    for (int w0 = 1, last_it = -1; w0 < kWaves; ++w0) {
      const int c = cut(w0);
      if (c >= pages) break;
      const int j = __builtin_ctzll(__ballot(h_end > c) | (1ull << 63));   // the item of page c
      if (c == begin_of(j) || j == last_it) continue;
      last_it = j;
      const int lo = begin_of(j), hi = lane_of(h_end, j);
      const int b = lane_of(h_b, j), h = lane_of(h_head, j), out_idx = lane_of(h_out, j);
      // where every wave left its part of the item, with its last item or parked; a wave
      // without a part is read all the same (the reads go out together) and not used
      uint32_t at_state[kWaves];
      int parts = 0;   // bit w: wave w has one
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        parts |= (cut(w) < hi && cut(w + 1) > lo && cut(w) < cut(w + 1)) << w;
        at_state[w] = w == 0 || cut(w + 1) <= hi ? w * wave_bytes : kWaves * wave_bytes + (w - 1) * park_bytes;
      }
#pragma unroll 1
      for (int o = threadIdx.x; o < G * (D / 4); o += kBlock) {
        const int g = o / (D / 4), e = o % (D / 4) * 4;
        int mine = parts;
        asm volatile("" : "+v"(mine));   // one body, not one for every set of waves: it is fetched cold
        float ms[kWaves], ls[kWaves];
        f32x4 x[kWaves];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float* ml = reinterpret_cast<const float*>(lds + at_state[w] + G * S::kRow) + 2 * g;
          ms[w] = ml[0];
          ls[w] = ml[1];
          x[w] = *reinterpret_cast<const f32x4*>(lds + at_state[w] + g * S::kRow + e * 4);
        }
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, mine >> w & 1 ? ms[w] : -INFINITY);
        f32x4 A = {0.f, 0.f, 0.f, 0.f};
        const float mref = M > -INFINITY ? M : 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const bool has = mine >> w & 1;
          const float f = has ? fast_exp2((ms[w] - mref) * cs) : 0.f;
          L = fmaf(has ? ls[w] : 0.f, f, L);
#pragma unroll
          for (int i = 0; i < 4; ++i) A[i] = fmaf(has ? x[w][i] : 0.f, f, A[i]);
        }
        const float inv = __builtin_amdgcn_rcpf(L == 0.f ? 1.f : L);
        write4(b, h, out_idx, g, e, f32x4{A[0] * inv, A[1] * inv, A[2] * inv, A[3] * inv}, lse_of(M, L));
      }
    }
    if (wave == 0 && lane < n_items) {   // every wave has read the lengths
      if (h_arow >= 0) p.live[(int64_t)h_b * p.live_stride + h_head] = h_arow + 1;
      if (h_arow == -2 && p.append_full) *p.append_full = 1;
    }
    if (chunk + 64 < it_end) __syncthreads();   // the states have been read
  }

  if (p.timestamps && threadIdx.x == 0) {
    p.timestamps[2 * blockIdx.x] = t_start;
    p.timestamps[2 * blockIdx.x + 1] = __builtin_amdgcn_s_memrealtime();
  }
}

using MxDecodeFn = void (*)(MxDecodeParams, const tg_work_item*, const int32_t*, const int32_t*);

struct Picked {
  MxDecodeFn fn;
  size_t lds;   // bytes of a workgroup
};

template <typename T, int D, int KB, int VB>
Picked picked(int gqa) {
  return {&tg_decode_mx_kernel<T, D, KB, VB>, Shape<D, KB, VB>::lds_bytes(gqa)};
}

template <typename T, int D>
Picked pick_bits(int kb, int vb, int gqa) {
  if (kb == 4) return vb == 4 ? picked<T, D, 4, 4>(gqa) : picked<T, D, 4, 8>(gqa);
  return vb == 4 ? picked<T, D, 8, 4>(gqa) : picked<T, D, 8, 8>(gqa);
}

Picked pick_decode_mx(int dtype, const tg_geometry& g, const tg_mx_format& f) {
  const int kb = tg::mx_bits(f.k_format), vb = tg::mx_bits(f.v_format), gqa = g.num_q_heads / g.num_kv_heads;
  if (dtype == TG_F32) return g.head_dim == 64 ? pick_bits<float, 64>(kb, vb, gqa) : pick_bits<float, 128>(kb, vb, gqa);
  return g.head_dim == 64 ? pick_bits<uint16_t, 64>(kb, vb, gqa) : pick_bits<uint16_t, 128>(kb, vb, gqa);
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
  const Picked k = pick_decode_mx(dtype, *geom, *format);
  int cus = 0, lds = 0, per_cu = 0, prev = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess ||
      hipDeviceGetAttribute(&lds, hipDeviceAttributeMaxSharedMemoryPerMultiprocessor, device) != hipSuccess)
    return tg::fail(TG_ERR_HIP, "hipDeviceGetAttribute failed for device %d", device);
  if (hipGetDevice(&prev) != hipSuccess) return tg::fail(TG_ERR_HIP, "hipGetDevice failed");
  if (prev != device && hipSetDevice(device) != hipSuccess) return tg::fail(TG_ERR_HIP, "hipSetDevice failed");
  const hipError_t e =
      hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, reinterpret_cast<const void*>(k.fn), kBlock, k.lds);
  if (prev != device) (void)hipSetDevice(prev);
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "occupancy query failed: %s", hipGetErrorString(e));
  // The query counts bytes, a CU gives its LDS out in units of 1280: of 768 workgroups of 54464 bytes (8 and 4 bits,
  // head_dim 128, gqa 2) a third starts when others have ended, of 52832 bytes (gqa 1) all start together.
  const int fit = (int)(lds / (tg::ceil_div((int64_t)k.lds, 1280) * 1280));
  if (fit < per_cu) per_cu = fit;
  // Two workgroups a CU, of three pages a bin at least: 40 ragged layers of 22 to 34000 pages at 16 / 8 / 4 / 3
  // / 2 / 1 pages a bin take 1.28 / 1.16 / 1.04 / 1.03 / 1.03 / 1.04 times their best.  Three a CU, where they fit
  // together, for 80 pages a bin and more.  32 requests of 8 heads, three in turn with two, as a share of the time of
  // two: from 63000 to 188000 pages 0.93 to 1.03 in 4 bits at head_dim 64, 0.94 to 0.98 with a cap or fp32 queries,
  // 1.00 to 1.04 at 128 without and 0.94 to 0.98 with a cap; 0.97 to 1.04 in 8 bits; 21000 to 60000 pages 0.96 to
  // 1.08.  More than three is behind everywhere.
  const int64_t three = 3 * (int64_t)cus, two = (per_cu < 2 ? per_cu : 2) * (int64_t)cus;
  const bool many = kv_len && per_cu >= 3 && pages >= 80 * three;
  const int64_t few = kv_len ? tg::ceil_div(pages, 3) : two;
  *n_bins = (int32_t)(many ? three : few < two ? few : two);
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
  p.page_bytes = (int64_t)tg_mx_page_bytes(&g, format);
  p.num_q_heads = g.num_q_heads;
  p.num_kv_heads = g.num_kv_heads;
  p.gqa = gqa;
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
  if (a->num_items == 0) return TG_OK;
  const Picked k = pick_decode_mx(a->dtype, g, *format);
  hipLaunchKernelGGL(k.fn, dim3(a->n_bins), dim3(kBlock), k.lds, static_cast<hipStream_t>(hip_stream), p, a->items,
                     a->pt_pages, a->bin_offsets);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "decode launch failed: %s", hipGetErrorString(e));
  if (a->num_partials > 0) return tg::launch_decode_merge(a, p.part_o, p.part_lse, hip_stream);
  return TG_OK;
}

}  // extern "C"
