// The quantised page layout and the quantiser, shared by the kernels that write,
// read back and attend over a cache of microscaled rows (tg_mx_format).
//
// A page of a group holds heads_per_group slabs, one a head:
//   [K codes][V codes][K scales][V scales]
// for 16 tokens of d dims.  The codes lie as the 64 lanes of a wave take them for
// the matrix products, so that the attention's loads are the slab in order and
// its operands need no movement between lanes:
//   K: lane 16 j + t holds quarter j of token t's row (the k index of q.k);
//   V: lane 16 j + c holds sixteenth c of the rows of tokens 4j .. 4j + 3 (the k
//      index of p.v is the token, 4j .. 4j + 3 for lane group j, as the scores
//      come out of q.k).
// A lane's codes are d / 4 elements, in chunks of up to 16 bytes that lie 64
// chunks apart.  Scales: K [group][token], V [j][group][token of 4j .. 4j + 3],
// one word a lane.
#pragma once
#include "tg_device.h"
#include "tg_internal.h"

namespace tgd {

constexpr int kMxPage = 16;    // tokens of a page
constexpr int kMxGroup = 32;   // dims that share a scale

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

// Byte offsets inside a slab (bits: of the part's format, 4 or 8).
__host__ __device__ constexpr int mx_codes_bytes(int d, int bits) { return kMxPage * d * bits / 8; }
__host__ __device__ constexpr int mx_scales_bytes(int d) { return kMxPage * d / kMxGroup; }
__host__ __device__ constexpr int mx_slab_bytes(int d, int kb, int vb) {
  return mx_codes_bytes(d, kb) + mx_codes_bytes(d, vb) + 2 * mx_scales_bytes(d);
}
struct MxParts {
  int v_codes, k_scales, v_scales;
};
__host__ __device__ constexpr MxParts mx_parts(int d, int kb, int vb) {
  const int v = mx_codes_bytes(d, kb), s = v + mx_codes_bytes(d, vb);
  return {v, s, s + mx_scales_bytes(d)};
}

// Byte of element e of token t among the codes of its part.  Elements that
// follow e up to the end of its run (mx_run) have the bytes behind it.  d and
// bits are powers of two: shifts, as a division costs more than the quantiser.
__device__ __forceinline__ int mx_code_at(int t, int e, int d, int bits, bool is_v) {
  const int ld = d == 128 ? 7 : 6, pack = bits == 4 ? 1 : 0;   // log2 of d, of codes in a byte
  const int lane = is_v ? (t >> 2) * 16 + (e >> (ld - 4)) : (e >> (ld - 2)) * 16 + t;
  const int el = is_v ? ((t & 3) << (ld - 4)) + (e & ((1 << (ld - 4)) - 1)) : e & ((1 << (ld - 2)) - 1);
  const int byte = el >> pack, chunk = min(4, ld - 2 - pack);  // log2 of a chunk's bytes
  return ((byte >> chunk) << (chunk + 6)) + (lane << chunk) + (byte & ((1 << chunk) - 1));
}
// Elements of a row that lie in consecutive bytes: at least this many, aligned.
__device__ __forceinline__ int mx_run(int d, bool is_v) { return is_v && d == 64 ? 4 : 8; }
__device__ __forceinline__ int mx_scale_at(int t, int group, int d, bool is_v) {
  return is_v ? (t >> 2) * (d == 128 ? 16 : 8) + group * 4 + (t & 3) : group * kMxPage + t;
}

// The 16 bytes of a row that a lane holds, as fp32.
template <typename T>
struct Row16;
template <>
struct Row16<uint16_t> {
  static constexpr int kElems = 8;
  __device__ __forceinline__ static void unpack(const u4& v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo(v[i]);
      f[2 * i + 1] = bf16_hi(v[i]);
    }
  }
};
template <>
struct Row16<float> {
  static constexpr int kElems = 4;
  __device__ __forceinline__ static void unpack(const u4& v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false));
}

// Codes of a lane's E elements (the lanes of a group of 32 lie side by side and
// call this together): the scale is 2^e, e the least integer with max|x| <= top
// 2^e, top 7 (4 bits) or 464 (8 bits), the midpoint between the largest value and
// the step that would follow; an element is x / 2^e to the nearest, ties to even,
// at most the largest.  All of it is exact but the one rounding of the element,
// so it depends on nothing but the input.  A group with a NaN or an infinity gets
// scale byte 255 and codes 0, which stand for NaN.
// Returns the codes, E * bits / 8 bytes, low bytes first, and *scale, e + 127.
template <int E>
__device__ __forceinline__ u2 mx_quantise(const float* x, int bits, uint32_t* scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);   // as integers: NaN above infinity
  top = dpp_max_u32<kQuadXor1>(top);
  top = dpp_max_u32<kQuadXor2>(top);
  if constexpr (E == 4) top = dpp_max_u32<kRowHalfMirror>(top);
  const int expo = (int)(top >> 23), frac = (int)(top & 0x7fffffu);
  const bool finite = top < 0x7f800000u;
  u2 r = {0u, 0u};
  if (bits == 4) {
    // 7 = 1.75 * 2^2; within [-125, 125] every value is a normal bf16 number
    const int e = min(max(expo - 2 + (frac > 0x600000), 2), 252);
    const float s = __uint_as_float((uint32_t)e << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    if constexpr (E == 8) {
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    }
    r.x = finite ? c : 0u;
    *scale = finite ? (uint32_t)e : 255u;
  } else {
    // 464 = 1.8125 * 2^8; [-117, 119]
    const int e = min(max(expo - 8 + (frac > 0x680000), 10), 246);
    const float s = __uint_as_float((uint32_t)e << 23);
    const float most = 448.f * s;   // the conversion makes NaN of what rounds past 448
    float y[E];
#pragma unroll
    for (int i = 0; i < E; ++i) y[i] = fminf(fmaxf(x[i], -most), most);
#pragma unroll
    for (int w = 0; w < E / 4; ++w) {
      s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * w], y[4 * w + 1], s, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, y[4 * w + 2], y[4 * w + 3], s, true);
      r[w] = finite ? __builtin_bit_cast(uint32_t, c) : 0u;
    }
    *scale = finite ? (uint32_t)e : 255u;
  }
  return r;
}

// Stores a lane's E elements, from element e0 of token t on, into a part's codes
// and, from the first lane of a group, its scale.
template <int E>
__device__ __forceinline__ void mx_store(uint8_t* codes, uint8_t* scales, int t, int e0, int d, int bits, bool is_v,
                                         const u2& c, uint32_t scale) {
  uint8_t* at = codes + mx_code_at(t, e0, d, bits, is_v);
  if (mx_run(d, is_v) >= E) {
    if constexpr (E == 8) {
      if (bits == 8) *reinterpret_cast<u2*>(at) = c;
      else *reinterpret_cast<uint32_t*>(at) = c.x;
    } else {
      if (bits == 8) *reinterpret_cast<uint32_t*>(at) = c.x;
      else *reinterpret_cast<uint16_t*>(at) = (uint16_t)c.x;
    }
  } else {   // two runs of 4
    uint8_t* next = codes + mx_code_at(t, e0 + 4, d, bits, is_v);
    if (bits == 8) {
      *reinterpret_cast<uint32_t*>(at) = c.x;
      *reinterpret_cast<uint32_t*>(next) = c.y;
    } else {
      *reinterpret_cast<uint16_t*>(at) = (uint16_t)c.x;
      *reinterpret_cast<uint16_t*>(next) = (uint16_t)(c.x >> 16);
    }
  }
  if (e0 % kMxGroup == 0) scales[mx_scale_at(t, e0 / kMxGroup, d, is_v)] = (uint8_t)scale;
}

// The same elements read back, without their scale: E * bits / 8 bytes.
template <int E>
__device__ __forceinline__ u2 mx_load(const uint8_t* codes, int t, int e0, int d, int bits, bool is_v) {
  const uint8_t* at = codes + mx_code_at(t, e0, d, bits, is_v);
  u2 r = {0u, 0u};
  if (mx_run(d, is_v) >= E) {
    if constexpr (E == 8) {
      if (bits == 8) r = *reinterpret_cast<const u2*>(at);
      else r.x = *reinterpret_cast<const uint32_t*>(at);
    } else {
      if (bits == 8) r.x = *reinterpret_cast<const uint32_t*>(at);
      else r.x = *reinterpret_cast<const uint16_t*>(at);
    }
  } else {
    const uint8_t* next = codes + mx_code_at(t, e0 + 4, d, bits, is_v);
    if (bits == 8) {
      r.x = *reinterpret_cast<const uint32_t*>(at);
      r.y = *reinterpret_cast<const uint32_t*>(next);
    } else {
      r.x = *reinterpret_cast<const uint16_t*>(at) | ((uint32_t)*reinterpret_cast<const uint16_t*>(next) << 16);
    }
  }
  return r;
}

__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Two elements as a pair of bf16, exactly: byte B of 4-bit codes, half B of 8-bit ones.
template <int B>
__device__ __forceinline__ uint32_t mx_pair4(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B));
}
template <int B>
__device__ __forceinline__ uint32_t mx_pair8(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, B != 0));
}

}  // namespace tgd

namespace tg {

// Bits of a part's format, or 0.
inline int mx_bits(int32_t format) { return format == TG_MX_FP4 ? 4 : format == TG_MX_FP8 ? 8 : 0; }

// What the calls of a quantised cache share.  On failure records a message.
inline int32_t check_mx(const tg_geometry* g, const tg_mx_format* f) {
  if (int32_t rc = check_geometry(g)) return rc;
  if (!f) return fail(TG_ERR_INVALID_ARG, "format is NULL");
  if (!mx_bits(f->k_format) || !mx_bits(f->v_format))
    return fail(TG_ERR_INVALID_ARG, "unknown format %d / %d", f->k_format, f->v_format);
  if (g->head_dim != 64 && g->head_dim != 128)
    return fail(TG_ERR_UNSUPPORTED, "a quantised cache has head_dim 64 or 128 (got %d)", g->head_dim);
  if (g->page_size != tgd::kMxPage)
    return fail(TG_ERR_UNSUPPORTED, "a quantised cache has page_size 16 (got %d)", g->page_size);
  return TG_OK;
}

}  // namespace tg
