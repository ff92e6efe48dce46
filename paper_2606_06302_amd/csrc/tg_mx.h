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

// The 16 bytes of a row that a lane holds: the bits of the largest magnitude among
// them as fp32 (as integers NaN is above infinity, and both above every number),
// and the conversions of 4 elements, word 2 i or 4 i on, with scale s.
template <typename T>
struct Row16;
template <>
struct Row16<uint16_t> {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  static constexpr int kElems = 8;
  // by value: a bit cast of a vector's element in place takes the first one
  __device__ __forceinline__ static bf16x2 words(u4 v, int i) {
    const uint32_t w = v[i];
    return __builtin_bit_cast(bf16x2, w);
  }
  __device__ __forceinline__ static uint32_t top(const u4& v) {
    u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
    return (uint32_t)max(m.x, m.y) << 16;
  }
  __device__ __forceinline__ static uint32_t fp4(const u4& v, float s) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, words(v, 0), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, words(v, 1), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, words(v, 2), s, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, words(v, 3), s, 3);
  }
  __device__ __forceinline__ static u2 fp8(const u4& v, float s) {
    u2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s16x2 c = {0, 0};
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, words(v, 2 * i), s, false);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, words(v, 2 * i + 1), s, true);
      r[i] = __builtin_bit_cast(uint32_t, c);
    }
    return r;
  }
  // magnitudes above bits `most` of fp32 become those (a bf16 number)
  __device__ __forceinline__ static u4 clamp(const u4& v, uint32_t most) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const u16x2 m = __builtin_elementwise_min(__builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu),
                                                u16x2{(uint16_t)(most >> 16), (uint16_t)(most >> 16)});
      r[i] = __builtin_bit_cast(uint32_t, m) | (v[i] & 0x80008000u);
    }
    return r;
  }
};
template <>
struct Row16<float> {
  static constexpr int kElems = 4;
  __device__ __forceinline__ static void unpack(const u4& v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  __device__ __forceinline__ static uint32_t top(const u4& v) {
    return max(max(v[0] & 0x7fffffffu, v[1] & 0x7fffffffu), max(v[2] & 0x7fffffffu, v[3] & 0x7fffffffu));
  }
  __device__ __forceinline__ static uint32_t fp4(const u4& v, float s) {
    float x[4];
    unpack(v, x);
    const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  }
  __device__ __forceinline__ static u2 fp8(const u4& v, float s) {
    float x[4];
    unpack(v, x);
    s16x2 c = {0, 0};
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[0], x[1], s, false);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[2], x[3], s, true);
    return u2{__builtin_bit_cast(uint32_t, c), 0u};
  }
  __device__ __forceinline__ static u4 clamp(const u4& v, uint32_t most) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = min(v[i] & 0x7fffffffu, most) | (v[i] & 0x80000000u);
    return r;
  }
};

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false));
}

// Codes of the elements that a lane holds (the lanes of a group of 32 lie side by
// side and call this together): the scale is 2^e, e the least integer with max|x|
// <= top 2^e, top 7 (4 bits) or 464 (8 bits), the midpoint between the largest
// value and the step that would follow; an element is x / 2^e to the nearest, ties
// to even, at most the largest.  All of it is exact but the one rounding of the
// element, so it depends on nothing but the input.  A group with a NaN or an
// infinity gets scale byte 255 and codes 0, which stand for NaN.
// Returns the codes, low bytes first, and *scale, e + 127.
template <typename T>
__device__ __forceinline__ u2 mx_quantise(u4 x, int bits, uint32_t* scale) {
  uint32_t top = Row16<T>::top(x);
  top = dpp_max_u32<kQuadXor1>(top);
  top = dpp_max_u32<kQuadXor2>(top);
  if constexpr (sizeof(T) == 4) top = dpp_max_u32<kRowHalfMirror>(top);
  // the exponent of top * 2^-2 (4 bits, 7 = 1.75 * 2^2) or top * 2^-8 (464 = 1.8125 * 2^8), one more past
  // 1.75 or 1.8125; within bounds that keep every value a normal bf16 number
  const int up = bits == 4 ? 0x1fffff : 0x17ffff, shift = bits == 4 ? 2 : 8;
  const int e = min(max((int)((top + up) >> 23) - shift, bits == 4 ? 2 : 10), bits == 4 ? 252 : 246);
  const float s = __uint_as_float((uint32_t)e << 23);
  const bool finite = top < 0x7f800000u;
  *scale = finite ? (uint32_t)e : 255u;
  u2 r = {0u, 0u};
  if (bits == 4) {
    r.x = finite ? Row16<T>::fp4(x, s) : 0u;
  } else {
    // past 464 * 2^119 alone is a value left that the conversion would make NaN of
    constexpr uint32_t kMost = (246u << 23) + (8u << 23) + 0x600000u;   // 448 * 2^119
    if (top > kMost) x = Row16<T>::clamp(x, kMost);
    r = Row16<T>::fp8(x, s);
    r.x = finite ? r.x : 0u;
    r.y = finite ? r.y : 0u;
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
