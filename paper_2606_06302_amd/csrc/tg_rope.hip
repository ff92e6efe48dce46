// Queries and keys between the projection and the cache: RMS norm per head,
// rotation by position, values copied beside them, for a chunk (tg_rope) or one
// new token per request straight into the ragged cache (tg_rope_append).
//
// A head is owned by D * sizeof(T) / 32 lanes, two 16-byte chunks each, so a
// wave holds 64 / that many heads at once (8 of bf16, head_dim 128).  With
// adjacent pairs lane i takes chunks i and i + the head's lanes; with halves the
// lanes that rotate take both members of their pairs, chunks i and i + rot_dim / 2
// dims, the others 2i and 2i + 1.  Nothing moves between lanes but the norm's sum
// of squares, and the lanes of an access lie next to each other (adjacent pairs
// with chunks 2i and 2i + 1: 44.2 us for 201 MB of f32, head_dim 64, 39.1 so).
//
// Bound by HBM where there are tokens enough (16 x 512 tokens of 32 + 16 heads of 128,
// 201 MB: 38.6 us, 5.2 TB/s, the rate of a large copy), by latency for a step's
// tokens (64 requests in 4.8 us, one in 3.9).
//
// Angles.  turns[j] is the rotation per token as a 64-bit fraction of a turn, so
// position * turns[j] modulo 2^64 is the angle with every whole turn dropped,
// exactly, at any position: no fp64 and no table over positions.  Its top 32
// bits give the quadrant and a remainder within an eighth of a turn, for which
// the Taylor series to x^9 and x^10 are within 4e-9 of sine and cosine.  Every
// angle of a token is worked out once per wave, lane j that of pair j, and goes
// to the head lanes through LDS.
#include <hip/hip_runtime.h>

#include <cmath>

#include "tg_device.h"
#include "tg_internal.h"

namespace {

using namespace tgd;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;

struct RopeParams {
  const u4* q_in;            // 16-byte chunks
  const u4* k_in;
  const u4* v_in;
  int64_t q_stride, k_stride, v_stride;   // chunks between tokens
  const int32_t* positions;  // [tokens] or NULL
  const int32_t* start;      // [B] or NULL
  const int32_t* chunk_tokens;   // [B] or NULL
  const uint64_t* turns;
  const u4* q_weight;
  const u4* k_weight;
  u4* q_out;
  u4* k_out;
  u4* v_out;
  int64_t tokens;
  int32_t chunk, Hq, H;      // Hq: 0 without queries; H: 0 without keys (and values)
  int32_t units;             // heads of a token that the launch works on
  int32_t splits;            // waves that share a token
  int32_t passes;            // head groups of a wave
  int32_t rot_dim, norm;
  float factor, eps, offset;
  // append
  u4* pool;
  const int32_t* pt_pages;
  const int64_t* pt_offsets;
  const int32_t* group_of;
  const int32_t* slot_of;
  int32_t* live_len;
  int32_t* full;
  int32_t L, G, Hp, P, layer;
};

template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
  static constexpr int kElems = 4;
  __device__ static void unpack(const u4& v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(v[i]);
  }
  __device__ static u4 pack(const float* f) {
    return u4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
  }
};
template <>
struct Chunk<uint16_t> {
  static constexpr int kElems = 8;
  __device__ static void unpack(const u4& v, float* f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16_lo(v[i]);
      f[2 * i + 1] = bf16_hi(v[i]);
    }
  }
  __device__ static u4 pack(const float* f) {
    u4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = uint32_t(f32_to_bf16(f[2 * i])) | (uint32_t(f32_to_bf16(f[2 * i + 1])) << 16);
    return r;
  }
};

// cosine and sine of position * turns (a fraction of a turn of 64 bits)
__device__ __forceinline__ void cos_sin(int32_t position, uint64_t turns, float* c, float* s) {
  const uint32_t at = (uint32_t)(((uint64_t)(int64_t)position * turns) >> 32);
  const uint32_t quadrant = (at + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(at - (quadrant << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float u = x * x;
  const float sx = x * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float cx =
      fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const bool swap = quadrant & 1;
  const float cv = swap ? sx : cx, sv = swap ? cx : sx;
  *c = ((quadrant + 1) & 2) ? -cv : cv;
  *s = (quadrant & 2) ? -sv : sv;
}

// One wave: heads [split * passes * heads per wave, ...) of one token.
template <typename T, int D, bool kInterleaved, bool kAppend, bool kStream>
__global__ void __launch_bounds__(kBlock) tg_rope_kernel(RopeParams p) {
  constexpr int E = Chunk<T>::kElems;
  constexpr int CPR = D / E;             // chunks per head
  constexpr int LPH = CPR / 2;           // lanes per head
  constexpr int HPW = 64 / LPH;          // heads of a wave at once
  __shared__ float sm_cos[kWaves][64], sm_sin[kWaves][64];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * kWaves + wave;
  const int64_t token = w / p.splits;
  const int split = (int)(w % p.splits);
  if (token >= p.tokens) return;
  const int b = (int)(token / p.chunk), i = (int)(token % p.chunk);
  if (p.chunk_tokens && i >= p.chunk_tokens[b]) return;

  const int sub = lane % LPH;
  const int rot_lanes = p.rot_dim / (2 * E);   // halves: lanes that rotate; adjacent pairs: half of the chunks that do
  const bool turns0 = kInterleaved ? sub < 2 * rot_lanes : sub < rot_lanes;         // whether the first chunk is rotated
  const bool turns1 = kInterleaved ? sub + LPH < 2 * rot_lanes : sub < rot_lanes;   // and the second
  const int c0 = kInterleaved || turns0 ? sub : 2 * sub;
  const int c1 = kInterleaved ? sub + LPH : turns0 ? sub + rot_lanes : 2 * sub + 1;

  if (p.rot_dim > 0) {
    const int32_t position = p.positions ? p.positions[token] : (int32_t)((p.start ? (uint32_t)p.start[b] : 0u) + (uint32_t)i);
    if (lane < p.rot_dim / 2) {
      float c, s;
      cos_sin(position, p.turns[lane], &c, &s);
      sm_cos[wave][lane] = c * p.factor;
      sm_sin[wave][lane] = s * p.factor;
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  float cs[E], sn[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    // halves: the lane's E pairs; adjacent pairs: E / 2 of each chunk
    const int j = kInterleaved ? (e < E / 2 ? c0 : c1) * (E / 2) + e % (E / 2) : sub * E + e;
    const bool turns = e < E / 2 ? turns0 : turns1;
    cs[e] = turns ? sm_cos[wave][j] : 1.f;
    sn[e] = turns ? sm_sin[wave][j] : 0.f;
  }
  const u4 one = u4(sizeof(T) == 2 ? 0x3f803f80u : 0x3f800000u);   // values of 1
  u4 wq[2], wk[2];
  wq[0] = p.norm && p.q_weight ? p.q_weight[c0] : one;
  wq[1] = p.norm && p.q_weight ? p.q_weight[c1] : one;
  wk[0] = p.norm && p.k_weight ? p.k_weight[c0] : one;
  wk[1] = p.norm && p.k_weight ? p.k_weight[c1] : one;
  const float q_offset = p.q_weight ? p.offset : 0.f, k_offset = p.k_weight ? p.offset : 0.f;

  // norm and rotation of a head's two chunks
  auto turn = [&](u4* x, bool is_k) {
    float y0[E], y1[E];
    Chunk<T>::unpack(x[0], y0);
    Chunk<T>::unpack(x[1], y1);
    if (p.norm) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) ss = fmaf(y0[e], y0[e], fmaf(y1[e], y1[e], ss));
      ss = group_sum<LPH>(ss);
      const float r = rsqrtf(fmaf(ss, 1.f / D, p.eps));
      const float off = is_k ? k_offset : q_offset;
      float w0[E], w1[E];
      Chunk<T>::unpack(is_k ? wk[0] : wq[0], w0);
      Chunk<T>::unpack(is_k ? wk[1] : wq[1], w1);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        y0[e] *= r * (off + w0[e]);
        y1[e] *= r * (off + w1[e]);
      }
    }
    if constexpr (kInterleaved) {
      auto pairs = [&](float* y, int first) {
#pragma unroll
        for (int e = 0; e < E / 2; ++e) {
          const float a = y[2 * e], bb = y[2 * e + 1];
          y[2 * e] = fmaf(a, cs[first + e], -(bb * sn[first + e]));
          y[2 * e + 1] = fmaf(bb, cs[first + e], a * sn[first + e]);
        }
      };
      if (turns0) pairs(y0, 0);
      if (turns1) pairs(y1, E / 2);
    } else if (turns0) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float a = y0[e], bb = y1[e];
        y0[e] = fmaf(a, cs[e], -(bb * sn[e]));
        y1[e] = fmaf(bb, cs[e], a * sn[e]);
      }
    }
    x[0] = Chunk<T>::pack(y0);
    x[1] = Chunk<T>::pack(y1);
  };

  for (int pass = 0; pass < p.passes; ++pass) {
    const int unit = (split * p.passes + pass) * HPW + lane / LPH;
    if (unit >= p.units) break;
    const bool is_q = unit < p.Hq;
    if constexpr (kAppend) {
      if (is_q) {
        const u4* src = p.q_in + token * p.q_stride + (int64_t)unit * CPR;
        u4* dst = p.q_out + (token * p.Hq + unit) * CPR;
        u4 x[2] = {src[c0], src[c1]};
        turn(x, false);
        dst[c0] = x[0];
        dst[c1] = x[1];
        continue;
      }
      const int h = unit - p.Hq;
      const int64_t lh = (int64_t)p.layer * p.H + h;
      int32_t* live = p.live_len + (token * p.L + p.layer) * p.H + h;
      const int n = *live;
      const TablePages table = table_of(p.pt_offsets, (token * p.L + p.layer) * p.G, p.group_of[lh], p.G);
      if (n < 0 || n >= table.pages * p.P) {
        if (p.full && sub == 0) *p.full = 1;
        continue;
      }
      const u4* ks = p.k_in + token * p.k_stride + (int64_t)h * CPR;
      const u4* vs = p.v_in + token * p.v_stride + (int64_t)h * CPR;
      u4 x[2] = {ks[c0], ks[c1]};
      const u4 v0 = vs[c0], v1 = vs[c1];
      const int64_t page = p.pt_pages[table.base + n / p.P];
      u4* dst = p.pool + ((page * 2 * p.Hp + p.slot_of[lh]) * p.P + n % p.P) * CPR;
      turn(x, true);
      dst[c0] = x[0];
      dst[c1] = x[1];
      dst += (int64_t)p.Hp * p.P * CPR;
      dst[c0] = v0;
      dst[c1] = v1;
      // the head's lanes have read n (same wave, same load)
      if (sub == 0) *live = n + 1;
    } else {
      const int kh = unit - p.Hq, vh = kh - p.H;
      const bool is_v = !is_q && vh >= 0;
      const u4* src = is_q ? p.q_in + token * p.q_stride + (int64_t)unit * CPR
                           : is_v ? p.v_in + token * p.v_stride + (int64_t)vh * CPR
                                  : p.k_in + token * p.k_stride + (int64_t)kh * CPR;
      u4* dst = is_q ? p.q_out + (token * p.Hq + unit) * CPR
                     : is_v ? p.v_out + (token * (p.units - p.Hq - p.H) + vh) * CPR : p.k_out + (token * p.H + kh) * CPR;
      u4 x[2];
      if constexpr (kStream) {
        x[0] = __builtin_nontemporal_load(src + c0);
        x[1] = __builtin_nontemporal_load(src + c1);
      } else {
        x[0] = src[c0];
        x[1] = src[c1];
      }
      const u4 raw[2] = {x[0], x[1]};
      turn(x, !is_q);
      __builtin_nontemporal_store(is_v ? raw[0] : x[0], dst + c0);
      __builtin_nontemporal_store(is_v ? raw[1] : x[1], dst + c1);
    }
  }
}

using RopeFn = void (*)(RopeParams);

template <typename T, int D, bool kAppend, bool kStream>
RopeFn pick_layout(int layout) {
  return layout == TG_ROPE_INTERLEAVED ? &tg_rope_kernel<T, D, true, kAppend, kStream>
                                       : &tg_rope_kernel<T, D, false, kAppend, kStream>;
}

template <bool kAppend, bool kStream>
RopeFn pick_rope(int dtype, int d, int layout) {
  if (dtype == TG_F32)
    return d == 64 ? pick_layout<float, 64, kAppend, kStream>(layout) : pick_layout<float, 128, kAppend, kStream>(layout);
  return d == 64 ? pick_layout<uint16_t, 64, kAppend, kStream>(layout) : pick_layout<uint16_t, 128, kAppend, kStream>(layout);
}

int32_t check_spec(const tg_rope_spec& s, int d) {
  if (s.layout != TG_ROPE_HALF && s.layout != TG_ROPE_INTERLEAVED)
    return tg::fail(TG_ERR_INVALID_ARG, "unknown rotary layout %d", s.layout);
  if (s.rot_dim < 0 || s.rot_dim > d) return tg::fail(TG_ERR_INVALID_ARG, "rot_dim %d outside 0..%d", s.rot_dim, d);
  if (s.rot_dim % 16 != 0) return tg::fail(TG_ERR_UNSUPPORTED, "rot_dim must be a multiple of 16 (got %d)", s.rot_dim);
  if (s.rot_dim > 0 && !s.turns) return tg::fail(TG_ERR_INVALID_ARG, "rotation needs turns");
  if (reinterpret_cast<uintptr_t>(s.turns) & 7u) return tg::fail(TG_ERR_INVALID_ARG, "turns must be 8-byte aligned");
  if (s.norm != 0 && s.norm != 1) return tg::fail(TG_ERR_INVALID_ARG, "norm must be 0 or 1");
  if (!std::isfinite(s.attn_factor) || !std::isfinite(s.weight_offset) || !(s.eps >= 0.f) || !std::isfinite(s.eps))
    return tg::fail(TG_ERR_INVALID_ARG, "attn_factor, weight_offset and eps must be finite, eps >= 0");
  if (!tg::aligned16({s.q_weight, s.k_weight})) return tg::fail(TG_ERR_INVALID_ARG, "norm weights must be 16-byte aligned");
  return TG_OK;
}

// One input: its stride covers a token's heads and is a multiple of 16 bytes.
int32_t check_stride(const char* what, int64_t stride, int64_t row, int esz) {
  if (stride < row || stride > (int64_t(1) << 40))
    return tg::fail(TG_ERR_INVALID_ARG, "%s_stride %lld is less than a token's %lld elements, or too large", what,
                    (long long)stride, (long long)row);
  if (stride * esz % 16) return tg::fail(TG_ERR_INVALID_ARG, "%s_stride must be a multiple of 16 bytes", what);
  return TG_OK;
}

int32_t check_shape(const tg_geometry& g, int dtype, const char* what) {
  if (int32_t rc = tg::check_geometry(&g)) return rc;
  if (dtype != TG_F32 && dtype != TG_BF16) return tg::fail(TG_ERR_UNSUPPORTED, "dtype must be f32 or bf16");
  if (g.head_dim != 64 && g.head_dim != 128)
    return tg::fail(TG_ERR_UNSUPPORTED, "%s supports head_dim 64 or 128 (got %d)", what, g.head_dim);
  return TG_OK;
}

void fill_spec(RopeParams& p, const tg_rope_spec& s) {
  p.turns = s.turns;
  p.q_weight = static_cast<const u4*>(s.q_weight);
  p.k_weight = static_cast<const u4*>(s.k_weight);
  p.rot_dim = s.rot_dim;
  p.norm = s.norm;
  p.factor = s.attn_factor != 0.f ? s.attn_factor : 1.f;
  p.eps = s.eps;
  p.offset = s.weight_offset;
}

// Waves of a token: one for all its heads once the tokens alone fill the chip,
// else as many as bring the launch to kFullWaves.
constexpr int64_t kFullWaves = 4096;

int32_t launch(RopeFn fn, RopeParams& p, int heads_per_wave, hipStream_t st, const char* what) {
  const int64_t groups = (p.units + heads_per_wave - 1) / heads_per_wave;
  const int64_t want = (kFullWaves + p.tokens - 1) / p.tokens;
  p.passes = (int)((groups + want - 1) / want);
  p.splits = (int)((groups + p.passes - 1) / p.passes);
  const int64_t blocks = (p.tokens * p.splits + kWaves - 1) / kWaves;
  if (blocks > INT32_MAX) return tg::fail(TG_ERR_INVALID_ARG, "batch * chunk_len too large");
  hipLaunchKernelGGL(fn, dim3((unsigned)blocks), dim3(kBlock), 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "%s launch failed: %s", what, hipGetErrorString(e));
  return TG_OK;
}

int heads_per_wave(int dtype, int d) { return 64 / (d * (dtype == TG_F32 ? 4 : 2) / 32); }

}  // namespace

extern "C" int32_t tg_rope(const tg_rope_args* a, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = check_shape(g, a->dtype, "rope")) return rc;
  if (int32_t rc = check_spec(a->spec, g.head_dim)) return rc;
  if (a->batch < 1 || a->chunk_len < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch and chunk_len must be >= 1");
  if (!a->q_in != !a->q_out || !a->k_in != !a->k_out || !a->v_in != !a->v_out)
    return tg::fail(TG_ERR_INVALID_ARG, "an input and its output go together");
  if (!a->q_in && !a->k_in && !a->v_in) return tg::fail(TG_ERR_INVALID_ARG, "no input");
  if (!tg::aligned16({a->q_in, a->k_in, a->v_in, a->q_out, a->k_out, a->v_out}))
    return tg::fail(TG_ERR_INVALID_ARG, "device buffers must be 16-byte aligned");
  const int esz = a->dtype == TG_F32 ? 4 : 2;
  const int64_t q_row = (int64_t)g.num_q_heads * g.head_dim, kv_row = (int64_t)g.num_kv_heads * g.head_dim;
  if (a->q_in)
    if (int32_t rc = check_stride("q", a->q_stride, q_row, esz)) return rc;
  if (a->k_in)
    if (int32_t rc = check_stride("k", a->k_stride, kv_row, esz)) return rc;
  if (a->v_in)
    if (int32_t rc = check_stride("v", a->v_stride, kv_row, esz)) return rc;
  RopeParams p = {};
  fill_spec(p, a->spec);
  p.q_in = static_cast<const u4*>(a->q_in);
  p.k_in = static_cast<const u4*>(a->k_in);
  p.v_in = static_cast<const u4*>(a->v_in);
  p.q_stride = a->q_stride * esz / 16;
  p.k_stride = a->k_stride * esz / 16;
  p.v_stride = a->v_stride * esz / 16;
  p.positions = a->positions;
  p.start = a->start;
  p.chunk_tokens = a->chunk_tokens;
  p.q_out = static_cast<u4*>(a->q_out);
  p.k_out = static_cast<u4*>(a->k_out);
  p.v_out = static_cast<u4*>(a->v_out);
  p.tokens = (int64_t)a->batch * a->chunk_len;
  p.chunk = a->chunk_len;
  p.Hq = a->q_in ? g.num_q_heads : 0;
  p.H = a->k_in ? g.num_kv_heads : 0;
  p.units = p.Hq + p.H + (a->v_in ? g.num_kv_heads : 0);
  // Loads that leave nothing in the caches, against plain ones, by where the rows are.
  // Behind the product that wrote them (32 + 16 heads of 128, bf16): input and output
  // 201 MB 36.6 -> 36.5 us, 403 MB 80.5 -> 70.0 (64 + 16 heads, 336 MB: 70.6 -> 71.8; head_dim 64,
  // 235 MB: 46.3 -> 46.0).  From HBM they pay 1 to 4 % from 60 MB on (201 MB 40.2 -> 39.0; bf16
  // of head_dim 64 loses as much: 43.1 -> 45.7), and rows still in the caches of a call before lose by
  // them at every size (100 MB 17.6 -> 19.7, 201 MB 33.6 -> 37.5, 400 MB 61.5 -> 70.3).
  // Between 151 and 201 MB nothing singles out a size: past it rows mostly come from HBM,
  // below it from the caches.  Stores that leave nothing pay at any size (201 MB 43.9 ->
  // 40.6, 101 MB 22.3 -> 18.4, 50 MB level, 13 MB 4.9 -> 4.3).
  const bool stream = 2 * p.tokens * p.units * g.head_dim * esz > ((int64_t)176 << 20);
  const RopeFn fn = stream ? pick_rope<false, true>(a->dtype, g.head_dim, a->spec.layout)
                           : pick_rope<false, false>(a->dtype, g.head_dim, a->spec.layout);
  return launch(fn, p, heads_per_wave(a->dtype, g.head_dim),
                static_cast<hipStream_t>(hip_stream), "rope");
}

extern "C" int32_t tg_rope_append(const tg_rope_append_args* a, void* hip_stream) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = check_shape(g, a->dtype, "rope append")) return rc;
  if (int32_t rc = check_spec(a->spec, g.head_dim)) return rc;
  if (a->batch < 1) return tg::fail(TG_ERR_INVALID_ARG, "batch must be >= 1");
  if (a->layer < 0 || a->layer >= g.num_layers) return tg::fail(TG_ERR_INVALID_ARG, "layer %d out of range", a->layer);
  if (!a->q_in != !a->q_out) return tg::fail(TG_ERR_INVALID_ARG, "an input and its output go together");
  if (!a->k_in || !a->v_in || !a->positions || !a->kv_pool || !a->pt_pages || !a->pt_offsets || !a->group_of ||
      !a->slot_of || !a->live_len)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  if (!tg::aligned16({a->q_in, a->k_in, a->v_in, a->q_out, a->kv_pool}))
    return tg::fail(TG_ERR_INVALID_ARG, "device buffers must be 16-byte aligned");
  const int esz = a->dtype == TG_F32 ? 4 : 2;
  const int64_t q_row = (int64_t)g.num_q_heads * g.head_dim, kv_row = (int64_t)g.num_kv_heads * g.head_dim;
  if (a->q_in)
    if (int32_t rc = check_stride("q", a->q_stride, q_row, esz)) return rc;
  if (int32_t rc = check_stride("k", a->k_stride, kv_row, esz)) return rc;
  if (int32_t rc = check_stride("v", a->v_stride, kv_row, esz)) return rc;
  RopeParams p = {};
  fill_spec(p, a->spec);
  p.q_in = static_cast<const u4*>(a->q_in);
  p.k_in = static_cast<const u4*>(a->k_in);
  p.v_in = static_cast<const u4*>(a->v_in);
  p.q_stride = a->q_stride * esz / 16;
  p.k_stride = a->k_stride * esz / 16;
  p.v_stride = a->v_stride * esz / 16;
  p.positions = a->positions;
  p.q_out = static_cast<u4*>(a->q_out);
  p.tokens = a->batch;
  p.chunk = 1;
  p.Hq = a->q_in ? g.num_q_heads : 0;
  p.H = g.num_kv_heads;
  p.units = p.Hq + p.H;
  p.pool = static_cast<u4*>(a->kv_pool);
  p.pt_pages = a->pt_pages;
  p.pt_offsets = a->pt_offsets;
  p.group_of = a->group_of;
  p.slot_of = a->slot_of;
  p.live_len = a->live_len;
  p.full = a->full;
  p.L = g.num_layers;
  p.G = g.num_kv_heads / g.heads_per_group;
  p.Hp = g.heads_per_group;
  p.P = g.page_size;
  p.layer = a->layer;
  return launch(pick_rope<true, false>(a->dtype, g.head_dim, a->spec.layout), p, heads_per_wave(a->dtype, g.head_dim),
                static_cast<hipStream_t>(hip_stream), "rope append");
}
