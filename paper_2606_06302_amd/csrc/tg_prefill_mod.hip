// Ragged chunked-prefill attention with modified scores for gfx950 (MI355X),
// bf16 MFMA: scores capped by a tanh, a range of visible chunk keys per row
// (prefix, document and window masks), the history seen by a row or not, chunks
// shorter than the batch's.
//
// Tiles, LDS layout, data movement and products are tg_prefill.hip's: one
// workgroup of 8 waves per 256 (chunk row, query head) rows of a (request, KV
// head), key tiles of 64 in a 4-deep LDS ring, S^T = K Q^T and O^T += V^T P^T
// per 32 keys and 32 rows of a wave.  What differs:
//
// Masks.  Row i sees the chunk keys [lo, hi), and all of the history or none of
// it.  A workgroup walks the tiles that any of its rows sees, a wave computes
// the 32-key blocks that any of its rows sees and masks those that not all of
// them see whole.
//
// Caps.  z = softcap * tanh(s / softcap) has exp's cost twice over, so where the
// scores let it (the scores of a trained model do) tanh is an odd
// polynomial whose last product goes into the exponent's subtraction: e = s *
// P(s^2) - m, four full-rate instructions instead of one up to 0.365 of the cap,
// five up to 0.625 of it.  Past that (and past scores of 33 and 42, which only caps past
// 66 reach) tanh itself.  The greatest of the 16 scores that a lane's row sees chooses for
// the lane, so that what a row does not see, other rows' scores among it, changes no bit;
// the wave takes the longest of its lanes' ways.
// 16 requests of 8 KV heads, chunk 512, 16384 tokens before it, gqa 4, head_dim 128, in us
// by cap over the scores' standard deviation: none 727, 50/3 (all within 0.365) 822, 50/6
// 883, 50/9 1080, 20/4 1156, 5/4 1324; head_dim 64: 418, 505, 546, 693, 730, 891.
// tanh is monotone: the running maximum is kept of the raw scores and capped only when
// it is raised.
//
// Infinities and NaN that a row does not see.  A hidden key has probability 0,
// and 0 * infinity is NaN.  Nothing is spent on it in the walk over the tiles: a
// workgroup that ends with an output that is not finite walks its tiles once
// more, with care (add_infinities).
//
// Key-split launch.  With masks the blocks differ in length even within one
// (request, KV head), so that a cut by the unit's length leaves most of the chip
// idle (documents, five requests of 8 KV heads, chunk 333, head_dim 64: 68 us, 57 by
// the blocks' lengths).  A first launch of one workgroup reads the masks, sums every
// block's key tiles, cuts blocks of more than T tiles (tg_prefill_mod_plan_kernel
// says which) into equal pieces and lays the pieces out in a list: the cut blocks'
// first, then the others in seven classes of descending length, every class dealt
// to the 8 XCDs in runs, so that the row tiles that share keys mostly run on one
// XCD.  Workgroup k runs entry k / 8 of XCD k mod 8.  The pieces' fp32 partials are
// merged by a third launch.
//
// Bound as tg_prefill.hip's kernel, by products and the softmax's vector work, which the
// two waves of a SIMD hardly overlap: counted on those 16 requests, the matrix cores are
// busy 43 % of a SIMD's cycles and its vector ALU 46 % without a cap (918 TFLOP/s), 37 and
// 57 % with one (813), LDS 19 to 22 %.  A short call is bound by its three
// launches (one request, chunk 512 behind 16384 tokens: plan 4, tiles 65, merge 9 us) and
// the 5 us that a workgroup needs to its first tile.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "tg_prefill.h"

namespace {

struct ModParams {
  const uint16_t* q;        // [B][C][Hq][d]
  const u4* k_new;          // [B][C][H][d]
  const u4* v_new;
  const u4* pool;           // [pages][2][Hp][P][d]
  const int32_t* pt_pages;
  const int64_t* pt_offsets;
  const int32_t* kv_len;    // [B][L][H]
  const int32_t* group_of;  // [L][H]
  const int32_t* slot_of;
  uint16_t* out;            // [B][C][Hq][d]
  const int32_t* block_order;   // [gridDim.x] (unit * row_tiles + row tile) or -1, or NULL
  const int32_t* tokens;    // [B] valid tokens of the chunk, or NULL
  const int32_t* key_begin; // [B][C] or NULL
  const int32_t* key_end;   // [B][C] or NULL
  int32_t batch, chunk, layer, num_layers, num_kv_heads, num_groups, heads_per_group, gqa;
  int32_t row_tiles;        // ceil(chunk*gqa / kRows)
  float scale_log2;         // sm_scale * log2(e)
  // capped scores, in log2 units: z = cap_log2 * tanh(s * cap_in); for |s| <= cap_split
  // s * (poly[0] + u (poly[1] + u (poly[2] + u poly[3]))), u = s^2, and for |s| <=
  // near_split s * (near[0] + u (near[1] + u near[2]))
  float cap_in, cap_log2, cap_split;
  float poly[4];
  float near_split, near[3];
  float cap_exp;            // log2 of e^(2 |s| cap_in) per |s|; 0: the polynomials end before kCapSplit of the cap
  // key-split launch only
  f32x4* part_o;            // [split_slots][part_waves][D/4][32 rows] unnormalised fp32 outputs
  float* part_ml;           // [split_slots][part_waves][2][32 rows]: reference maximum in log2 units, sum
  int2* pieces;             // [units * row_tiles]: first partial slot and piece count of every block
  struct ListEntry* list;   // [8 * list_per_xcd]
  int32_t part_waves;       // waves of a block that own rows: min(8, ceil(chunk*gqa / 32))
  int32_t list_len;
};

// One workgroup of the key-split launch: a piece of a block of rows.
struct ListEntry {
  int32_t block;            // unit * row_tiles + row tile, or -1: nothing
  int32_t t_begin, t_end;   // key tiles of the block's walk
  int32_t nh, ct0;          // the walk: history tiles, first chunk tile
  int32_t slot;             // partial slot, or -1: the whole block, the output is written
  int32_t unused[2];
};
static_assert(sizeof(ListEntry) == tg::kPrefillListEntryBytes, "split_layout counts these");

// The chunk keys [lo, hi) that row i of request b sees; the history where lo was
// negative.  No key of the chunk: lo = INT32_MAX, hi = 0, neutral for the least
// lo and the greatest hi.
struct Seen {
  int lo, hi;
  bool hist;
};
__device__ __forceinline__ Seen row_sees(const ModParams& p, int b, int i, int n_valid) {
  Seen s;
  const int64_t at = (int64_t)b * p.chunk + i;
  s.lo = p.key_begin ? p.key_begin[at] : -1;
  s.hi = min(p.key_end ? p.key_end[at] : i + 1, n_valid);
  s.hist = s.lo < 0;
  s.lo = max(s.lo, 0);
  if (s.hi <= s.lo) {
    s.lo = INT32_MAX;
    s.hi = 0;
  }
  return s;
}

__device__ __forceinline__ int valid_tokens(const ModParams& p, int b) {
  return p.tokens ? max(0, min(p.tokens[b], p.chunk)) : p.chunk;
}

// A block's walk: history tiles nh (0 where no row sees the history), then the
// chunk tiles ct0, ct0 + 1, ... from its rows' least lo and greatest hi.
struct Walk {
  int nh, ct0, n_tiles;
};
__device__ __forceinline__ Walk block_walk(int hist_tiles, int min_lo, int max_hi, bool any_hist) {
  Walk w;
  w.nh = any_hist ? hist_tiles : 0;
  w.ct0 = max_hi > 0 ? min_lo / kTile : 0;
  w.n_tiles = w.nh + (max_hi > 0 ? (max_hi + kTile - 1) / kTile - w.ct0 : 0);
  return w;
}

// x of another lane of the 16-lane row (lanes without a source get `none`)
template <int kCtrl>
__device__ __forceinline__ int row_lane(int x, int none = 0) {
  return __builtin_amdgcn_update_dpp(none, x, kCtrl, 0xF, 0xF, false);
}

// Reductions by lane moves inside the vector unit (a shuffle goes through LDS):
// over the aligned 16 lanes, and over the wave; every lane receives the result.
template <typename Op>
__device__ __forceinline__ int row_reduce(int x, Op op) {
  x = op(x, row_lane<kQuadXor1>(x));
  x = op(x, row_lane<kQuadXor2>(x));
  x = op(x, row_lane<kRowHalfMirror>(x));
  return op(x, row_lane<kRowMirror>(x));
}
template <typename Op>
__device__ __forceinline__ int wave_reduce(int x, Op op) {
  x = row_reduce(x, op);
  auto r = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  x = op((int)r[0], (int)r[1]);
  r = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  return op((int)r[0], (int)r[1]);
}
struct Least {
  __device__ int operator()(int a, int b) const { return min(a, b); }
};
struct Greatest {
  __device__ int operator()(int a, int b) const { return max(a, b); }
};
struct Sum {
  __device__ int operator()(int a, int b) const { return a + b; }
};

// Least of a wave's values, in scalar registers.
__device__ __forceinline__ int wave_min(int x) { return __builtin_amdgcn_readfirstlane(wave_reduce(x, Least())); }

// Sum of the values of the lanes up to and with this one: within the 16-lane
// rows, then the rows before.
__device__ __forceinline__ int wave_inclusive_sum(int x) {
  x += row_lane<0x111>(x);   // row_shr 1, 2, 4, 8
  x += row_lane<0x112>(x);
  x += row_lane<0x114>(x);
  x += row_lane<0x118>(x);
  const int row = (threadIdx.x & 63) >> 4;
  const int s0 = __builtin_amdgcn_readlane(x, 15), s1 = __builtin_amdgcn_readlane(x, 31), s2 = __builtin_amdgcn_readlane(x, 47);
  return x + (row > 0 ? s0 : 0) + (row > 1 ? s1 : 0) + (row > 2 ? s2 : 0);
}

// n / d for 0 <= n < 2^28, d >= 1, by the reciprocal and two corrections.
__device__ __forceinline__ int quotient(int n, int d) {
  int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d));
  int r = n - q * d;
#pragma unroll
  for (int i = 0; i < 2; ++i) {   // off by one at most where n has 24 bits, by 32 with 28 bits and a small d
    const int e = (int)floorf((float)r * __builtin_amdgcn_rcpf((float)d));
    q += e;
    r -= e * d;
  }
  q += r >= d ? 1 : 0;
  q -= r < 0 ? 1 : 0;
  return q;
}

// Bits 15 and 31: whether the bf16 of a word's lower and upper half are infinite or NaN.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// 0xffff in the halves whose bit 15 or 31 is set
__device__ __forceinline__ uint32_t halves(uint32_t bits) { return (bits >> 15) * 0xffffu; }

// 32 dims of 32 keys of which some rows may not see all: takes the infinities
// and NaN out of the V operands and adds what the seen ones make of every
// output.  Two sets of products with operands of 0 and 1 count the positive and
// the negative ones (NaN counts as both) among the keys with a probability.
__device__ __forceinline__ void add_infinities(f32x16& acc, u4& v0, u4& v1, u4& p0, u4& p1) {
#pragma unroll
  for (int sign = 0; sign < 2; ++sign) {
    f32x16 n = f32x16(0.f);
    // nothing is kept from one use for the next: registers
    asm volatile("" : "+v"(v0), "+v"(v1), "+v"(p0), "+v"(p1));
#pragma unroll
    for (int q16 = 0; q16 < 2; ++q16) {
      u4 found, seen;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t v = q16 ? v1[w] : v0[w], pw = q16 ? p1[w] : p0[w];
        const uint32_t odd = halves(not_finite(v));
        const uint32_t nan = halves((((v & 0x007f007fu) + 0x007f007fu) << 8) & 0x80008000u);
        const uint32_t neg = halves(v & 0x80008000u);
        found[w] = 0x3f803f80u & odd & (nan | (sign ? neg : ~neg));
        // probabilities are not negative, 0 where a key is not seen
        seen[w] = 0x3f803f80u & halves(((pw & 0x7fff7fffu) + 0x7fff7fffu) & 0x80008000u);
      }
      n = mfma(found, seen, n);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] += n[r] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
    __builtin_amdgcn_sched_barrier(0);
  }
  asm volatile("" : "+v"(v0), "+v"(v1));
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    v0[w] &= ~halves(not_finite(v0[w]));
    v1[w] &= ~halves(not_finite(v1[w]));
  }
  __builtin_amdgcn_sched_barrier(0);
}

template <int D, bool kSplit, int kWavesPerSimd, bool kCap>
__global__ void __launch_bounds__(kBlock, kWavesPerSimd) tg_prefill_mod_kernel(ModParams p) {
  using S = Shape<D>;
  constexpr int kChunks = S::kChunks, kDmaInst = S::kDmaInst, kDmaPerTile = S::kDmaPerTile;
  constexpr int kTileBytes = S::kTileBytes, kRowsPerDma = S::kRowsPerDma;
  static_assert(kCB == 1, "one row per lane pair");
  constexpr bool kLateV = D == 64;
  __shared__ u4 ring[kRing][2][kTile * kChunks];   // [slot][K, V][key row * kChunks + chunk position]
  __shared__ int32_t shared_int[kWaves][3];

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n_units = p.batch * p.num_kv_heads;
  const int C = p.chunk, gqa = p.gqa;
  const int Hq = p.num_kv_heads * gqa;
  const int rows_total = C * gqa;

  const TG_CONST int32_t* kv_len = (const TG_CONST int32_t*)p.kv_len;
  const TG_CONST int32_t* group_of = (const TG_CONST int32_t*)p.group_of;
  const TG_CONST int32_t* slot_of = (const TG_CONST int32_t*)p.slot_of;
  const TG_CONST int64_t* pt_offsets = (const TG_CONST int64_t*)p.pt_offsets;
  const TG_CONST int32_t* pt_pages = (const TG_CONST int32_t*)p.pt_pages;

  // block -> (unit, row tile): the key-split launch's list, the host schedule,
  // or units round-robin over the 8 XCDs
  int unit, rt;
  const TG_CONST int32_t* const entry = (const TG_CONST int32_t*)(p.list + blockIdx.x);   // key-split launch
  if constexpr (kSplit) {
    const int block = entry[0];
    if (block < 0) return;
    unit = block / p.row_tiles;
    rt = block % p.row_tiles;
  } else if (p.block_order) {
    const int code = ((const TG_CONST int32_t*)p.block_order)[blockIdx.x];
    if (code < 0 || code >= n_units * p.row_tiles) return;
    unit = code / p.row_tiles;
    rt = code % p.row_tiles;
  } else {
    const int xcd = blockIdx.x & 7, local = blockIdx.x >> 3;
    unit = xcd + 8 * (local / p.row_tiles);
    rt = local % p.row_tiles;
    if (unit >= n_units) return;
  }

  const int b = unit / p.num_kv_heads, h = unit % p.num_kv_heads;
  const int grp = group_of[(int64_t)p.layer * p.num_kv_heads + h];
  const int slot = slot_of[(int64_t)p.layer * p.num_kv_heads + h];
  const TablePages table = table_of(pt_offsets, ((int64_t)b * p.num_layers + p.layer) * p.num_groups, grp, p.num_groups);
  const int64_t tbase = table.base;
  // the history is clamped to the head's table: [0, pages * page_size]
  const int64_t cap = table.pages * kPage;
  const int hist = (int)max<int64_t>(0, min<int64_t>(kv_len[((int64_t)b * p.num_layers + p.layer) * p.num_kv_heads + h], cap));
  const int npages = (hist + kPage - 1) / kPage;
  const int row0 = rt * kRows;
  const int n_valid = valid_tokens(p, b);

  // this lane's row, and what the rows of this wave see
  const int row = row0 + wave * kRowsPerWave + (lane & 31);
  const int my_i = min(row / gqa, C - 1);
  const bool row_ok = row < rows_total && my_i < n_valid;
  const Seen mine = row_sees(p, b, my_i, n_valid);
  const int w_min_lo = wave_min(row_ok ? mine.lo : INT32_MAX);
  const int w_max_lo = -wave_min(row_ok ? -mine.lo : 0);
  const int w_min_hi = wave_min(row_ok ? mine.hi : INT32_MAX);
  const int w_max_hi = -wave_min(row_ok ? -mine.hi : 0);
  const bool w_hist_any = __any(row_ok && mine.hist);
  const bool w_hist_all = !__any(row_ok && !mine.hist);

  Walk walk;
  int t_begin = 0, t_end, slot_out = -1;
  if constexpr (kSplit) {
    t_begin = entry[1];
    t_end = entry[2];
    walk.nh = entry[3];
    walk.ct0 = entry[4];
    slot_out = entry[5];
  } else {
    if (lane == 0) {
      shared_int[wave][0] = w_min_lo;
      shared_int[wave][1] = w_max_hi;
      shared_int[wave][2] = w_hist_any;
    }
    __syncthreads();
    int first = INT32_MAX, last = 0, any = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      first = min(first, shared_int[w][0]);
      last = max(last, shared_int[w][1]);
      any |= shared_int[w][2];
    }
    __syncthreads();   // written again after the walk
    walk = block_walk((hist + kTile - 1) / kTile, __builtin_amdgcn_readfirstlane(first),
                      __builtin_amdgcn_readfirstlane(last), __builtin_amdgcn_readfirstlane(any));
    t_end = walk.n_tiles;
  }
  const int nh = walk.nh, ct0 = walk.ct0;
  // head_dim 64: two workgroups fit a CU with 128 registers, so what is cheap to
  // work out again is not kept over the loop
  auto fresh_lane = [&] {
    int ln = lane;
    if constexpr (D == 64) asm volatile("" : "+v"(ln));
    return ln;
  };
  const int hf = lane >> 5;
  const uint32_t ring_lds = lds_address(&ring[0][0][0]);
  const int rb0 = (wave * kDmaRows) % kPage;   // first row of the wave's share within its page

  // DMA of this wave's share (key rows kDmaRows*w .. kDmaRows*(w+1)-1) of tile
  // t into ring slot s
  auto issue = [&](int t, int s) {
    const int ln = fresh_lane();
    const int rl = ln / kChunks;   // row within a DMA instruction
    const int pos = ln % kChunks;  // chunk position within the row
    const uint32_t dst = ring_lds + (uint32_t)s * kTileBytes + (uint32_t)wave * (kDmaRows * kChunks * 16);
    if (t < nh) {
      // past the history: any valid page, masked later
      const int pg = min(t * (kTile / kPage) + wave * kDmaRows / kPage, npages - 1);
      const int64_t id = pt_pages[tbase + pg];
      const u4* kb = p.pool + ((id * 2 + 0) * p.heads_per_group + slot) * (kPage * kChunks);
      const u4* vb = p.pool + ((id * 2 + 1) * p.heads_per_group + slot) * (kPage * kChunks);
#pragma unroll
      for (int j = 0; j < kDmaInst; ++j) {
        const int r = rb0 + j * kRowsPerDma + rl;   // key row within the page (== tile row mod 16)
        lds_dma16(kb, r * kChunks + (pos ^ S::k_swz(r)), dst + j * 1024);
        lds_dma16(vb, r * kChunks + (pos ^ S::v_swz(r)), dst + kTile * kChunks * 16 + j * 1024);
      }
    } else {
      const int c0 = min((t - nh + ct0) * kTile + wave * kDmaRows, C - 1);   // first chunk key of the share
      const int64_t first = (((int64_t)b * C + c0) * p.num_kv_heads + h) * kChunks;
      const u4* kb = p.k_new + first;
      const u4* vb = p.v_new + first;
#pragma unroll
      for (int j = 0; j < kDmaInst; ++j) {
        const int r = j * kRowsPerDma + rl;
        const int rr = rb0 + r;             // tile row mod 16
        const int roff = min(r, C - 1 - c0) * p.num_kv_heads * kChunks;   // rows past the chunk repeat its last key (masked later)
        lds_dma16(kb, roff + (pos ^ S::k_swz(rr)), dst + j * 1024);
        lds_dma16(vb, roff + (pos ^ S::v_swz(rr)), dst + kTile * kChunks * 16 + j * 1024);
      }
    }
  };

  f32x16 acc[S::kDB];
  // the greatest raw score so far that raised it, its value in the exponent (log2
  // units, capped), and the sum of the probabilities relative to that.  tanh is
  // monotone and no steeper than its argument, so the raw maximum bounds the
  // capped scores too
  float m = -INFINITY, z = -INFINITY, l = 0.f;
  auto reference = [&](float raw) { return kCap ? p.cap_log2 * tanh_f32(raw * p.cap_in) : raw * p.scale_log2; };
#pragma unroll
  for (int d = 0; d < S::kDB; ++d) acc[d] = f32x16(0.f);

  u4 qb[S::kK];
  // the lane's row in q and out
  auto q_row = [&] {
    const int r = row0 + wave * kRowsPerWave + (fresh_lane() & 31);
    return ((int64_t)b * C + min(r / gqa, C - 1)) * Hq + h * gqa + r % gqa;
  };
  {
    const u4* qp = reinterpret_cast<const u4*>(p.q + q_row() * D);
#pragma unroll
    for (int kk = 0; kk < S::kK; ++kk) qb[kk] = row_ok ? qp[kk * 2 + hf] : u4(0u);
    // settled here, once: the compiler's wait-count pass cannot see the DMAs,
    // so a load still pending in the loop would make it wait for all of them
#pragma unroll
    for (int kk = 0; kk < S::kK; ++kk) asm volatile("" : "+v"(qb[kk]));
  }

  auto walk_tiles = [&](auto careful) __attribute__((always_inline)) {
    constexpr bool kCareful = decltype(careful)::value;
    // the first kRing-1 tiles in flight (ring slot = tile - t_begin modulo kRing)
#pragma unroll
    for (int r = 0; r < kRing - 1; ++r)
      if (t_begin + r < t_end) issue(t_begin + r, r);

    for (int t = t_begin; t < t_end; ++t) {
      // tile t has landed once at most the DMAs of the tiles after it are pending
      const int after = min(kRing - 2, t_end - 1 - t);
      if (after >= 2)
        wait_vmcnt<2 * kDmaPerTile>();
      else if (after == 1)
        wait_vmcnt<kDmaPerTile>();
      else
        wait_vmcnt<0>();
      const bool is_chunk = t >= nh;
      const int key0 = (is_chunk ? t - nh + ct0 : t) * kTile;   // first key of the tile
      const int key_end = is_chunk ? n_valid : hist;            // keys >= this are none
      if (key0 + wave * kDmaRows + kDmaRows > key_end) {
        // this wave's share holds V rows past the keys: they may hold anything
        // (NaN included) and p = 0 does not cancel NaN, so zero them
        u4* vq = &ring[(t - t_begin) % kRing][1][wave * kDmaRows * kChunks];
        const int ln = fresh_lane();
        uint32_t zero = 0;
        asm volatile("" : "+v"(zero));   // no vector of zeros is kept in registers
#pragma unroll
        for (int j = 0; j < kDmaInst; ++j)
          if (key0 + wave * kDmaRows + j * kRowsPerDma + ln / kChunks >= key_end) vq[j * 64 + ln] = u4(zero);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      barrier();   // tile t complete in LDS; every wave is done with tile t-1
      if (t + kRing - 1 < t_end) issue(t + kRing - 1, (t - t_begin + kRing - 1) % kRing);

      const int s = (t - t_begin) % kRing;
      const unsigned char* kt = reinterpret_cast<const unsigned char*>(&ring[s][0][0]);
      const unsigned char* vt = reinterpret_cast<const unsigned char*>(&ring[s][1][0]);
      if (is_chunk ? key0 >= w_max_hi || key0 + kTile <= w_min_lo : !w_hist_any) continue;   // no row of this wave sees it

#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int kbase = key0 + kb * 32;
        if (is_chunk && (kbase >= w_max_hi || kbase + 32 <= w_min_lo)) continue;
        // whether not all rows of the wave see all of the 32 keys
        const bool masked = is_chunk ? kbase < w_max_lo || kbase + 32 > w_min_hi : kbase + 32 > hist || !w_hist_all;
        const int ln = kCareful ? fresh_lane() : lane;
        const int half = ln >> 5;
        const int krow = kb * 32 + (ln & 31);                       // A of S^T: its key row
        const int tr_key = (ln & 15) >> 2;                          // transposed read: key within a group of 4
        const int tr_dim = 16 * ((ln >> 4) & 1) + 4 * (ln & 3);     // dims within a 32-dim block
        const int tr_chunk = tr_dim >> 3, tr_half = (tr_dim >> 2) & 1;
        u4 va[2][S::kDB];
        auto read_v = [&](int q16, int db) {
          const int g0 = kb * 32 + q16 * 16 + 4 * half;      // tile row of the A operand's first key
          const int r0 = g0 + tr_key, r1 = g0 + 8 + tr_key;  // source rows of the two transposed reads
          const int c = 4 * db + tr_chunk;
          const u2v lo = lds_read_tr16(vt + r0 * (2 * D) + ((c ^ S::v_swz(r0)) << 4) + tr_half * 8);
          const u2v hi = lds_read_tr16(vt + r1 * (2 * D) + ((c ^ S::v_swz(r1)) << 4) + tr_half * 8);
          va[q16][db] = u4{lo.x, lo.y, hi.x, hi.y};
        };
        f32x16 sc = f32x16(0.f);
        {
          // all K operands of the block, and at head_dim 128 the V^T operands of its
          // p.v products (they do not depend on p), are requested before the first
          // product; at 64 their registers would cost the second workgroup
          u4 ka[S::kK];
#pragma unroll
          for (int kk = 0; kk < S::kK; ++kk)
            ka[kk] = *reinterpret_cast<const u4*>(kt + krow * (2 * D) + (((kk * 2 + half) ^ S::k_swz(krow)) << 4));
          if constexpr (!kCareful && !kLateV) {
#pragma unroll
            for (int q16 = 0; q16 < 2; ++q16)
#pragma unroll
              for (int db = 0; db < S::kDB; ++db) read_v(q16, db);
          }
          __builtin_amdgcn_sched_barrier(0);   // keep the reads ahead of the products
#pragma unroll
          for (int kk = 0; kk < S::kK; ++kk) sc = mfma(ka[kk], qb[kk], sc);
        }
        // the lane's keys are kbase + 4*half + 8*(r/4) + r%4; the row's bounds
        // relative to the first of them
        const int first = kbase + 4 * half;
        int from = is_chunk ? mine.lo - first : mine.hist ? 0 : 32;
        int to = (is_chunk ? mine.hi : hist) - first;
        auto sees = [&](int r) { return 8 * (r >> 2) + (r & 3) >= from && 8 * (r >> 2) + (r & 3) < to; };
        // a seen score of -infinity is a score of -softcap where there is a cap
        float mx = kCap ? -FLT_MAX : -INFINITY, big = 0.f;
        if (masked) {
          if (max(from + 4 * half, 0) >= min(to + 4 * half, 32)) mx = -INFINITY;   // no key of the block
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool seen = sees(r);
            mx = fmaxf(mx, seen ? sc[r] : -INFINITY);
            if constexpr (kCap) big = fmaxf(big, seen ? fabsf(sc[r]) : 0.f);
          }
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
          if constexpr (kCap) {
#pragma unroll
            for (int r = 0; r < 16; ++r) big = fmaxf(big, fabsf(sc[r]));
          }
        }
        mx = swap32_max(mx);
        const bool raise = (mx - m) * p.scale_log2 > kSlack;
        if (__any(raise)) {   // raise the running max (rare after the first block)
          const float m_new = raise ? mx : m;
          const float z_new = raise ? reference(m_new) : z;
          // 0 when m was -inf, and 1, not NaN, where it still is beside a row that raises
          const float alpha = raise ? fast_exp2(z - z_new) : 1.f;
          m = m_new;
          z = z_new;
          l *= alpha;
#pragma unroll
          for (int d = 0; d < S::kDB; ++d) acc[d] *= alpha;
        }
        // a row whose scores so far are all -inf has no probabilities yet, not NaN
        const float zr = z == -INFINITY ? 0.f : z;
        if constexpr (!kCap) {
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[r] = fmaf(sc[r], p.scale_log2, -zr);
        } else if (!__any(big > p.near_split)) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float u = sc[r] * sc[r];
            sc[r] = fmaf(sc[r], fmaf(u, fmaf(u, p.near[2], p.near[1]), p.near[0]), -zr);
          }
        } else {
          // the lane's own greatest seen score chooses its polynomial: near's with a
          // fourth coefficient of 0 is near's, bit for bit
          const bool far = big > p.near_split;
          const float c0 = far ? p.poly[0] : p.near[0], c1 = far ? p.poly[1] : p.near[1];
          const float c2 = far ? p.poly[2] : p.near[2], c3 = far ? p.poly[3] : 0.f;
          auto polynomial = [&](float x) {
            const float u = x * x;
            return fmaf(x, fmaf(u, fmaf(u, fmaf(u, c3, c2), c1), c0), -zr);
          };
          const bool beyond = big > p.cap_split;
          if (!__any(beyond)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[r] = polynomial(sc[r]);
          } else if (p.cap_exp > 0.f) {
            // tanh as 1 - 2 / (e^(2|x|) + 1), which does not cancel past the polynomial
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float s = sc[r];
              const float large =
                  fmaf(-2.f * p.cap_log2, __builtin_amdgcn_rcpf(fast_exp2(fabsf(s) * p.cap_exp) + 1.f), p.cap_log2);
              sc[r] = fabsf(s) > p.cap_split ? copysignf(large, s) - zr : polynomial(s);
              __builtin_amdgcn_sched_barrier(0);   // one after the other: registers
            }
          } else {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float e = fmaf(p.cap_log2, tanh_f32(sc[r] * p.cap_in), -zr);
              sc[r] = beyond ? e : polynomial(sc[r]);
              __builtin_amdgcn_sched_barrier(0);   // one after the other: registers
            }
          }
        }
        if (masked) {
          asm volatile("" : "+v"(from), "+v"(to));   // compared again: 16 lane masks are too many to keep
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[r] = sees(r) ? sc[r] : -INFINITY;
        }
        // P is rounded to bf16 (2^-8) for its product and not for its sum: with normal
        // values that is 1.3e-3 to 1.6e-3 of an output beside the 1.7e-3 of its own
        // rounding; products for the rest of P would add half to the block's
        u4 pb[2];
        {
          uint32_t pw[8];
#pragma unroll
          for (int r = 0; r < 16; r += 2) {
            const float p0 = fast_exp2(sc[r]);
            const float p1 = fast_exp2(sc[r + 1]);
            l += p0 + p1;
            pw[r >> 1] = pack_bf16(p0, p1);
          }
          pb[0] = u4{pw[0], pw[1], pw[2], pw[3]};
          pb[1] = u4{pw[4], pw[5], pw[6], pw[7]};
        }
        // O^T += V^T P^T over the two 16-key halves of the block
        if constexpr (kCareful) {
#pragma unroll
          for (int db = 0; db < S::kDB; ++db) {
            __builtin_amdgcn_sched_barrier(0);   // one block of V at a time: registers
            read_v(0, db);
            read_v(1, db);
            if (masked) add_infinities(acc[db], va[0][db], va[1][db], pb[0], pb[1]);
            acc[db] = mfma(va[0][db], pb[0], acc[db]);
            acc[db] = mfma(va[1][db], pb[1], acc[db]);
          }
        } else {
          if constexpr (kLateV) {
#pragma unroll
            for (int q16 = 0; q16 < 2; ++q16)
#pragma unroll
              for (int db = 0; db < S::kDB; ++db) read_v(q16, db);
          }
#pragma unroll
          for (int q16 = 0; q16 < 2; ++q16)
#pragma unroll
            for (int db = 0; db < S::kDB; ++db) acc[db] = mfma(va[q16][db], pb[q16], acc[db]);
        }
      }
    }
    wait_vmcnt<0>();
  };

  walk_tiles(std::false_type{});
  // an output that is not finite: 0 * infinity in a key that the row does not
  // see, or an infinity that it does see
  float odd = 0.f;
#pragma unroll
  for (int db = 0; db < S::kDB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) odd = fmaf(acc[db][r], 0.f, odd);
  const int again = __any(row_ok && odd != 0.f);   // NaN is not equal to 0
  if (lane == 0) shared_int[wave][0] = again;
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) any |= shared_int[w][0];
  if (__builtin_amdgcn_readfirstlane(any)) {
    float zero = 0.f;
    asm volatile("" : "+v"(zero));
#pragma unroll
    for (int d = 0; d < S::kDB; ++d) acc[d] = f32x16(zero);
    m = z = -INFINITY;
    l = 0.f;
    walk_tiles(std::true_type{});
  }

  // row sum over both halves of the row, then O = O^T / l
  const float lt = swap32_sum(l);
  if constexpr (kSplit) {
    if (slot_out >= 0) {   // a piece: its partials, 16-byte stores contiguous over the 32 rows
      if (wave < p.part_waves) {
        const int64_t part = (int64_t)slot_out * p.part_waves + wave;
        f32x4* po = p.part_o + part * (D / 4) * 32 + (lane & 31);
#pragma unroll
        for (int db = 0; db < S::kDB; ++db)
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4)
            po[(db * 8 + 2 * r4 + hf) * 32] =
                f32x4{acc[db][r4 * 4 + 0], acc[db][r4 * 4 + 1], acc[db][r4 * 4 + 2], acc[db][r4 * 4 + 3]};
        p.part_ml[part * 64 + lane] = hf ? lt : z;
      }
      return;
    }
  }
  if (!row_ok) return;
  const float inv = lt == 0.f ? 0.f : 1.f / lt;   // zeros where no key is seen
  uint16_t* orow = p.out + q_row() * D;
#pragma unroll
  for (int db = 0; db < S::kDB; ++db)
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      const int dv = db * 32 + 8 * r4 + 4 * hf;
      const uint32_t w0 = pack_bf16(acc[db][r4 * 4 + 0] * inv, acc[db][r4 * 4 + 1] * inv);
      const uint32_t w1 = pack_bf16(acc[db][r4 * 4 + 2] * inv, acc[db][r4 * 4 + 3] * inv);
      *reinterpret_cast<uint2*>(orow + dv) = make_uint2(w0, w1);
    }
}

// The work list of the key-split launch, by one workgroup: one thread per block
// of rows.
constexpr int kPlanBlock = 1024;
constexpr int kPlanWaves = kPlanBlock / 64;
constexpr int kPairLanes = 16;   // row_reduce's
constexpr int kClasses = 8;   // 0: the pieces of cut blocks; 1..7 the other blocks by descending length

// every thread's LDS accesses before, all threads' after (__syncthreads would
// wait for the loads and stores of global memory too)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Bound by latency: four memory round trips (the head's group, its table beside
// the masks, the list cleared, the list written).
template <int D>
__global__ void __launch_bounds__(kPlanBlock) tg_prefill_mod_plan_kernel(ModParams p) {
  // per (request, row tile): least lo, greatest hi, whether a row sees the history
  __shared__ int32_t min_lo[tg::kPrefillSplitMaxBlocks], max_hi[tg::kPrefillSplitMaxBlocks];
  __shared__ int32_t any_hist[tg::kPrefillSplitMaxBlocks];
  __shared__ Walk walks[tg::kPrefillSplitMaxBlocks];
  __shared__ int2 shares[tg::kPrefillSplitMaxBlocks];
  __shared__ int32_t starts[tg::kPrefillSplitMaxBlocks];   // first entry (and partial slot) of every cut block
  __shared__ int2 sums[kPlanWaves];
  __shared__ int32_t fits[kPlanWaves];
  __shared__ int32_t counts[kClasses][kPlanWaves], in_class[kClasses];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int pairs = p.batch * p.row_tiles, blocks = pairs * p.num_kv_heads;
  const int k = threadIdx.x;
  // the block's history (threads past the last block read the last one's): asked
  // for here, used after the masks
  const int kk = min(k, blocks - 1);
  const int unit = kk / p.row_tiles, b_k = unit / p.num_kv_heads, h_k = unit % p.num_kv_heads;
  const int pair = b_k * p.row_tiles + kk % p.row_tiles;
  const int64_t bl = (int64_t)b_k * p.num_layers + p.layer;
  const TablePages table =
      table_of(p.pt_offsets, bl * p.num_groups, p.group_of[(int64_t)p.layer * p.num_kv_heads + h_k], p.num_groups);
  const int64_t len = p.kv_len[bl * p.num_kv_heads + h_k];
  for (int i = threadIdx.x; i < p.list_len; i += kPlanBlock) p.list[i].block = -1;
  // kPairLanes lanes per (request, row tile)
  const int sub = lane % kPairLanes;
  for (int at = threadIdx.x / kPairLanes; at < pairs; at += kPlanBlock / kPairLanes) {
    const int b = at / p.row_tiles, rt = at % p.row_tiles;
    const int last = min(p.chunk - 1, ((rt + 1) * kRows - 1) / p.gqa);
    const int n_valid = valid_tokens(p, b);
    int lo = INT32_MAX, hi = 0, seen = 0;
#pragma unroll 4
    for (int i = rt * kRows / p.gqa + sub; i <= last; i += kPairLanes) {
      const Seen s = row_sees(p, b, i, n_valid);
      const bool row = i < n_valid;
      lo = min(lo, row ? s.lo : INT32_MAX);
      hi = max(hi, row ? s.hi : 0);
      seen |= row && s.hist;
    }
    lo = row_reduce(lo, Least());
    hi = row_reduce(hi, Greatest());
    seen = row_reduce(seen, Greatest());
    if (sub == 0) {
      min_lo[at] = lo;
      max_hi[at] = hi;
      any_hist[at] = seen;
    }
  }
  lds_barrier();
  Walk w = {0, 0, 0};
  if (k < blocks) {
    const int hist = (int)max<int64_t>(0, min<int64_t>(len, table.pages * kPage));
    w = block_walk((hist + kTile - 1) / kTile, min_lo[pair], max_hi[pair], any_hist[pair]);
    walks[k] = w;
  }
  // the sum of all, in two parts: a block has up to 2^26 tiles
  const int low = wave_reduce(w.n_tiles & 0xffff, Sum()), high = wave_reduce(w.n_tiles >> 16, Sum());
  if (lane == 0) sums[wave] = make_int2(low, high);
  lds_barrier();
  const int2 part = sums[lane % kPlanWaves];
  const int64_t total = row_reduce(part.x, Sum()) + ((int64_t)row_reduce(part.y, Sum()) << 16);
  // T: the shortest of a few that give no more pieces than run at once, so that
  // all end together, or total / target where that is shorter: many short
  // blocks leave their places early
  constexpr int kSlots = split_at_once(D), kTarget = split_target(D);
  const int fair = (int)((total + kSlots - 1) / kSlots);
  const int try_T = max(tg::kPrefillSplitMinTiles, fair + (fair * wave + 31) / 32);   // this wave's
  int tried = 0;
  for (int i = lane; i < blocks; i += 64) tried += max(1, quotient(walks[i].n_tiles + try_T - 1, try_T));
  tried = wave_reduce(tried, Sum());
  if (lane == 0) fits[wave] = tried <= kSlots ? try_T : INT32_MAX;
  lds_barrier();
  int T = row_reduce(fits[lane % kPlanWaves], Least());
  T = min(T, (int)max<int64_t>(tg::kPrefillSplitMinTiles, (total + kTarget - 1) / kTarget));
  const int np = k < blocks ? max(1, quotient(w.n_tiles + T - 1, T)) : 0;
  // descending length: n_tiles <= T there
  const int cls = np == 0 ? -1 : np > 1 ? 0 : 7 - (int)(6.f * (float)w.n_tiles * __builtin_amdgcn_rcpf((float)T));
  // place of the block's first entry in its class: within the wave, then over the waves
  int before = 0, count = 0;   // count, lane c: entries of class c in this wave
#pragma unroll
  for (int c = 1; c < kClasses; ++c) {
    const uint64_t in = __ballot(cls == c);
    if (cls == c) before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(in >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)in, 0u));
    if (lane == c) count = __popcll(in);
  }
  const int cut = cls == 0 ? np : 0;
  const int cut_sum = wave_inclusive_sum(cut);
  const int cut_all = __builtin_amdgcn_readlane(cut_sum, 63);
  if (lane == 0) count = cut_all;
  if (lane < kClasses) counts[lane][wave] = count;
  lds_barrier();
  if (wave < kClasses) {   // counts: entries of the class in the waves before; in_class: in all
    const int c = lane < kPlanWaves ? counts[wave][lane] : 0;
    const int sum = wave_inclusive_sum(c);
    if (lane < kPlanWaves) counts[wave][lane] = sum - c;
    if (lane == 63) in_class[wave] = sum;
  }
  lds_barrier();
  if (cls > 0) before += counts[cls][wave];
  const int cut_before = counts[0][wave] + cut_sum - cut;
  if (k < blocks) {
    starts[k] = cut_before;
    const int q = quotient(w.n_tiles, np);   // tiles of a piece; the first few have one more
    shares[k] = make_int2(q, w.n_tiles - q * np);
    p.pieces[k] = make_int2(cut_before, np);
  }
  // entry r of class c: XCD 8 r / n, there behind the classes before c
  auto place = [&](int c, int r) {
    const int n = in_class[c];
    const int x = quotient(8 * r, n);   // n is at most the list's length
    int pos = r - (x * n + 7) / 8;
    for (int i = 0; i < c; ++i) pos += ((x + 1) * in_class[i] + 7) / 8 - (x * in_class[i] + 7) / 8;
    return 8 * pos + x;
  };
  __syncthreads();   // starts complete, and the list cleared before its entries are written
  if (cls > 0) p.list[place(cls, before)] = ListEntry{k, 0, w.n_tiles, w.nh, w.ct0, -1, {0, 0}};
  for (int r = threadIdx.x; r < in_class[0]; r += kPlanBlock) {
    int lo = 0, hi = blocks - 1;   // the last block that starts at or before r
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (starts[mid] <= r)
        lo = mid;
      else
        hi = mid - 1;
    }
    const Walk cw = walks[lo];
    const int2 share = shares[lo];
    const int piece = r - starts[lo], t = piece * share.x + min(piece, share.y);
    p.list[place(0, r)] = ListEntry{lo, t, t + share.x + (piece < share.y ? 1 : 0), cw.nh, cw.ct0, r, {0, 0}};
  }
}

// Merge of the key-split launch: the pieces of a block are combined at the
// largest of their reference maxima (the pieces' sums and accumulators are
// relative to them).  Grid (blocks, waves with rows x D/32): thread = (row,
// four consecutive dims), so partial loads are contiguous over a wave's 32 rows.
template <int D>
__global__ void __launch_bounds__(256) tg_prefill_mod_merge_kernel(ModParams p) {
  const int2 k = p.pieces[blockIdx.x];
  const int n = k.y;
  if (n <= 1) return;
  constexpr int kParts = D / 32;   // workgroups per 32 rows
  const int unit = blockIdx.x / p.row_tiles, rt = blockIdx.x % p.row_tiles;
  const int wave = blockIdx.y / kParts;
  const int chunk = (threadIdx.x >> 5) + 8 * (blockIdx.y % kParts);
  const int b = unit / p.num_kv_heads, h = unit % p.num_kv_heads;
  const int row = threadIdx.x & 31;
  const int r = rt * kRows + wave * kRowsPerWave + row;
  if (r >= p.chunk * p.gqa || r / p.gqa >= valid_tokens(p, b)) return;
  auto part = [&](int i) { return ((int64_t)k.x + i) * p.part_waves + wave; };
  constexpr int kBatch = 4;
  float M = -INFINITY, L = 0.f;
  f32x4 A = f32x4(0.f);
  // kBatch pieces are requested before the first is used; past the last piece
  // it is read again and not used
  for (int i0 = 0; i0 < n; i0 += kBatch) {
    float mv[kBatch], lv[kBatch];
    f32x4 ov[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int64_t pt = part(min(i0 + j, n - 1));
      mv[j] = p.part_ml[pt * 64 + row];
      lv[j] = p.part_ml[pt * 64 + 32 + row];
      ov[j] = p.part_o[(pt * (D / 4) + chunk) * 32 + row];
    }
    float Mn = M;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) Mn = fmaxf(Mn, mv[j]);
    // a piece whose keys the row does not see leaves m = -inf and zeros; while
    // there is no other, nothing is rescaled and the weights are 0
    const float Mr = Mn == -INFINITY ? 0.f : Mn;
    const float a = fast_exp2(M - Mr);
    L *= a;
    A *= a;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const bool use = i0 + j < n;
      const float w = fast_exp2(mv[j] - Mr);
      L = use ? fmaf(lv[j], w, L) : L;
#pragma unroll
      for (int q = 0; q < 4; ++q) A[q] = use ? fmaf(ov[j][q], w, A[q]) : A[q];
    }
    M = Mn;
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int Hq = p.num_kv_heads * p.gqa;
  uint16_t* orow = p.out + (((int64_t)b * p.chunk + r / p.gqa) * Hq + h * p.gqa + r % p.gqa) * D;
  *reinterpret_cast<uint2*>(orow + 4 * chunk) =
      make_uint2(pack_bf16(A[0] * inv, A[1] * inv), pack_bf16(A[2] * inv, A[3] * inv));
}

using ModFn = void (*)(ModParams);

template <bool kSplit, bool kCap>
ModFn pick_dim(int d) {
  return d == 128 ? &tg_prefill_mod_kernel<128, kSplit, 2, kCap> : &tg_prefill_mod_kernel<64, kSplit, 4, kCap>;
}

template <bool kSplit>
ModFn pick_mod(int d, bool cap) {
  return cap ? pick_dim<kSplit, true>(d) : pick_dim<kSplit, false>(d);
}

// tanh(x) / x as a polynomial in x^2 up to kCapSplit, and with one term less up to
// kNearSplit, both fitted for the smallest relative error.  They are an exponent's error
// by the score's size, so both also end at the score where it reaches 2^-13, a 32nd of
// P's own rounding: 41.8 and 33.3, which caps up to 66 and 91 do not reach within the
// splits, and past which tanh_f32 (2e-7) has it.
constexpr double kCapSplit = 0.625;
constexpr double kTanhPoly[4] = {0.99999709, -0.333092316, 0.130154592, -0.0400295162};
constexpr double kTanhError = 2.92e-6;
constexpr double kNearSplit = 0.365;
constexpr double kNearPoly[3] = {0.999996334, -0.332835182, 0.123176933};
constexpr double kNearError = 3.67e-6;
constexpr double kPolyError = 0x1p-13;

}  // namespace

extern "C" int32_t tg_prefill_mod(const tg_prefill_args* a, const tg_score_mod* mod, void* hip_stream) {
  if (int32_t rc = check_prefill(a)) return rc;
  if (!mod) return tg::fail(TG_ERR_INVALID_ARG, "mod is NULL");
  // without a cap the check is the scale's alone
  if (int32_t rc = tg::check_softcap(mod->softcap == 0.f ? 1.f : mod->softcap, a->sm_scale)) return rc;
  const tg_geometry& g = a->geom;
  const int gqa = g.num_q_heads / g.num_kv_heads;
  if (!a->q || !a->k_new || !a->v_new || !a->kv_pool || !a->pt_pages || !a->pt_offsets || !a->kv_len ||
      !a->group_of || !a->slot_of || !a->out)
    return tg::fail(TG_ERR_INVALID_ARG, "NULL device pointer");
  if (!tg::aligned16({a->q, a->k_new, a->v_new, a->kv_pool, a->out}))
    return tg::fail(TG_ERR_INVALID_ARG, "device buffers must be 16-byte aligned");
  if (a->block_order && a->num_blocks < 1) return tg::fail(TG_ERR_INVALID_ARG, "block_order needs num_blocks >= 1");
  ModParams p = {};
  p.q = static_cast<const uint16_t*>(a->q);
  p.k_new = static_cast<const u4*>(a->k_new);
  p.v_new = static_cast<const u4*>(a->v_new);
  p.pool = static_cast<const u4*>(a->kv_pool);
  p.pt_pages = a->pt_pages;
  p.pt_offsets = a->pt_offsets;
  p.kv_len = a->kv_len;
  p.group_of = a->group_of;
  p.slot_of = a->slot_of;
  p.out = static_cast<uint16_t*>(a->out);
  p.block_order = a->block_order;
  p.tokens = mod->chunk_tokens;
  p.key_begin = mod->key_begin;
  p.key_end = mod->key_end;
  p.batch = a->batch;
  p.chunk = a->chunk_len;
  p.layer = a->layer;
  p.num_layers = g.num_layers;
  p.num_kv_heads = g.num_kv_heads;
  p.num_groups = g.num_kv_heads / g.heads_per_group;
  p.heads_per_group = g.heads_per_group;
  p.gqa = gqa;
  p.row_tiles = (a->chunk_len * gqa + kRows - 1) / kRows;
  const float scale = a->sm_scale != 0.f ? a->sm_scale : 1.0f / std::sqrt((float)g.head_dim);
  p.scale_log2 = scale * kLog2e;
  const bool cap = mod->softcap > 0.f;
  if (cap) {
    p.cap_in = scale / mod->softcap;
    p.cap_log2 = mod->softcap * kLog2e;
    const double reach = kPolyError / kTanhError / mod->softcap;   // of the cap
    p.cap_split = (float)(std::min(kCapSplit, reach) / p.cap_in);
    double power = (double)p.cap_log2 * p.cap_in;
    for (int i = 0; i < 4; ++i, power *= (double)p.cap_in * p.cap_in) {
      p.poly[i] = (float)(kTanhPoly[i] * power);
      // a coefficient that is no normal number: every block takes tanh itself
      if (!std::isnormal(p.poly[i])) p.cap_split = -1.f;
    }
    p.cap_exp = p.cap_split > 0.f && reach >= kCapSplit ? (float)(2.0 * kLog2e * p.cap_in) : 0.f;
    p.near_split = p.cap_split < 0.f ? -1.f : (float)(std::min(kNearSplit, kPolyError / kNearError / mod->softcap) / p.cap_in);
    power = (double)p.cap_log2 * p.cap_in;
    for (int i = 0; i < 3; ++i, power *= (double)p.cap_in * p.cap_in) p.near[i] = (float)(kNearPoly[i] * power);
  }
  const int units = a->batch * g.num_kv_heads;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const SplitLayout sl = split_layout(g, a->batch, a->chunk_len);
  hipError_t e;
  if (sl.bytes > 0 && a->workspace && a->workspace_bytes >= sl.bytes && tg::aligned16({a->workspace})) {
    char* ws = static_cast<char*>(a->workspace);
    p.part_o = reinterpret_cast<f32x4*>(ws);
    p.part_ml = reinterpret_cast<float*>(ws + sl.o_bytes);
    p.pieces = reinterpret_cast<int2*>(ws + sl.o_bytes + sl.ml_bytes);
    p.list = reinterpret_cast<ListEntry*>(ws + sl.o_bytes + sl.ml_bytes + sl.pieces_bytes);
    p.part_waves = sl.part_waves;
    p.list_len = 8 * sl.list_per_xcd;
    auto plan = g.head_dim == 128 ? &tg_prefill_mod_plan_kernel<128> : &tg_prefill_mod_plan_kernel<64>;
    hipLaunchKernelGGL(plan, dim3(1), dim3(kPlanBlock), 0, st, p);
    e = hipGetLastError();
    if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "prefill plan launch failed: %s", hipGetErrorString(e));
    hipLaunchKernelGGL(pick_mod<true>(g.head_dim, cap), dim3(p.list_len), dim3(kBlock), 0, st, p);
    e = hipGetLastError();
    if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "prefill launch failed: %s", hipGetErrorString(e));
    auto merge = g.head_dim == 128 ? &tg_prefill_mod_merge_kernel<128> : &tg_prefill_mod_merge_kernel<64>;
    hipLaunchKernelGGL(merge, dim3(units * p.row_tiles, sl.part_waves * (g.head_dim / 32)), dim3(256), 0, st, p);
    e = hipGetLastError();
    if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "prefill merge launch failed: %s", hipGetErrorString(e));
    return TG_OK;
  }
  const int blocks = a->block_order ? a->num_blocks : 8 * ((units + 7) / 8) * p.row_tiles;
  // head_dim 64: one workgroup per CU while there are few blocks, as in tg_prefill
  const size_t one_per_cu = g.head_dim == 64 && blocks <= tg::kPrefillOnePerCuBlocks ? 24 << 10 : 0;
  hipLaunchKernelGGL(pick_mod<false>(g.head_dim, cap), dim3(blocks), dim3(kBlock), one_per_cu, st, p);
  e = hipGetLastError();
  if (e != hipSuccess) return tg::fail(TG_ERR_HIP, "prefill launch failed: %s", hipGetErrorString(e));
  return TG_OK;
}
