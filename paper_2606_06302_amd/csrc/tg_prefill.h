// Shared by the chunked-prefill kernels of tg_prefill.hip and tg_prefill_mod.hip:
// tile shapes, LDS swizzles, the instructions the compiler is not asked to
// schedule, and the checks and workspace of a call.
#pragma once
#include <hip/hip_runtime.h>

#include "tg_device.h"
#include "tg_internal.h"

namespace {

using namespace tgd;

typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_vs __attribute__((__vector_size__(4 * sizeof(__bf16))));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

#define TG_CONST __attribute__((address_space(4)))
#define TG_LDS __attribute__((address_space(3)))

constexpr int kPage = 16;
constexpr int kWaves = 8;
constexpr int kBlock = 64 * kWaves;
constexpr int kCB = 1;                         // 32-row MFMA column blocks per wave
constexpr int kRowsPerWave = 32 * kCB;
constexpr int kRows = kRowsPerWave * kWaves;   // query rows per workgroup
constexpr int kTile = 64;                      // keys per tile = 4 pages
static_assert(kRows == TG_PREFILL_ROWS && kTile == TG_PREFILL_TILE, "tg_prefill_schedule costs these tiles");
constexpr int kRing = 4;                       // LDS tile buffers
static_assert(kRing >= 2 && kRing <= 4, "the wait below covers up to two tiles in flight after the current one");
constexpr int kDmaRows = kTile / kWaves;       // key rows each wave fetches per tile
constexpr float kSlack = 8.0f;

// Shape constants of the kernel for head_dim D (64 or 128).  A key row is
// 2*D bytes = kChunks 16-byte chunks; one 1 KiB DMA instruction (64 lanes x
// 16 bytes) moves kRowsPerDma rows.  LDS swizzles: chunk c of key row r of a
// tile sits at position c ^ k_swz(r) in the K tile and c ^ v_swz(r) in the V
// tile (r taken mod 16, which is also the row within its page), chosen so
// that the q.k operand reads and the transposed V reads are bank-conflict free.
template <int D>
struct Shape {
  static_assert(D == 64 || D == 128, "head_dim 64 or 128");
  static constexpr int kChunks = D / 8;
  static constexpr int kRowsPerDma = 64 / kChunks;
  static constexpr int kDmaInst = kDmaRows / kRowsPerDma;   // 1 KiB instructions per K or V slab and wave
  static constexpr int kDmaPerTile = 2 * kDmaInst;
  static constexpr int kTileBytes = 2 * kTile * D * 2;      // K + V
  static constexpr int kK = D / 16;                         // 16-deep k steps of q.k
  static constexpr int kDB = D / 32;                        // 32-dim blocks of the output
  __device__ static constexpr int k_swz(int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); }
  __device__ static constexpr int v_swz(int r) { return D == 128 ? 4 * (r & 3) : 2 * (r & 3); }
};

__device__ __forceinline__ f32x16 mfma(const u4& a, const u4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

__device__ __forceinline__ uint32_t lds_address(const void* ptr) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const TG_LDS void*)ptr));
}

// 16 bytes per lane from global memory (a wave-uniform base plus 16 * chunk
// bytes per lane) into LDS at m0_base + 16 * lane.  The scalar base keeps
// 64-bit addresses out of the vector registers.
__device__ __forceinline__ void lds_dma16(const u4* base, uint32_t chunk, uint32_t m0_base) {
  asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(chunk * 16), "s"(base), "{m0}"(m0_base) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt is 6 bits");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }

// (lo, hi) rounded to bf16 and packed into one dword (one v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2v));
}

// Lane l of each 16-lane block receives element l % 4 of the 8-byte rows
// addressed by lanes l/4, l/4 + 4, l/4 + 8, l/4 + 12 of the block.
__device__ __forceinline__ u2v lds_read_tr16(const void* ptr) {
  return __builtin_bit_cast(u2v, __builtin_amdgcn_ds_read_tr16_b64_v4bf16((TG_LDS bf16x4_vs*)ptr));
}

constexpr int split_target(int d) { return tg::prefill_split_target(d); }
// a cut unit of n tiles has at most n / T + 1 <= 2n / T pieces
constexpr int split_slots(int d) { return 2 * split_target(d); }
// workgroups that run at once: one per CU at head_dim 128, two at 64
constexpr int split_at_once(int d) { return d == 128 ? 256 : 512; }

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Workspace of the key-split launch for this shape, 0 where it is not taken.
// tg_prefill_mod also keeps its work list there.
struct SplitLayout {
  int row_tiles, part_waves, groups;
  int list_per_xcd;   // tg_prefill_mod: entries of its work list per XCD
  size_t o_bytes, ml_bytes, pieces_bytes, bytes;
};

SplitLayout split_layout(const tg_geometry& g, int batch, int chunk_len) {
  SplitLayout s = {};
  const int64_t rows = (int64_t)chunk_len * (g.num_q_heads / g.num_kv_heads);
  const int64_t row_tiles = (rows + kRows - 1) / kRows;
  const int64_t units = (int64_t)batch * g.num_kv_heads;
  if (units > tg::kPrefillSplitMaxUnits || units * row_tiles > tg::kPrefillSplitMaxBlocks) return s;
  s.row_tiles = (int)row_tiles;
  s.part_waves = (int)((rows < kRows ? rows : kRows) + 31) / 32;
  s.groups = split_target(g.head_dim) / s.row_tiles + (int)units;   // sum over units of ceil(n / T)
  const size_t parts = (size_t)split_slots(g.head_dim) * s.part_waves;
  s.o_bytes = align256(parts * 32 * g.head_dim * sizeof(float));
  s.ml_bytes = align256(parts * 64 * sizeof(float));
  s.pieces_bytes = align256((size_t)(units * row_tiles) * sizeof(int2));
  // sum over blocks of ceil(n / T) entries in eight classes, each class dealt to the 8 XCDs
  const int entries = split_target(g.head_dim) + (int)(units * row_tiles);
  s.list_per_xcd = (entries > split_at_once(g.head_dim) ? entries : split_at_once(g.head_dim)) / 8 + 9;
  s.bytes = s.o_bytes + s.ml_bytes + s.pieces_bytes + align256((size_t)s.list_per_xcd * 8 * tg::kPrefillListEntryBytes);
  return s;
}

int32_t check_prefill(const tg_prefill_args* a) {
  if (!a) return tg::fail(TG_ERR_INVALID_ARG, "args is NULL");
  const tg_geometry& g = a->geom;
  if (int32_t rc = tg::check_geometry(&g)) return rc;
  if (a->dtype != TG_BF16) return tg::fail(TG_ERR_UNSUPPORTED, "prefill supports bf16 only");
  if (g.head_dim != 64 && g.head_dim != 128)
    return tg::fail(TG_ERR_UNSUPPORTED, "prefill supports head_dim 64 or 128 (got %d)", g.head_dim);
  if (g.page_size != kPage) return tg::fail(TG_ERR_UNSUPPORTED, "prefill supports page_size 16 only");
  const int gqa = g.num_q_heads / g.num_kv_heads;
  if (gqa < 1 || gqa > 16) return tg::fail(TG_ERR_UNSUPPORTED, "prefill supports 1..16 query heads per KV head");
  if (a->batch < 1 || a->chunk_len < 1 || a->layer < 0 || a->layer >= g.num_layers)
    return tg::fail(TG_ERR_INVALID_ARG, "batch and chunk_len must be >= 1, layer in range");
  return TG_OK;
}

}  // namespace
