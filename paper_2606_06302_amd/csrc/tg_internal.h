// Internal helpers shared by the host and device translation units of
// libtangram.so (not part of the public ABI).
#pragma once
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <initializer_list>

#include "tangram.h"

namespace tg {

// Records a thread-local message for tg_last_error() and returns `code`.
int32_t fail(int32_t code, const char* fmt, ...);

// Validates a geometry for the host integer calls.  On failure records a
// message and returns TG_ERR_INVALID_ARG.
int32_t check_geometry(const tg_geometry* g);

// Validates the score cap of the calls that take one, and their softmax scale
// (a negative one would turn the running maximum into a minimum).
int32_t check_softcap(float softcap, float sm_scale);

// What the decode calls share: the shapes they take, their arguments (ws_ptr of
// ws_bytes bytes standing for the workspace), and the merge of the split units'
// partials as a launch of its own: in one chain per unit where the plan has few
// pieces a unit, which the kernels may then merge themselves.
int32_t check_decode_shape(const tg_geometry* g, int dtype);
int32_t check_decode_args(const tg_decode_args* a, const void* ws_ptr, size_t ws_bytes);
bool decode_merges_in_one_chain(const tg_decode_args* a);
int32_t launch_decode_merge(const tg_decode_args* a, const float* part_o, const float* part_lse, void* hip_stream);

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// True when every pointer given is 16-byte aligned (NULL counts as aligned):
// the device calls move Q, K, V, outputs, partials and pool rows with 8- and
// 16-byte vector accesses.
inline bool aligned16(std::initializer_list<const void*> ptrs) {
  for (const void* q : ptrs)
    if (reinterpret_cast<uintptr_t>(q) & 15u) return false;
  return true;
}

// The cut of the key-split prefill launch, made on the device and foreseen by
// tg_prefill_split_pays: pieces of at least kPrefillSplitMinTiles key tiles,
// about prefill_split_target() of them, for at most so many units and blocks.
constexpr int kPrefillSplitMinTiles = 3;
constexpr int kPrefillSplitMaxUnits = 512;    // one thread of a workgroup per unit
constexpr int kPrefillSplitMaxBlocks = 1024;  // past it blocks outnumber the CUs by far and even out by themselves
// A little under the workgroups that run at once (one per CU at head_dim 128,
// two at 64), because cutting into equal pieces rounds up.  One request, chunk
// 512, 16384 tokens, with 160 / 208 / 256 / 320: 94 / 81 / 110 / 99 us at 128.
// At 64, chunk 512, with 352 / 448 / 512: one request over 16384 tokens 60 / 56
// / 65 us, two over 8192 61 / 57 / 68, four 95 / 109 / 110; over 57 shapes 0.99
// / 1 / 1.02.
constexpr int prefill_split_target(int head_dim) { return head_dim == 128 ? 208 : 448; }
// One entry of tg_prefill_mod's work list.
constexpr int kPrefillListEntryBytes = 32;
// Whole-block launches of head_dim 64 with more blocks than this run two
// workgroups per CU.
constexpr int kPrefillOnePerCuBlocks = 512;

}  // namespace tg
