// Arithmetic of the cut of attention over keys of another set (attn_kv.hip) that is the same on the host, where it is tested.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lv {

// Where a sequence's units (or slots) begin: what the sequences before it have, `before` + `own`, and no more than there is room for.  With
// offsets that ascend the room is never reached; with others every sequence may claim all rows, and a sum of 32 bits would wrap.
__host__ __device__ inline int start_of(int before, int own, int room) { return before + own < room ? before + own : room; }
// One sequence's share of such a sum (64 of them stay below 2^31: room is below 2^24)
__host__ __device__ inline int share_of(int own, int room) { return own < room ? own : room; }

// Whether a sequence of `units` units has number `local` of them, and the workspace the slot of it (cut: it needs one).  Numbers below 0
// are none: offsets that do not ascend make the starts say nothing.
__host__ __device__ inline bool unit_there(int local, int units, bool cut, int slot, int slots) {
  return (uint32_t)local < (uint32_t)units && (!cut || (uint32_t)slot < (uint32_t)slots);
}

}  // namespace lv
