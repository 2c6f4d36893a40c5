// Arithmetic of the cut of attention over keys of another set (attn_kv.hip) that is the same on the host, where it is tested.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lv {

// A candidate's cost (0 or more) and its number, such that the least of these belongs to the least cost, of equal ones to the last
// candidate: a float's bits are ordered as it is.  (To 17 bits, at any size: costs are whole numbers.)
__host__ __device__ inline uint32_t cost_key(float cost, int candidate) { return (__builtin_bit_cast(uint32_t, cost) & ~63u) | (uint32_t)(63 - candidate); }
__host__ __device__ inline int candidate_of(uint32_t key) { return 63 - (int)(key & 63u); }

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
