// How the attention's lines of work are cut (prefix_attention.hip): integer arithmetic only, host and device.
//
// A line is a run of steps, cut into `parts` stretches of equal length.  It consists of units, a unit of items that take the same
// number of steps each, so a step of a unit lies in item offset / steps of it.  An item's steps fit 32 bits, a unit's do not: 65,536 items
// of 32,772 steps (4096 rows of 128 queries a key head and eight key heads, on a prefix of 2^20 tokens) are more than 2^31.  A line has
// less than 2^53 of them (fewer than 2^27 items of fewer than 2^26 steps), so products with up to 768 (lines of workgroups) and, with
// 2^51 steps, 3072 parts (lines of waves) stay below 2^63.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace e3 {

// x / by, x >= 0, by > 0 (in 32 bits where both fit: a division in 64 takes a hundred instructions more)
__host__ __device__ __forceinline__ int64_t divide(int64_t x, int64_t by)
{
    return (uint64_t)(x | by) >> 32 == 0 ? (int64_t)((uint32_t)x / (uint32_t)by) : x / by;
}

// stretch w: steps [begin_of(w), begin_of(w + 1)); and the stretch that holds a step
__host__ __device__ __forceinline__ int64_t begin_of(int w, int64_t steps, int parts) { return divide(w * steps, parts); }
__host__ __device__ __forceinline__ int part_of(int64_t step, int64_t steps, int parts)
{
    return (int)divide((step + 1) * parts + steps - 1, steps) - 1;
}

// The item of a unit that holds the unit's step `offset`, and how much of it lies in the next `left` steps.
struct Piece { int item, from, n; };
__host__ __device__ __forceinline__ Piece piece_at(int64_t offset, int64_t left, int item_steps)
{
    Piece p;
    p.item = (int)divide(offset, item_steps);
    p.from = (int)(offset - (int64_t)p.item * item_steps);
    p.n = left < item_steps - p.from ? (int)left : item_steps - p.from;
    return p;
}

}  // namespace e3
