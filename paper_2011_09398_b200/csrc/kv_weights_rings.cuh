// What the warps of the kernels for attention weights of many rows (kv_weights_prompt.cu) may be ahead of one another by: plain
// arithmetic, no CUDA headers, so that every order in which they can take their steps can be walked through without a GPU.
//
// A block's units come one after the other; each has some steps, and in each step one product, or one for each half of what stays where there
// is a second half.  Each half has two accumulators, which its steps use in turn: step s may be issued when step s - 2 of that half is read
// out (phase s / 2 of barrier s % 2).
//
// What the warps that decode keys say about a tile of them lies in a ring of eight places, which nobody waits for: it is read before a step's
// accumulator is given back, and so what is written there is held back by the products.
//   first kernel    a place for each tile of keys, which streams.  The tile behind the one that the products have begun is decoded at most two
//                   tiles ahead, and the products are two steps ahead of a half that has not read its own: less than eight
//   second kernel   two places for each unit, whose keys stay: a half's two steps may be of two units, decoding is two units ahead of the
//                   products: less than four units
// Both hold for the second half only while units have one.  So a unit without one begins when the second half has read out all it was given.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define LCE_KV_BOTH __host__ __device__ __forceinline__
#else
#define LCE_KV_BOTH inline
#endif

namespace lce {

constexpr uint32_t kInfos = 8;

// Place of what is said about tile `tile`, counted through the block (first kernel), or about the unit's half (second; units that have steps).
LCE_KV_BOTH uint32_t info_place(bool second_kernel, uint32_t tile, uint32_t unit, uint32_t half) { return (second_kernel ? 2 * unit + half : tile) % kInfos; }

// Barrier and parity of a half's step.
LCE_KV_BOTH uint32_t step_buffer(uint32_t step) { return step & 1; }
LCE_KV_BOTH uint32_t step_parity(uint32_t step) { return step >> 1 & 1; }

// Calls wait(half, step) for the step that must have been read out before a unit with so many halves begins, and before a half's next
// step.  steps: of each half so far.
template <class Wait>
LCE_KV_BOTH bool before_unit(int halves, const uint32_t (&steps)[2], const Wait &wait)
{
    return halves == 2 || steps[1] == 0 || wait(1, steps[1] - 1);
}
template <class Wait>
LCE_KV_BOTH bool before_step(int half, const uint32_t (&steps)[2], const Wait &wait)
{
    return steps[half] < 2 || wait(half, steps[half] - 2);
}

}  // namespace lce
