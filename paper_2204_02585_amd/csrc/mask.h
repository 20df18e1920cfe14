// The masks of dropout: made from a counter wherever they are needed, never
// stored.
//
// Element (row, col) of a matrix of `cols` columns takes 32 bits of word number
// row * pairs + col / 2, pairs = ceil(cols / 2), of a SplitMix64 stream (Steele,
// Lea & Flood 2014): the low half for an even column.  Two elements share a
// word, whose two 64-bit products are most of what a mask costs; a row starts
// with a word of its own, so that runs of an even number of columns never split
// one.  The stream starts at the mixed seed: streams of seeds that follow each
// other would otherwise be the same words, shifted.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sqn {

struct Mask {
    uint64_t seed;
    const uint64_t* step;    // device, added to the seed, or null
    uint32_t on;             // 0: everything is kept, unscaled
    uint32_t all;            // 1: everything is dropped
    uint32_t bound;          // bits below it are dropped
    float scale;             // of what is kept
    uint64_t pairs;          // words of a row
};

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;

__device__ __forceinline__ uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// Where the stream starts.
__device__ __forceinline__ uint64_t mask_key(const Mask& m)
{
    return mix64(m.seed + (m.step ? *m.step : 0));
}

// v[k] for columns col + k of a row, col even: times `scale` where kept, 0
// where dropped (whatever it was).
template <int V>
__device__ __forceinline__ void apply_mask(const Mask& m, uint64_t key, uint64_t row, uint32_t col, float scale, float (&v)[V])
{
    static_assert(V % 2 == 0, "whole words");
    uint64_t at = key + (row * m.pairs + (col >> 1) + 1) * kGolden;
#pragma unroll
    for (int k = 0; k < V; k += 2, at += kGolden) {
        const uint64_t word = mix64(at);
        const bool low = m.all || static_cast<uint32_t>(word) < m.bound, high = m.all || static_cast<uint32_t>(word >> 32) < m.bound;
        v[k] = low ? 0.0f : v[k] * scale;
        v[k + 1] = high ? 0.0f : v[k + 1] * scale;
    }
}

}  // namespace sqn
