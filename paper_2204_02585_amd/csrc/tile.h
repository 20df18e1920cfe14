// Tiles of products C = P Q^T whose factors have their rows contiguous along
// the sum, on the 32 x 32 matrix instructions.
//
// A workgroup of WM x WN waves computes TM x TN of C.  The sum goes in steps of
// 128 bytes of every row (64 binary16 or 256 4-bit elements): the rows of a
// step stream from global memory straight into LDS, into one buffer while the
// matrix cores work on the other, one barrier a step.  A step is four
// instructions deep: instruction o takes from row r, in lane r % 32 + 32 g, the
// row's 16-byte piece 4 g + o.  (Any assignment of pieces to lanes gives the
// same sum; this one lets a lane's four scales of a 4-bit step lie side by
// side.)  Piece c of row r lies in slot c ^ (r / 2 % 8) of its row: two rows
// take the 64 banks once, so of the lanes that LDS serves together those in rows
// of one parity must differ in their slot (with r % 8 instead a third of the
// LDS cycles were conflicts).
//
// A wave's part of C is FM x FN accumulators of 32 x 32: element q of a lane is
// row 8 (q / 4) + 4 (lane / 32) + q % 4, column lane % 32.
//
// Two waves share a SIMD in every shape (eight waves in the largest tile, two
// workgroups of four otherwise): one wave with the whole register file needs
// fewer LDS reads per product, but kept moving its 256 accumulators about.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace sqn {

typedef float float16v __attribute__((ext_vector_type(16)));

constexpr uint32_t kStepBytes = 128;         // of a row, a step
constexpr uint32_t kSlot = 16;

// 8 rows of a step, 64 pieces, by one wave: lane l brings slot l % 8 of row l / 8.
// `from` is the lane's own piece, `to` the wave's 1024 bytes.
__device__ __forceinline__ void bring(const char* from, char* to)
{
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint32_t*>(from), reinterpret_cast<uint32_t*>(to), kSlot, 0, 0);
}

// The piece that a lane brings into the group of 8 rows `group`.
__device__ __forceinline__ uint32_t brought_piece(uint32_t lane, uint32_t group)
{
    return (lane & 7) ^ (4 * (group & 1) + (lane >> 4));
}

// Byte of piece 4 (lane / 32) + o of row lane % 32 in a step's buffer, from the
// wave's first row.
__device__ __forceinline__ uint32_t piece_at(uint32_t lane, uint32_t o)
{
    return (lane & 31) * kStepBytes + ((4 * (lane >> 5) + o) ^ (lane >> 1 & 7)) * kSlot;
}

// f(row, column, elements) over a wave's accumulators, from its first row and
// column: element q is at row + row_of(q).
template <int FM, int FN, typename F>
__device__ __forceinline__ void each_block(const float16v (&acc)[FM][FN], F f)
{
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < FM; ++s)
#pragma unroll
        for (int t = 0; t < FN; ++t)
            f(32 * s + 4 * (lane >> 5), 32 * t + (lane & 31), acc[s][t]);
}

constexpr uint32_t row_of(int q) { return 8 * (q >> 2) + (q & 3); }

}  // namespace sqn
