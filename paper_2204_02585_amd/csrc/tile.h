// Tiles of products C = P Q^T whose factors have their rows contiguous along
// the sum, on the 32 x 32 matrix instructions.
//
// A workgroup computes a tile of C.  The sum goes in steps of 128 bytes (a
// line of the caches) of every row, 64 binary16 or 256 4-bit elements, whose
// rows stream from global memory straight into one of the LDS buffers.  A step
// is four instructions deep: instruction o takes from row r, in lane r % 32 +
// 32 g, the row's 16-byte piece 4 g + o.  (Any assignment of pieces to lanes
// gives the same sum; with this one a lane's scales of 4-bit elements lie side
// by side.)  Piece c of row r lies in slot c ^ (r / 2 % 8) of its row: two rows
// take the 64 banks once, so of the lanes that LDS serves together those in rows
// of one parity must differ in their slot (with r % 8 a third of the LDS
// cycles were conflicts).
//
// A depth's fragments are read between the products of the one before.  The
// barrier of a step stands before its last depth, whose fragments are then in
// registers: behind it the buffer takes the step that comes when all others are
// through, and the next step's first fragments can be read at once.  So with
// two buffers a step's loads have a whole step to land, with four (the tiles
// of 64, whose steps are short) three, and no reads wait behind a barrier.
//
// A wave's part of C is FM x FN accumulators of 32 x 32: element q of a lane is
// row 8 (q / 4) + 4 (lane / 32) + q % 4, column lane % 32.  Two waves share a
// SIMD (eight waves in the largest tile, two workgroups of four otherwise),
// one where high and low parts of the factors fill a CU's LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "numeric.h"

namespace sqn {

typedef float float16v __attribute__((ext_vector_type(16)));

constexpr uint32_t kStepBytes = 128;         // of a row, a step
constexpr uint32_t kSlot = 16;
constexpr uint32_t kBlockBytes = 32 * kStepBytes;    // of the rows of an instruction
constexpr int kDepths = 4;

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

// Byte of piece 4 (lane / 32) + o of row lane % 32, from the wave's first row.
__device__ __forceinline__ uint32_t piece_at(uint32_t lane, uint32_t o)
{
    return (lane & 31) * kStepBytes + ((4 * (lane >> 5) + o) ^ (lane >> 1 & 7)) * kSlot;
}

// This wave's loads into LDS but the LATER newest have landed, its reads are
// done, and so for every wave of the workgroup.
template <int LATER>
__device__ __forceinline__ void landed()
{
    static_assert(LATER < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    // vmcnt(LATER) lgkmcnt(0); through the builtin, so that the compiler knows
    // what has landed and adds no waits for it
    __builtin_amdgcn_s_waitcnt((LATER & 15) | 0x70 | (LATER >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// This wave's loads into LDS but the LATER newest have landed, for itself.
template <int LATER>
__device__ __forceinline__ void landed_own()
{
    static_assert(LATER < 64, "vmcnt has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LATER & 15) | 0xf70 | (LATER >> 4) << 14);
    asm volatile("" ::: "memory");
}

// This wave's reads of LDS are in registers: what they read may be loaded over.
__device__ __forceinline__ void reads_done()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
}

// A kernel's LDS for the steps of shape S: arrays of their own, so that reads of
// one do not wait for loads into another.
#define BUFFERS_IN_LDS(S)                                                            \
    __shared__ __align__(16) char buffer0[S::BUFFER];                                \
    __shared__ __align__(16) char buffer1[S::BUFFER];                                \
    __shared__ __align__(16) char buffer2[S::BUFFERS == 4 ? S::BUFFER : 16];         \
    __shared__ __align__(16) char buffer3[S::BUFFERS == 4 ? S::BUFFER : 16];         \
    char* buffers[S::BUFFERS];                                                       \
    buffers[0] = buffer0;                                                            \
    buffers[1] = buffer1;                                                            \
    if constexpr (S::BUFFERS == 4) {                                                 \
        buffers[2] = buffer2;                                                        \
        buffers[3] = buffer3;                                                        \
    }

// The steps of a tile's sum.  bring(step, buffer) issues LOADS loads a wave,
// read(fragments, buffer, o) reads a depth's fragments and multiply(fragments,
// depth) multiplies them: the steps go in rounds of as many as there are
// buffers, the last round may end early.  ahead(step, in_round) starts what a
// step takes from elsewhere.
template <int LOADS, typename Fragments, int BUFFERS, typename A, typename B, typename R, typename M>
__device__ __forceinline__ void pipeline(uint32_t steps, char* (&buffers)[BUFFERS], A ahead, B bring_step, R read,
                                         M multiply)
{
    const uint32_t end = steps - 1;
    Fragments f0, f1;
#pragma unroll
    for (int b = 0; b < BUFFERS - 1; ++b)
        ahead(min(static_cast<uint32_t>(b), end), b);
#pragma unroll
    for (int b = 0; b < BUFFERS; ++b)
        bring_step(min(static_cast<uint32_t>(b), end), buffers[b]);
    landed<(BUFFERS - 1) * LOADS>();
    read(f0, buffers[0], 0);
    // buffer b holds step k and will hold k + BUFFERS; past the end the last step
    // comes once more and is not used
    auto work = [&](uint32_t k, int b) {
        ahead(min(k + BUFFERS - 1, end), (b + BUFFERS - 1) % BUFFERS);
        read(f1, buffers[b], 1);
        multiply(f0, kDepths * b);
        read(f0, buffers[b], 2);
        multiply(f1, kDepths * b + 1);
        read(f1, buffers[b], 3);
        multiply(f0, kDepths * b + 2);
        // what `ahead` loads may be among the newest too: then more has landed
        landed<(BUFFERS - 2) * LOADS>();
        bring_step(min(k + BUFFERS, end), buffers[b]);
        read(f0, buffers[(b + 1) % BUFFERS], 0);
        multiply(f1, kDepths * b + 3);
    };
    uint32_t k = 0;
    for (; k + BUFFERS <= steps; k += BUFFERS) {
#pragma unroll
        for (int b = 0; b < BUFFERS; ++b)
            work(k + b, b);
    }
#pragma unroll
    for (int b = 0; b < BUFFERS - 1; ++b)
        if (k + b < steps)
            work(k + b, b);
    // the loads still under way end before their buffers do
    landed<0>();
}

// f(row, column, elements) over a wave's accumulators, from its first row and
// column: element q is at row + row_of(q).  The loads of one row of blocks are
// under way together; those of more would not fit the registers.
template <int FM, int FN, typename F>
__device__ __forceinline__ void each_block(float16v (&acc)[FM][FN], F f)
{
    const uint32_t lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < FM; ++s) {
#pragma unroll
        for (int t = 0; t < FN; ++t)
            f(32 * s + 4 * (lane >> 5), 32 * t + (lane & 31), acc[s][t]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

constexpr uint32_t row_of(int q) { return 8 * (q >> 2) + (q & 3); }

// ---- a wave's part of C on its way out
//
// As the lanes hold it, C would leave in pieces of 8 to 32 bytes, and cache
// lines go to memory more than once (of a product's outputs 1.9 times).  It
// goes through LDS instead, kOwn bytes of it a wave, and leaves in runs of 16
// bytes that fill lines: emit(column, row, run) for runs down the columns,
// emit(row, column, run) for runs along the rows, from the wave's first row
// and column.  convert(value) is an element as it is stored.

template <int FM>
constexpr int kOwn = FM * 32 * 32 * 4;

// The wave's own bytes of the buffers.
template <int FM, int BUFFER>
__device__ __forceinline__ char* own_part(char* b0, char* b1, uint32_t wave)
{
    static_assert(BUFFER % kOwn<FM> == 0, "no part lies in both buffers");
    const int at = static_cast<int>(wave) * kOwn<FM>;
    return at < BUFFER ? b0 + at : b1 + at - BUFFER;
}

// LDS accesses of a wave stay on their side.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// COUNT rows of blocks from S0 on; kOwn<COUNT> bytes.
template <typename T, int S0, int COUNT, int FM, int FN, typename C, typename E>
__device__ __forceinline__ void columns_out_of(const float16v (&acc)[FM][FN], char* own, C convert, E emit)
{
    constexpr int WORDS = sizeof(T);                              // of four elements
    constexpr uint32_t PITCH = COUNT * 32 * sizeof(T), PIECES = PITCH / 16;
    const uint32_t lane = threadIdx.x & 63, half = lane >> 5, mine = lane & 31;
#pragma unroll
    for (int t = 0; t < FN; ++t) {
#pragma unroll
        for (int s = 0; s < COUNT; ++s) {
            uint32_t word[4][WORDS];
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                T e[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    e[r] = convert(acc[S0 + s][t][4 * g + r]);
                __builtin_memcpy(word[g], e, sizeof(e));
            }
            // the lower half of the wave gives its groups 2 and 3 for the upper
            // half's 0 and 1: a lane then has 16 rows running
            uint32_t run[WORDS][4];
            uint32_t* flat = &run[0][0];
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int w = 0; w < WORDS; ++w) {
                    const auto swapped = __builtin_amdgcn_permlane32_swap(word[g][w], word[g + 2][w], false, false);
                    flat[2 * g * WORDS + w] = swapped[0];
                    flat[(2 * g + 1) * WORDS + w] = swapped[1];
                }
#pragma unroll
            for (int k = 0; k < WORDS; ++k) {
                const uint32_t at = (2 * s + half) * WORDS + k;       // piece of the column
                *reinterpret_cast<uint4*>(own + mine * PITCH + (at ^ (mine & (PIECES - 1))) * 16)
                    = uint4{run[k][0], run[k][1], run[k][2], run[k][3]};
            }
        }
        wave_fence();
#pragma unroll
        for (uint32_t i = 0; i < 32 * PIECES / 64; ++i) {
            const uint32_t column = (64 * i + lane) / PIECES, at = lane & (PIECES - 1);
            emit(32 * t + column, 32 * S0 + at * (16 / sizeof(T)),
                 *reinterpret_cast<const uint4*>(own + column * PITCH + (at ^ (column & (PIECES - 1))) * 16));
        }
        wave_fence();
    }
}

template <typename T, int FM, int FN, typename C, typename E>
__device__ __forceinline__ void columns_out(const float16v (&acc)[FM][FN], char* own, C convert, E emit)
{
    columns_out_of<T, 0, FM>(acc, own, convert, emit);
}

template <typename T, int FM, int FN, typename C, typename E>
__device__ __forceinline__ void rows_out(const float16v (&acc)[FM][FN], char* own, C convert, E emit)
{
    constexpr uint32_t PITCH = FN * 32 * sizeof(T), PIECES = PITCH / 16;
    const uint32_t lane = threadIdx.x & 63, mine = lane & 31;
    // rows r and r + 4 are written together: apart by half a row
    auto slot = [](uint32_t row, uint32_t piece) { return row * PITCH + (piece ^ (row >> 2 & 1) * (PIECES / 2)) * 16; };
#pragma unroll
    for (int s = 0; s < FM; ++s) {
#pragma unroll
        for (int t = 0; t < FN; ++t)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const uint32_t byte = (32 * t + mine) * sizeof(T);
                *reinterpret_cast<T*>(own + slot(row_of(q) + 4 * (lane >> 5), byte >> 4) + (byte & 15)) = convert(acc[s][t][q]);
            }
        wave_fence();
#pragma unroll
        for (uint32_t i = 0; i < 32 * PIECES / 64; ++i) {
            const uint32_t row = (64 * i + lane) / PIECES, at = lane & (PIECES - 1);
            emit(32 * s + row, at * (16 / sizeof(T)), *reinterpret_cast<const uint4*>(own + slot(row, at)));
        }
        wave_fence();
    }
}

// A run of 16 bytes to `to`, of whose places `left` are inside the matrix.
template <typename T>
__device__ __forceinline__ void store_inside(T* to, int64_t left, const uint4& run)
{
    constexpr int N = 16 / sizeof(T);
    if (left >= N) {
        Run<T, N> r;
        __builtin_memcpy(&r, &run, 16);
        *reinterpret_cast<Run<T, N>*>(to) = r;
    } else {
        T e[N];
        __builtin_memcpy(e, &run, 16);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < left)
                to[k] = e[k];
    }
}

}  // namespace sqn
