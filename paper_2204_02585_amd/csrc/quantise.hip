// Matrices in 4-bit blocks (MXFP4: 32 E2M1 elements and an E8M0 scale) and
// the layers evaluated on them.
#include <type_traits>

#include "learn.h"
#include "numeric.h"
#include "sqn_internal.h"
#include "tile.h"

namespace sqn {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr uint32_t kOne = 127;           // E8M0 of 1

// ---- to blocks and back: four lanes share a block, eight elements each

struct QuantParams {
    const void* x;
    void* values;
    uint8_t* codes;
    uint8_t* scales;
    uint64_t items;          // eighths: rows * blocks * 4
    int64_t stride;          // elements
    uint32_t cols, blocks;
};

// Row and place in it of item i of a matrix with `per_row` in a row.  The 64-bit
// division is most of a kernel's instructions, so it is left to matrices of
// 2^32 items or more.
__device__ __forceinline__ void split_item(uint64_t i, uint32_t per_row, uint64_t items, uint32_t& row, uint32_t& at)
{
    row = items >> 32 ? static_cast<uint32_t>(i / per_row) : static_cast<uint32_t>(i) / per_row;
    at = static_cast<uint32_t>(i) - row * per_row;
}

// ---- scales beside the tiles' products
//
// An instruction of a tile takes 32 rows, and a lane of it a scale byte, that
// of block 8 k + 4 g + o of row lane % 32 for instruction o of step k, with g =
// lane / 32.  The packed scales of a matrix hold these bytes as the lanes take
// them: a word for each of 64 lanes (o its byte) for each step of each 32 rows.
// Blocks past the matrix's have the scale of 1, so that the zeros there stay
// zeros.

struct PackedScales {
    uint8_t* to;             // [rows / 32, rounded up to a tile][steps][64] words
    uint32_t steps;
};

__host__ __device__ constexpr uint32_t steps_of(uint32_t blocks) { return (blocks + 7) / 8; }

// Where the byte of a row's block lies.
__device__ __forceinline__ uint64_t packed_at(uint32_t row, uint32_t block, uint32_t steps)
{
    const uint32_t lane = (row & 31) + 32 * (block >> 2 & 1);
    return (static_cast<uint64_t>(row >> 5) * steps + (block >> 3)) * 256 + 4 * lane + (block & 3);
}

struct PackParams {
    const uint8_t* from;     // [rows][blocks]
    PackedScales packed;
    uint64_t words;          // rows * steps * 2
    uint32_t blocks;
    // codes to copy with rows filled up to whole steps by zeros, or null
    const uint4* codes;
    uint4* codes_to;
};

// A workgroup's share of the words: row by row, a word of four blocks a thread.
__device__ __forceinline__ void pack_share(const PackParams& p, uint32_t group, uint32_t groups)
{
    const uint32_t per_row = 2 * p.packed.steps;
    for (uint64_t i = static_cast<uint64_t>(group) * kThreads + threadIdx.x; i < p.words;
         i += static_cast<uint64_t>(groups) * kThreads) {
        uint32_t row, block;
        split_item(i, per_row, p.words, row, block);
        block *= 4;
        uint32_t word = 0;
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
            word |= (block + k < p.blocks ? p.from[static_cast<uint64_t>(row) * p.blocks + block + k] : kOne) << (8 * k);
        *reinterpret_cast<uint32_t*>(p.packed.to + packed_at(row, block, p.packed.steps)) = word;
        if (p.codes) {
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k)
                p.codes_to[row * static_cast<uint64_t>(4 * per_row) + block + k]
                    = block + k < p.blocks ? p.codes[static_cast<uint64_t>(row) * p.blocks + block + k] : uint4{0, 0, 0, 0};
        }
    }
}

// Two matrices' scales (of Quantised factors).
__global__ __launch_bounds__(kThreads) void pack_kernel(PackParams a, PackParams b, uint32_t groups_a)
{
    if (blockIdx.x < groups_a)
        pack_share(a, blockIdx.x, groups_a);
    else
        pack_share(b, blockIdx.x - groups_a, gridDim.x - groups_a);
}

// The largest magnitude's exponent field (0 for subnormals and zero) to the
// block's scale byte; 255 marks a NaN or an infinity.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits)
{
    const uint32_t e = top_bits >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}

// Eight elements of a row as they lie in memory.
template <typename T>
using Eight = Run<T, 8>;

// The largest magnitude's bits, of T.
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Eight<T>& e)
{
    uint32_t top = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            top = max(top, e.word[k] & 0x7fffffffu);
    } else {
        typedef uint16_t ushort2v __attribute__((ext_vector_type(2)));
        ushort2v most = {0, 0};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            most = __builtin_elementwise_max(most, __builtin_bit_cast(ushort2v, e.word[k] & 0x7fff7fffu));
        top = max(most[0], most[1]);
    }
    return top;
}

// ... to the block's scale byte.
template <typename T>
__device__ __forceinline__ uint32_t byte_of(uint32_t top)
{
    if constexpr (sizeof(T) == 4)
        return scale_byte(top);
    else
        return scale_byte(__float_as_uint(to_f32(__builtin_bit_cast(T, static_cast<uint16_t>(top)))));
}

// Eight elements over 2^(byte - 127), as codes: rounded to nearest even, at
// most 6.
template <typename T>
__device__ __forceinline__ uint32_t encode(const Eight<T>& e, uint32_t byte)
{
    // a marked block's codes are those of scale 1
    const float scale = byte == 255 ? 1.0f : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
    uint32_t c = 0;
    if constexpr (sizeof(T) == 4) {
        float v[8];
        __builtin_memcpy(v, &e, sizeof(v));
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
    } else {
        typedef T pair __attribute__((ext_vector_type(2)));
        pair v[4];
        __builtin_memcpy(v, &e, sizeof(v));
        if constexpr (std::is_same<T, _Float16>::value) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, v[0], scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, v[1], scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, v[2], scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, v[3], scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[0], scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[1], scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[2], scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, v[3], scale, 3);
        }
    }
    return c;
}

// Elements at..at+8 of a row, zeros past its end.
template <typename T>
__device__ __forceinline__ Eight<T> load_eight(const T* row, uint32_t at, uint32_t cols)
{
    Eight<T> e;
    if (at + 8 <= cols) {
        e = *reinterpret_cast<const Eight<T>*>(row + at);
    } else {
        T v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = at + k < cols ? row[at + k] : from_f32<T>(0.0f);
        __builtin_memcpy(&e, v, sizeof(e));
    }
    return e;
}

// The scale byte of four lanes' elements.
template <typename T>
__device__ __forceinline__ uint32_t shared_scale(const Eight<T>& e)
{
    uint32_t top = top_of<T>(e);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
    return byte_of<T>(top);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void quantise_kernel(QuantParams p)
{
    const uint32_t per_row = 4 * p.blocks;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.items;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        uint32_t r, q;
        split_item(i, per_row, p.items, r, q);
        const Eight<T> e = load_eight<T>(static_cast<const T*>(p.x) + r * p.stride, 8 * q, p.cols);
        const uint32_t byte = shared_scale<T>(e);
        reinterpret_cast<uint32_t*>(p.codes)[i] = encode<T>(e, byte);
        if ((i & 3) == 0)
            p.scales[i >> 2] = static_cast<uint8_t>(byte);
    }
}

// x to blocks with their scales packed, and by further workgroups the scales
// of w.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantise_packed_kernel(QuantParams p, PackedScales packed, PackParams w,
                                                                   uint32_t groups)
{
    if (blockIdx.x >= groups) {
        pack_share(w, blockIdx.x - groups, gridDim.x - groups);
        return;
    }
    // all blocks of the steps, zeros in those past the matrix
    const uint32_t per_row = 32 * packed.steps;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.items;
         i += static_cast<uint64_t>(groups) * kThreads) {
        uint32_t r, q;
        split_item(i, per_row, p.items, r, q);
        const uint32_t block = q >> 2;
        uint32_t byte = kOne, codes = 0;
        if (block < p.blocks) {
            const Eight<T> e = load_eight<T>(static_cast<const T*>(p.x) + r * p.stride, 8 * q, p.cols);
            byte = shared_scale<T>(e);
            codes = encode<T>(e, byte);
        }
        reinterpret_cast<uint32_t*>(p.codes)[i] = codes;
        if ((q & 3) == 0)
            packed.to[packed_at(r, block, packed.steps)] = static_cast<uint8_t>(byte);
    }
}

// The values of eight codes, rounded once to T: NaN for a marked block.
template <typename T>
__device__ __forceinline__ Eight<T> decode(uint32_t codes, uint32_t byte)
{
    const float scale = byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
    Eight<T> e;
    typedef T pair __attribute__((ext_vector_type(2)));
    pair v[4];
    if constexpr (sizeof(T) == 4) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    } else if constexpr (std::is_same<T, _Float16>::value) {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3);
    } else {
        v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
        v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
        v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
        v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    }
    if (byte == 255) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = pair{from_f32<T>(__builtin_nanf("")), from_f32<T>(__builtin_nanf(""))};
    }
    __builtin_memcpy(&e, v, sizeof(e));
    return e;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void values_kernel(QuantParams p)
{
    const uint32_t per_row = 4 * p.blocks;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.items;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        uint32_t r, q;
        split_item(i, per_row, p.items, r, q);
        const Eight<T> e = decode<T>(reinterpret_cast<const uint32_t*>(p.codes)[i], p.scales[i >> 2]);
        T* row = static_cast<T*>(p.values) + r * p.stride;
        if (8 * q + 8 <= p.cols) {
            *reinterpret_cast<Eight<T>*>(row + 8 * q) = e;
        } else {
            T v[8];
            __builtin_memcpy(v, &e, sizeof(v));
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
                if (8 * q + k < p.cols)
                    row[8 * q + k] = v[k];
        }
    }
}

uint32_t stream_blocks(uint64_t items)
{
    const uint64_t want = (items + kThreads - 1) / kThreads;
    return static_cast<uint32_t>(want < 16384 ? want : 16384);
}

// ---- products
//
// out^T = W x^T on v_mfma_scale_f32_32x32x64_f8f6f4, in the tiles of tile.h:
// W is the first factor, so a lane holds units of one point, of which a swap
// between the halves of a wave makes sixteen in a row.

struct ProductParams {
    const uint8_t *x, *x_packed, *w, *w_packed;
    const float* bias;
    void* out;
    int64_t out_stride;
    uint32_t points, units, steps;
    uint32_t x_row, w_row;           // bytes from row to row of the codes
    int32_t relu;
};

template <int SIDE_>
struct Shape {
    static constexpr int SIDE = SIDE_;
    static constexpr int WN = SIDE == 256 ? 4 : 2;
    static constexpr int WAVES = 2 * WN, THREADS = 64 * WAVES;
    static constexpr int FM = SIDE / 64, FN = SIDE / (32 * WN);    // blocks of units and points of a wave
    static constexpr int ROWS = SIDE * static_cast<int>(kStepBytes);
    static constexpr int BUFFER = 2 * ROWS;
    static constexpr int LOADS = BUFFER / (1024 * WAVES);
    static constexpr int BRINGS = LOADS / 2;                       // of either factor
    static constexpr int BUFFERS = SIDE == 64 ? 4 : 2;
};

template <typename S>
struct Fragments {
    int4v w[S::FM], x[S::FN];
};

// A step's rows of one factor, each lane's pieces from `at` on; pieces past
// `limit` are that one instead.
template <typename S>
__device__ __forceinline__ void bring_rows(const uint8_t* rows, const uint32_t (&at)[S::BRINGS], uint32_t limit,
                                           uint32_t wave, char* to)
{
#pragma unroll
    for (int i = 0; i < S::BRINGS; ++i)
        bring(reinterpret_cast<const char*>(rows) + min(at[i], limit), to + (S::WAVES * i + wave) * 1024);
}

template <int O>
__device__ __forceinline__ float16v multiply(int4v a, int4v b, int scale_a, int scale_b, float16v acc)
{
    const int8v a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const int8v b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a8, b8, acc, 4, 4, O, scale_a, O, scale_b);
}

template <typename S, int O>
__device__ __forceinline__ void multiply_fragments(const Fragments<S>& f, const int (&scale_w)[S::FM],
                                                   const int (&scale_x)[S::FN], float16v (&acc)[S::FM][S::FN])
{
    constexpr int READS = S::FM + S::FN, PRODUCTS = S::FM * S::FN;
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t)
            acc[s][t] = multiply<O>(f.w[s], f.x[t], scale_w[s], scale_x[t], acc[s][t]);
    constexpr int EACH = (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
    for (int k = 0; k < PRODUCTS; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

// Bias and activation of a wave's part, units `unit` on.
template <int FM, int FN>
__device__ __forceinline__ void activate(const float* bias, int32_t relu, uint32_t units, uint32_t unit,
                                         float16v (&acc)[FM][FN])
{
    const uint32_t half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < FM; ++s) {
        // the lane's units of the block
        float b[16];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const uint32_t u = unit + 32 * s + 8 * g + 4 * half;
            if (bias && u + 4 <= units) {
                load_run<float, 4>(bias + u, b + 4 * g);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    b[4 * g + r] = bias ? bias[min(u + r, units - 1)] : 0.0f;
            }
        }
#pragma unroll
        for (int t = 0; t < FN; ++t)
#pragma unroll
            for (int q = 0; q < 16; ++q) {
                const float v = acc[s][t][q] + b[q];
                acc[s][t][q] = relu && v < 0.0f ? 0.0f : v;
            }
    }
}

template <typename S, typename T>
__global__ __launch_bounds__(S::THREADS, 2) void product_kernel(ProductParams p)
{
    BUFFERS_IN_LDS(S)
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t unit_tiles = (p.units + S::SIDE - 1) / S::SIDE;
    const uint32_t tj = blockIdx.x / unit_tiles, ti = blockIdx.x - tj * unit_tiles;
    const uint32_t unit0 = ti * S::SIDE, point0 = tj * S::SIDE;
    const uint8_t* w = p.w + static_cast<uint64_t>(unit0) * p.w_row;
    const uint8_t* x = p.x + static_cast<uint64_t>(point0) * p.x_row;
    // this lane's pieces; rows past the end read the last one, and are not stored
    uint32_t w_at[S::BRINGS], x_at[S::BRINGS];
#pragma unroll
    for (int i = 0; i < S::BRINGS; ++i) {
        const uint32_t row = 8 * (S::WAVES * i + wave) + (lane >> 3), piece = brought_piece(lane, wave) * kSlot;
        w_at[i] = min(row, p.units - 1 - unit0) * p.w_row + piece;
        x_at[i] = min(row, p.points - 1 - point0) * p.x_row + piece;
    }
    // past a row's end a step takes what lies there, the rows' last piece at most:
    // x has zeros there
    const uint64_t w_bytes = static_cast<uint64_t>(p.units - unit0) * p.w_row - kSlot;
    const uint32_t w_limit = static_cast<uint32_t>(min(w_bytes, uint64_t{0xffffffffu}));
    const uint32_t wave_u = (wave & 1) * S::FM, wave_p = (wave >> 1) * S::FN;      // blocks of 32
    const int* w_packed = reinterpret_cast<const int*>(p.w_packed) + static_cast<uint64_t>(unit0 / 32 + wave_u) * p.steps * 64;
    const int* x_packed = reinterpret_cast<const int*>(p.x_packed) + static_cast<uint64_t>(point0 / 32 + wave_p) * p.steps * 64;
    int scale_w[S::BUFFERS][S::FM], scale_x[S::BUFFERS][S::FN];
    float16v acc[S::FM][S::FN];
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t)
            acc[s][t] = float16v{};
    pipeline<S::LOADS, Fragments<S>>(
        p.steps, buffers,
        [&](uint32_t k, int in_round) {
#pragma unroll
            for (int s = 0; s < S::FM; ++s)
                scale_w[in_round][s] = (w_packed + (s * p.steps + k) * 64)[lane];
#pragma unroll
            for (int t = 0; t < S::FN; ++t)
                scale_x[in_round][t] = (x_packed + (t * p.steps + k) * 64)[lane];
        },
        [&](uint32_t k, char* buffer) {
            const uint32_t on = k * kStepBytes;
            bring_rows<S>(w + on, w_at, w_limit - on, wave, buffer);
            bring_rows<S>(x + on, x_at, 0xffffffffu, wave, buffer + S::ROWS);
            // the loads stay ahead of the products that hide them
            __builtin_amdgcn_sched_barrier(0);
        },
        [&](Fragments<S>& f, const char* buffer, uint32_t o) {
            const char* from_w = buffer + wave_u * kBlockBytes + piece_at(lane, o);
            const char* from_x = buffer + S::ROWS + wave_p * kBlockBytes + piece_at(lane, o);
#pragma unroll
            for (int s = 0; s < S::FM; ++s)
                f.w[s] = *reinterpret_cast<const int4v*>(from_w + s * kBlockBytes);
#pragma unroll
            for (int t = 0; t < S::FN; ++t)
                f.x[t] = *reinterpret_cast<const int4v*>(from_x + t * kBlockBytes);
        },
        [&](const Fragments<S>& f, int depth) {
            const int k = depth >> 2;
            switch (depth & 3) {
            case 0: multiply_fragments<S, 0>(f, scale_w[k], scale_x[k], acc); break;
            case 1: multiply_fragments<S, 1>(f, scale_w[k], scale_x[k], acc); break;
            case 2: multiply_fragments<S, 2>(f, scale_w[k], scale_x[k], acc); break;
            default: multiply_fragments<S, 3>(f, scale_w[k], scale_x[k], acc); break;
            }
        });
    const uint32_t unit = unit0 + 32 * wave_u, point = point0 + 32 * wave_p;
    activate(p.bias, p.relu, p.units, unit, acc);
    columns_out<T>(acc, own_part<S::FM, S::BUFFER>(buffers[0], buffers[1], wave), from_f32<T>,
                   [&](uint32_t q, uint32_t u, const uint4& run) {
                       if (point + q < p.points)
                           store_inside(static_cast<T*>(p.out) + (point + q) * p.out_stride + unit + u,
                                        static_cast<int64_t>(p.units) - unit - u, run);
                   });
}

// ---- layers of up to 256 units and 8 to 512 inputs
//
// All weights fit LDS beside the blocks of 128 points, so the points' blocks
// need not go through memory: a workgroup loads its points, puts them into
// blocks in LDS, multiplies and stores; 8 waves, of 128 units and 32 points
// each.  Workgroups on a CU fill each other's waits (one that went through
// many tiles with its weights kept lost more to spilled addresses).

constexpr uint32_t kLayerUnits = 256, kLayerPoints = 128;
constexpr int kLayerThreads = 512;

struct LayerParams {
    const uint8_t *w, *w_scales;
    const void* x;
    const float* bias;
    void* out;
    int64_t x_stride, out_stride;
    uint32_t points, units, cols, blocks;
    int32_t relu;
};

template <typename X, typename T, int STEPS>
__global__ __launch_bounds__(kLayerThreads) void layer_kernel(LayerParams p)
{
    constexpr uint32_t W_STEP = kLayerUnits * kStepBytes, X_STEP = kLayerPoints * kStepBytes;
    constexpr int FM = 4, PARTS = sizeof(T) == 4 ? 4 : 2;         // blocks of units; parts of them that leave together
    constexpr uint32_t OWN = 32 * 128;                            // a wave's bytes on the way out: a line of 32 points
    constexpr int EIGHTHS = 8 * STEPS;                            // of blocks, a thread
    __shared__ __align__(16) char w[STEPS * W_STEP];
    __shared__ __align__(16) char x[STEPS * X_STEP > 8 * OWN ? STEPS * X_STEP : 8 * OWN];
    __shared__ __align__(4) uint8_t w_packed[STEPS * kLayerUnits * 8];
    __shared__ __align__(4) uint8_t x_packed[STEPS * kLayerPoints * 8];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // the weights, as the tiles bring them
    const uint32_t row_bytes = 16 * p.blocks, limit = p.units * row_bytes - kSlot;
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
#pragma unroll
        for (uint32_t i = 0; i < kLayerUnits / 64; ++i) {
            const uint32_t row = 8 * (8 * i + wave) + (lane >> 3);
            const uint32_t at = min(row, p.units - 1) * row_bytes + brought_piece(lane, wave) * kSlot + k * kStepBytes;
            bring(reinterpret_cast<const char*>(p.w) + min(at, limit), w + k * W_STEP + (8 * i + wave) * 1024);
        }
    for (uint32_t i = tid; i < kLayerUnits * 8 * STEPS; i += kLayerThreads) {
        const uint32_t row = i / (8 * STEPS), block = i % (8 * STEPS);
        w_packed[packed_at(row, block, STEPS)]
            = row < p.units && block < p.blocks ? p.w_scales[row * p.blocks + block] : static_cast<uint8_t>(kOne);
    }

    // eighth e of the blocks: eight elements of point e / (32 STEPS)
    const uint32_t first = blockIdx.x * kLayerPoints;
    Eight<X> raw[EIGHTHS];
#pragma unroll
    for (int i = 0; i < EIGHTHS; ++i) {
        const uint32_t e = tid + kLayerThreads * i, q = e % (32 * STEPS);
        const uint32_t point = min(first + e / (32 * STEPS), p.points - 1);
        // past the row's last eight elements, those
        raw[i] = *reinterpret_cast<const Eight<X>*>(static_cast<const X*>(p.x) + point * p.x_stride
                                                     + min(8 * q, p.cols - 8));
    }
#pragma unroll
    for (int i = 0; i < EIGHTHS; ++i) {
        const uint32_t e = tid + kLayerThreads * i, q = e % (32 * STEPS), row = e / (32 * STEPS), block = q >> 2;
        if (p.cols < 256 * STEPS) {
            // what was read lies `early` before the eighth
            const uint32_t early = 8 * q - min(8 * q, p.cols - 8);
            X v[8];
            __builtin_memcpy(v, &raw[i], sizeof(v));
            if (p.cols & 7) {
#pragma unroll
                for (uint32_t b = 4; b; b /= 2)
#pragma unroll
                    for (uint32_t k = 0; k < 8; ++k)
                        v[k] = early & b ? (k + b < 8 ? v[k + b] : from_f32<X>(0.0f)) : v[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k)
                v[k] = early < 8 ? v[k] : from_f32<X>(0.0f);
            __builtin_memcpy(&raw[i], v, sizeof(v));
        }
        const uint32_t byte = block < p.blocks ? shared_scale<X>(raw[i]) : kOne;
        *reinterpret_cast<uint32_t*>(x + (block >> 3) * X_STEP + row * kStepBytes
                                     + ((block & 7) ^ (row >> 1 & 7)) * kSlot + (q & 3) * 4) = encode<X>(raw[i], byte);
        if ((q & 3) == 0)
            x_packed[packed_at(row, block, STEPS)] = static_cast<uint8_t>(byte);
    }
    landed<0>();
    const uint32_t wave_u = (wave & 1) * FM, wave_p = wave >> 1;          // blocks of 32
    float16v acc[FM][1];
#pragma unroll
    for (int s = 0; s < FM; ++s)
        acc[s][0] = float16v{};
#pragma unroll
    for (int k = 0; k < STEPS; ++k) {
        int scale_w[FM];
#pragma unroll
        for (int s = 0; s < FM; ++s)
            scale_w[s] = reinterpret_cast<const int*>(w_packed)[((wave_u + s) * STEPS + k) * 64 + lane];
        const int scale_x = reinterpret_cast<const int*>(x_packed)[(wave_p * STEPS + k) * 64 + lane];
        const char* from_w = w + k * W_STEP + wave_u * kBlockBytes;
        const char* from_x = x + k * X_STEP + wave_p * kBlockBytes;
        auto depth = [&](auto o) {
            constexpr int O = decltype(o)::value;
            const int4v b = *reinterpret_cast<const int4v*>(from_x + piece_at(lane, O));
#pragma unroll
            for (int s = 0; s < FM; ++s)
                acc[s][0] = multiply<O>(*reinterpret_cast<const int4v*>(from_w + s * kBlockBytes + piece_at(lane, O)), b,
                                        scale_w[s], scale_x, acc[s][0]);
        };
        depth(std::integral_constant<int, 0>());
        depth(std::integral_constant<int, 1>());
        depth(std::integral_constant<int, 2>());
        depth(std::integral_constant<int, 3>());
    }
    __syncthreads();          // the blocks of the points make room for what leaves
    const uint32_t unit = 32 * wave_u, point = first + 32 * wave_p;
    activate(p.bias, p.relu, p.units, unit, acc);
    auto emit = [&](uint32_t q, uint32_t u, const uint4& run) {
        if (point + q < p.points)
            store_inside(static_cast<T*>(p.out) + (point + q) * p.out_stride + unit + u,
                         static_cast<int64_t>(p.units) - unit - u, run);
    };
    char* own = x + wave * OWN;
    if constexpr (PARTS == 2) {
        columns_out_of<T, 0, 2>(acc, own, from_f32<T>, emit);
        columns_out_of<T, 2, 2>(acc, own, from_f32<T>, emit);
    } else {
        columns_out_of<T, 0, 1>(acc, own, from_f32<T>, emit);
        columns_out_of<T, 1, 1>(acc, own, from_f32<T>, emit);
        columns_out_of<T, 2, 1>(acc, own, from_f32<T>, emit);
        columns_out_of<T, 3, 1>(acc, own, from_f32<T>, emit);
    }
}

template <typename X, typename T>
void launch_layer_steps(const LayerParams& p, hipStream_t stream)
{
    const uint32_t grid = (p.points + kLayerPoints - 1) / kLayerPoints;
    if (p.blocks <= 8)
        layer_kernel<X, T, 1><<<grid, kLayerThreads, 0, stream>>>(p);
    else
        layer_kernel<X, T, 2><<<grid, kLayerThreads, 0, stream>>>(p);
}

template <typename X>
hipError_t launch_layer(const sqn_matrix& x, const sqn_quantised& w, const float* bias, bool relu, const sqn_matrix& out,
                        hipStream_t stream)
{
    LayerParams p;
    p.w = static_cast<const uint8_t*>(w.codes);
    p.w_scales = static_cast<const uint8_t*>(w.scales);
    p.x = x.data;
    p.bias = bias;
    p.out = out.data;
    p.x_stride = x.row_stride;
    p.out_stride = out.row_stride;
    p.points = static_cast<uint32_t>(x.rows);
    p.units = static_cast<uint32_t>(w.rows);
    p.cols = static_cast<uint32_t>(x.cols);
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.relu = relu ? 1 : 0;
    if (out.dtype == SQN_F32)
        launch_layer_steps<X, float>(p, stream);
    else if (out.dtype == SQN_F16)
        launch_layer_steps<X, _Float16>(p, stream);
    else
        launch_layer_steps<X, __bf16>(p, stream);
    return hipGetLastError();
}

// All 256 units are multiplied, fewer as copies of the last.  (A call so and in
// tiles, us: 65,536 points of 256 elements by 256 units 23.7 and 23.6, by 128 22.6
// and 23.5, by 3 19.5 and 23.8; 1000 points 10 and 15; 2^20 points of 256 by 256 300
// and 330, of 32 by 3 286 and 260.)
bool is_layer(int64_t units, int64_t cols) { return units <= kLayerUnits && cols >= 8 && quant_blocks(cols) <= 16; }

// ---- products of few points
//
// For few points (one token's activations among them) the weights' bytes are
// all that takes time, and a launch of its own for the activations' blocks
// would take longer than the product.  A workgroup computes 16 units of all
// points, or 32 or 64 where there are many units, on
// v_mfma_scale_f32_16x16x128_f8f6f4; its waves share the sum and add up in LDS,
// in the order of the waves.  Every wave puts the points' elements of its
// stretch into blocks by itself, which costs it more instructions than its
// products: hence more units a workgroup (one point of 8192 by 8192 units 12.9
// us a call, 18.1 with 16), and tiles for many elements (16 points of 16384
// binary32 by 4096 units 24 us, 39 here; of 4096 binary16 14.0 and 10.2).

constexpr uint32_t kFew = 16;
bool is_few(int64_t points, int64_t cols) { return points <= 4 || (points <= kFew && points * cols <= 65536); }
// Steps whose weights are under way together: as many as the registers take.
template <typename T, int UNITS>
constexpr int kFewAhead = sizeof(T) == 4 || UNITS == 4 ? 1 : 2;
constexpr int kFewMaxWaves = 16;
constexpr uint32_t kFewGroups = 256;    // of 16 units: a workgroup takes more where there are more

struct FewParams {
    const uint8_t *w, *w_scales;
    const void* x;                   // rows of elements, or codes
    const uint8_t* x_scales;         // of codes
    const float* bias;
    void* out;
    int64_t x_stride, out_stride;    // elements
    uint32_t points, units, cols, blocks;
    uint32_t steps;                  // of four blocks, per wave
    int32_t relu, dtype;
};

// the type of x where it is in blocks already
struct Blocks {};

struct Operand {
    int4v codes;
    int scale;
};

// The loads of a block are the same for every lane, from a place inside the
// row where it has none, so that all of a wave's are under way together; zeros
// of scale 1 take the place of what is not there.

__device__ __forceinline__ Operand load_block(const uint8_t* codes, const uint8_t* scales, uint32_t row, uint32_t block,
                                              uint32_t blocks, bool there)
{
    const uint64_t at = static_cast<uint64_t>(row) * blocks + min(block, blocks - 1);
    Operand o;
    o.codes = *reinterpret_cast<const int4v*>(codes + 16 * at);
    o.scale = scales[at];
    if (!there || block >= blocks)
        o = Operand{int4v{0, 0, 0, 0}, static_cast<int>(kOne)};
    return o;
}

// A block of a row of elements as it lies in memory.
template <typename T>
struct Elements {
    Eight<T> part[4];
};

template <typename T>
__device__ __forceinline__ Elements<T> load_elements(const T* row, uint32_t block, uint32_t cols)
{
    Elements<T> e;
    if (cols >= 32) {
        const T* from = row + min(32 * block, cols - 32);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            e.part[q] = *reinterpret_cast<const Eight<T>*>(from + 8 * q);
    }
    return e;
}

template <typename T>
__device__ __forceinline__ Operand encode_block(Elements<T> e, const T* row, uint32_t block, uint32_t cols, bool there)
{
    if (!there) {
        e = Elements<T>{};
    } else if (32 * block + 32 > cols) {        // a row's last block, or none
#pragma unroll
        for (int q = 0; q < 4; ++q)
            e.part[q] = load_eight<T>(row, 32 * block + 8 * q, cols);
    }
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        top = max(top, top_of<T>(e.part[q]));
    Operand o;
    o.scale = static_cast<int>(byte_of<T>(top));
#pragma unroll
    for (int q = 0; q < 4; ++q)
        o.codes[q] = static_cast<int>(encode<T>(e.part[q], o.scale));
    return o;
}

template <typename T, int UNITS>
__global__ __launch_bounds__(64 * kFewMaxWaves) void few_kernel(FewParams p)
{
    constexpr int AHEAD = kFewAhead<T, UNITS>;
    __shared__ float4v sums[kFewMaxWaves][UNITS][64];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const uint32_t row = lane & 15;
    uint32_t unit[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
        unit[u] = min((blockIdx.x * UNITS + u) * 16 + row, p.units - 1);
    const bool there = row < p.points;
    const uint32_t first = wave * p.steps, last = min(first + p.steps, (p.blocks + 3) / 4);
    float4v acc[UNITS];
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
        acc[u] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t k = first; k < last; k += AHEAD) {
        Operand w[AHEAD][UNITS], x[AHEAD];
        Elements<std::conditional_t<std::is_same<T, Blocks>::value, float, T>> e[AHEAD];
        const T* row_x = nullptr;
        if constexpr (!std::is_same<T, Blocks>::value)
            row_x = static_cast<const T*>(p.x) + (there ? row : 0) * p.x_stride;
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            const uint32_t block = 4 * (k + a) + (lane >> 4);
#pragma unroll
            for (int u = 0; u < UNITS; ++u)
                w[a][u] = load_block(p.w, p.w_scales, unit[u], block, p.blocks, k + a < last);
            if constexpr (std::is_same<T, Blocks>::value)
                x[a] = load_block(static_cast<const uint8_t*>(p.x), p.x_scales, there ? row : 0, block, p.blocks,
                                  there && k + a < last);
            else
                e[a] = load_elements(row_x, block, p.cols);
        }
#pragma unroll
        for (int a = 0; a < AHEAD; ++a) {
            if constexpr (!std::is_same<T, Blocks>::value)
                x[a] = encode_block(e[a], row_x, 4 * (k + a) + (lane >> 4), p.cols, there && k + a < last);
            const int8v x8 = __builtin_shufflevector(x[a].codes, x[a].codes, 0, 1, 2, 3, -1, -1, -1, -1);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const int4v c = w[a][u].codes;
                const int8v w8 = __builtin_shufflevector(c, c, 0, 1, 2, 3, -1, -1, -1, -1);
                acc[u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w8, x8, acc[u], 4, 4, 0, w[a][u].scale, 0,
                                                                          x[a].scale);
            }
        }
    }
#pragma unroll
    for (int u = 0; u < UNITS; ++u)
        sums[wave][u][lane] = acc[u];
    __syncthreads();
    // a wave for each 16 units, or one after another where there are fewer
    for (uint32_t g = wave; g < UNITS; g += waves) {
        float4v sum = sums[0][g][lane];
        for (uint32_t k = 1; k < waves; ++k)
            sum += sums[k][g][lane];
        // element q: unit 4 (lane / 16) + q of point lane % 16
        if (!there)
            continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t u = (blockIdx.x * UNITS + g) * 16 + 4 * (lane >> 4) + q;
            if (u >= p.units)
                break;
            float v = sum[q];
            if (p.bias)
                v += p.bias[u];
            if (p.relu)
                v = v < 0.0f ? 0.0f : v;
            const int64_t at = row * p.out_stride + u;
            if (p.dtype == SQN_F32)
                static_cast<float*>(p.out)[at] = v;
            else if (p.dtype == SQN_F16)
                static_cast<_Float16*>(p.out)[at] = static_cast<_Float16>(v);
            else
                static_cast<__bf16*>(p.out)[at] = static_cast<__bf16>(v);
        }
    }
}

template <typename T>
hipError_t launch_few(const void* x, const uint8_t* x_scales, int64_t x_stride, int64_t points, const sqn_quantised& w,
                      const float* bias, bool relu, const sqn_matrix& out, hipStream_t stream)
{
    FewParams p;
    p.w = static_cast<const uint8_t*>(w.codes);
    p.w_scales = static_cast<const uint8_t*>(w.scales);
    p.x = x;
    p.x_scales = x_scales;
    p.bias = bias;
    p.out = out.data;
    p.x_stride = x_stride;
    p.out_stride = out.row_stride;
    p.points = static_cast<uint32_t>(points);
    p.units = static_cast<uint32_t>(w.rows);
    p.cols = static_cast<uint32_t>(w.cols);
    p.blocks = static_cast<uint32_t>(quant_blocks(w.cols));
    p.relu = relu ? 1 : 0;
    p.dtype = out.dtype;
    const uint32_t groups = (p.units + 15) / 16, steps = (p.blocks + 3) / 4;
    const uint32_t each = groups >= 4 * kFewGroups ? 4 : groups >= 2 * kFewGroups ? 2 : 1;
    const uint32_t grid = (groups + each - 1) / each;
    // a wave takes a batch of steps or more, unless that leaves CUs with little
    uint32_t waves = 1;
    while (waves < kFewMaxWaves && waves < steps && (grid * waves < 2048 || steps > 2 * waves))
        waves *= 2;
    p.steps = (steps + waves - 1) / waves;
    if (each == 4)
        few_kernel<T, 4><<<grid, 64 * waves, 0, stream>>>(p);
    else if (each == 2)
        few_kernel<T, 2><<<grid, 64 * waves, 0, stream>>>(p);
    else
        few_kernel<T, 1><<<grid, 64 * waves, 0, stream>>>(p);
    return hipGetLastError();
}

// Scratch of a product in tiles: the packed scales of its factors, rows up to
// whole tiles, and the codes of x with rows of whole steps.
struct ProductScratch {
    PackedScales x_packed, w_packed;
    uint8_t* x_codes;
    size_t bytes;

    ProductScratch(int64_t points, int64_t units, int64_t cols, void* base)
    {
        const uint32_t steps = steps_of(static_cast<uint32_t>(quant_blocks(cols)));
        auto size = [&](int64_t rows) { return static_cast<size_t>((rows + 255) / 256) * 8 * steps * 256; };
        x_packed.to = static_cast<uint8_t*>(base);
        w_packed.to = x_packed.to + size(points);
        x_codes = w_packed.to + size(units);
        x_packed.steps = w_packed.steps = steps;
        bytes = size(points) + size(units) + static_cast<size_t>(points) * steps * kStepBytes;
    }
};

PackParams pack_of(const sqn_quantised& x, const PackedScales& packed)
{
    PackParams p;
    p.from = static_cast<const uint8_t*>(x.scales);
    p.packed = packed;
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.words = static_cast<uint64_t>(x.rows) * packed.steps * 2;
    p.codes = nullptr;
    p.codes_to = nullptr;
    return p;
}

QuantParams quant_of(const sqn_matrix& x, const sqn_quantised& q)
{
    QuantParams p;
    p.x = x.data;
    p.values = nullptr;
    p.codes = static_cast<uint8_t*>(q.codes);
    p.scales = static_cast<uint8_t*>(q.scales);
    p.stride = x.row_stride;
    p.cols = static_cast<uint32_t>(x.cols);
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.items = static_cast<uint64_t>(x.rows) * p.blocks * 4;
    return p;
}

template <typename S>
void launch_shape(const ProductParams& p, int32_t dtype, hipStream_t stream)
{
    const uint32_t grid = (p.points + S::SIDE - 1) / S::SIDE * ((p.units + S::SIDE - 1) / S::SIDE);
    if (dtype == SQN_F32)
        product_kernel<S, float><<<grid, S::THREADS, 0, stream>>>(p);
    else if (dtype == SQN_F16)
        product_kernel<S, _Float16><<<grid, S::THREADS, 0, stream>>>(p);
    else
        product_kernel<S, __bf16><<<grid, S::THREADS, 0, stream>>>(p);
}

// The codes of x in rows of whole steps.
hipError_t launch_tiles(const void* x_codes, int64_t points, const ProductScratch& t, const sqn_quantised& w,
                        const float* bias, bool relu, const sqn_matrix& out, hipStream_t stream)
{
    ProductParams p;
    p.x = static_cast<const uint8_t*>(x_codes);
    p.x_packed = t.x_packed.to;
    p.w = static_cast<const uint8_t*>(w.codes);
    p.w_packed = t.w_packed.to;
    p.bias = bias;
    p.out = out.data;
    p.out_stride = out.row_stride;
    p.points = static_cast<uint32_t>(points);
    p.units = static_cast<uint32_t>(w.rows);
    p.steps = t.x_packed.steps;
    p.x_row = p.steps * kStepBytes;
    p.w_row = static_cast<uint32_t>(16 * quant_blocks(w.cols));
    p.relu = relu ? 1 : 0;
    auto tiles = [&](int64_t side) { return ((p.points + side - 1) / side) * ((p.units + side - 1) / side); };
    if (tiles(256) >= 200)
        launch_shape<Shape<256>>(p, out.dtype, stream);
    else if (tiles(128) >= 200)
        launch_shape<Shape<128>>(p, out.dtype, stream);
    else
        launch_shape<Shape<64>>(p, out.dtype, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantise(const sqn_matrix& x, const sqn_quantised& out, hipStream_t stream)
{
    const QuantParams p = quant_of(x, out);
    const uint32_t grid = stream_blocks(p.items);
    if (x.dtype == SQN_F32)
        quantise_kernel<float><<<grid, kThreads, 0, stream>>>(p);
    else if (x.dtype == SQN_F16)
        quantise_kernel<_Float16><<<grid, kThreads, 0, stream>>>(p);
    else
        quantise_kernel<__bf16><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_quantised_values(const sqn_quantised& x, const sqn_matrix& out, hipStream_t stream)
{
    QuantParams p;
    p.x = nullptr;
    p.values = out.data;
    p.codes = static_cast<uint8_t*>(x.codes);
    p.scales = static_cast<uint8_t*>(x.scales);
    p.stride = out.row_stride;
    p.cols = static_cast<uint32_t>(x.cols);
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.items = static_cast<uint64_t>(x.rows) * p.blocks * 4;
    const uint32_t grid = stream_blocks(p.items);
    if (out.dtype == SQN_F32)
        values_kernel<float><<<grid, kThreads, 0, stream>>>(p);
    else if (out.dtype == SQN_F16)
        values_kernel<_Float16><<<grid, kThreads, 0, stream>>>(p);
    else
        values_kernel<__bf16><<<grid, kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_quantised_product(const sqn_quantised& x, const sqn_quantised& w, const float* bias, bool relu,
                                    const sqn_matrix& out, void* workspace, hipStream_t stream)
{
    if (is_few(x.rows, x.cols))
        return launch_few<Blocks>(x.codes, static_cast<const uint8_t*>(x.scales), 0, x.rows, w, bias, relu, out, stream);
    const ProductScratch t(x.rows, w.rows, x.cols, workspace);
    const PackParams pw = pack_of(w, t.w_packed);
    PackParams px = pack_of(x, t.x_packed);
    const void* codes = x.codes;
    if (px.blocks % 8 != 0) {
        px.codes = static_cast<const uint4*>(x.codes);
        px.codes_to = reinterpret_cast<uint4*>(t.x_codes);
        codes = t.x_codes;
    }
    const uint32_t groups_w = stream_blocks(pw.words), groups_x = stream_blocks(px.words);
    pack_kernel<<<groups_w + groups_x, kThreads, 0, stream>>>(pw, px, groups_w);
    return launch_tiles(codes, x.rows, t, w, bias, relu, out, stream);
}

size_t quantised_product_bytes(int64_t points, int64_t units, int64_t cols)
{
    return is_few(points, cols) ? 0 : ProductScratch(points, units, cols, nullptr).bytes;
}

size_t quantised_layer_bytes(int64_t points, int64_t units, int64_t cols)
{
    return is_layer(units, cols) ? 0 : quantised_product_bytes(points, units, cols);
}

hipError_t launch_quantised_layer(const sqn_matrix& x, const sqn_quantised& w, const float* bias, bool relu,
                                  const sqn_matrix& out, void* workspace, hipStream_t stream)
{
    if (is_few(x.rows, x.cols)) {
        if (x.dtype == SQN_F32)
            return launch_few<float>(x.data, nullptr, x.row_stride, x.rows, w, bias, relu, out, stream);
        if (x.dtype == SQN_F16)
            return launch_few<_Float16>(x.data, nullptr, x.row_stride, x.rows, w, bias, relu, out, stream);
        return launch_few<__bf16>(x.data, nullptr, x.row_stride, x.rows, w, bias, relu, out, stream);
    }
    if (is_layer(w.rows, w.cols)) {
        if (x.dtype == SQN_F32)
            return launch_layer<float>(x, w, bias, relu, out, stream);
        if (x.dtype == SQN_F16)
            return launch_layer<_Float16>(x, w, bias, relu, out, stream);
        return launch_layer<__bf16>(x, w, bias, relu, out, stream);
    }
    const ProductScratch t(x.rows, w.rows, x.cols, workspace);
    sqn_quantised q;
    q.rows = x.rows;
    q.cols = x.cols;
    q.codes = t.x_codes;
    q.scales = nullptr;
    QuantParams p = quant_of(x, q);
    p.items = static_cast<uint64_t>(x.rows) * t.x_packed.steps * 32;
    const PackParams pw = pack_of(w, t.w_packed);
    const uint32_t groups = stream_blocks(p.items), grid = groups + stream_blocks(pw.words);
    if (x.dtype == SQN_F32)
        quantise_packed_kernel<float><<<grid, kThreads, 0, stream>>>(p, t.x_packed, pw, groups);
    else if (x.dtype == SQN_F16)
        quantise_packed_kernel<_Float16><<<grid, kThreads, 0, stream>>>(p, t.x_packed, pw, groups);
    else
        quantise_packed_kernel<__bf16><<<grid, kThreads, 0, stream>>>(p, t.x_packed, pw, groups);
    return launch_tiles(t.x_codes, x.rows, t, w, bias, relu, out, stream);
}

}  // namespace sqn
