// Update matrices orthogonalised by Newton-Schulz products.
//
//   X <- G / (||G||_F + eps);  `steps` times:  A = X X^T,
//   X <- a X + (b A + c A A) X
//
// X is held with its shorter side as rows (m <= n), so the square products
// are m x m.  All products are of the form C = P Q^T with rows of P and Q
// contiguous along the sum, on v_mfma_f32_32x32x16_f16:
//
//   A   = X X^T      P = Q = X            only the tiles on and below the
//   A A = A A^T      P = Q = A            diagonal, mirrored when written
//   B X = B (X^T)^T  P = B, Q = X^T       X^T is kept beside X
//
// Rounding.  binary16 factors, scaled by powers of two into its range
// (|X| <= 2, |A| <= 4, |B| <= 16 by the check of the coefficients).  Two
// things would otherwise cost most of the result's digits.  The diagonals of A
// and B = b A + c A A are near 1 and -2.7 while the rest is near 0: they are
// kept in binary32 and applied in the epilogues, (A A)_ij = (O O)_ij +
// (d_i + d_j) O_ij + [i = j] d_i^2 with O = A - diag(d) (the error of a
// 256 x 256 update falls from 1.7e-3 to 7.5e-4 of its norm).  And updates of low
// rank have singular values that one rounding of X would bury: X is kept as
// hi + lo, two binary16, and a X takes both.  What is left is less than the
// rounding of a bfloat16 result (1.7e-3).  For binary16 and binary32 results
// every factor is hi + lo, a product sums hi hi + hi lo + lo hi (4e-7), and
// X is kept in binary32 beside its factors: what an element of it loses in a
// step is a change in every direction, and comes back as large as those of the
// smallest singular values (8e-6 instead of 3e-6 in a rank of 8 with noise).
#include <math.h>

#include "learn.h"
#include "numeric.h"
#include "sqn_internal.h"
#include "tile.h"

namespace sqn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kNormBlocks = 256;         // workgroups per matrix that sum squares

constexpr float kScaleX = 4096.0f;       // hi + lo = 2^12 X
constexpr float kScaleA = 4096.0f;       // 2^12 O
constexpr float kScaleB = 2048.0f;       // 2^11 (b A + c A A) off the diagonal

// One matrix's scratch; the matrices of a batch follow each other.
struct Scratch {
    _Float16 *x, *x_lo;                  // [mp][np]; x_lo where factors are split
    _Float16 *xt, *xt_to;                // [np][mp], read and written by a step
    _Float16 *xt_lo, *xt_to_lo;          // the same where factors are split, one and the same otherwise
    float* xt_full;                      // [np][mp], where factors are split
    _Float16 *o, *o_lo;                  // [mp][mp]
    _Float16 *b, *b_lo;                  // [mp][mp]
    float *d, *d_b;                      // [mp] diagonals of A, and of a + b A + c A A
    double* norms;                       // [kNormBlocks]
};

struct OrthParams {
    Scratch s;
    const void* in;
    void* out;
    int64_t in_batch, in_row, in_col;    // elements, of X (rows <= cols)
    int64_t out_batch, out_row, out_col;
    int32_t m, n, mp, np;                // mp, np: rows and columns of the scratch
    uint32_t steps_m, steps_n;           // of sums over m and n
    int32_t out_dtype;
    float a, b, c, eps;
};

__device__ __forceinline__ void store_any(void* p, int64_t i, float v, int32_t dtype)
{
    if (dtype == SQN_F32)
        static_cast<float*>(p)[i] = v;
    else if (dtype == SQN_F16)
        static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v);
    else
        static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v);
}

// Whether X's rows run along the larger stride of the matrix, so that loads go
// down a column.
__device__ __forceinline__ bool down(const OrthParams& p) { return p.in_row < p.in_col; }

// V elements from (i, j) on along the smaller stride, zeros past the matrix.
template <typename T, int V>
__device__ __forceinline__ void load_line(const OrthParams& p, int64_t base, uint32_t i, uint32_t j, float v[V])
{
    const bool d = down(p);
    const uint32_t at = d ? i : j, end = d ? p.m : p.n, across = d ? j : i, lines = d ? p.n : p.m;
    const int64_t step = d ? p.in_row : p.in_col;
    const T* from = static_cast<const T*>(p.in) + base + i * p.in_row + j * p.in_col;
    if (across < lines && at + V <= end && step == 1) {
        load_run<T, V>(from, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] = across < lines && at + k < end ? to_f32(from[k * step]) : 0.0f;
    }
}

// A matrix's sum of squares in kNormBlocks parts, in binary64: gradients may be
// so small that their squares vanish in binary32.  Its lines along the smaller
// stride go to the workgroups in turn, one line or, of short lines, several
// to a workgroup at a time.
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_kernel(OrthParams p)
{
    constexpr int V = 16 / sizeof(T);
    const int64_t base = blockIdx.y * p.in_batch;
    const bool d = down(p);
    const uint32_t inner = d ? p.m : p.n, outer = d ? p.n : p.m;
    // threads along a line: a power of two
    uint32_t along = 8;
    while (along < kThreads && along * V < inner)
        along *= 2;
    const uint32_t lines = kThreads / along;
    double sum = 0.0;
    for (uint32_t line = blockIdx.x * lines + threadIdx.x / along; line < outer; line += kNormBlocks * lines)
        for (uint32_t at = threadIdx.x % along * V; at < inner; at += 2 * along * V) {
            float v[2][V];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                load_line<T, V>(p, base, d ? at + k * along * V : line, d ? line : at + k * along * V, v[k]);
#pragma unroll
            for (int k = 0; k < 2 * V; ++k) {
                const double x = v[k / V][k % V];
                sum = __builtin_fma(x, x, sum);
            }
        }
    for (int s = 32; s; s /= 2)
        sum += __shfl_xor(sum, s);
    __shared__ double part[kThreads / 64];
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x / 64] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        p.s.norms[blockIdx.y * kNormBlocks + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo)
{
    hi = static_cast<_Float16>(v);
    lo = static_cast<_Float16>(v - static_cast<float>(hi));
}

// X and X^T of 64 x 64 elements a workgroup, zeros past m and n; moved in runs
// of eight elements, turned in LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void start_kernel(OrthParams p)
{
    __shared__ float tile[64][65];
    const uint32_t b = blockIdx.z;
    double sum = 0.0;
    for (int k = threadIdx.x & 63; k < kNormBlocks; k += 64)
        sum += p.s.norms[b * kNormBlocks + k];
    for (int s = 32; s; s /= 2)
        sum += __shfl_xor(sum, s);
    const double norm = sqrt(sum) + static_cast<double>(p.eps);
    const double scale = norm > 0.0 ? kScaleX / norm : 0.0;
    // a NaN or an infinity anywhere gives NaN everywhere
    const float nan = isfinite(norm) ? 0.0f : __builtin_nanf("");
    const uint32_t i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const bool d = down(p);
#pragma unroll
    for (uint32_t k = threadIdx.x; k < 512; k += kThreads) {
        const uint32_t line = k >> 3, at = 8 * (k & 7);
        float v[8];
        load_line<T, 8>(p, b * p.in_batch, i0 + (d ? at : line), j0 + (d ? line : at), v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            tile[d ? at + e : line][d ? line : at + e] = static_cast<float>(v[e] * scale) + nan;
    }
    __syncthreads();
    const uint64_t base = static_cast<uint64_t>(b) * p.mp * p.np;
#pragma unroll
    for (uint32_t k = threadIdx.x; k < 512; k += kThreads) {
        const uint32_t line = k >> 3, at = 8 * (k & 7);
        half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(tile[line][at + e], h, l);
            hi[e] = h;
            lo[e] = l;
        }
        const uint64_t x = base + static_cast<uint64_t>(i0 + line) * p.np + j0 + at;
        *reinterpret_cast<half8*>(p.s.x + x) = hi;
        if (p.s.x_lo)
            *reinterpret_cast<half8*>(p.s.x_lo + x) = lo;
        const uint64_t xt = base + static_cast<uint64_t>(j0 + line) * p.mp + i0 + at;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(tile[at + e][line], h, l);
            hi[e] = h;
            lo[e] = l;
            if (p.s.xt_full)
                p.s.xt_full[xt + e] = tile[at + e][line];
        }
        *reinterpret_cast<half8*>(p.s.xt + xt) = hi;
        *reinterpret_cast<half8*>(p.s.xt_lo + xt) = lo;
    }
}

// no steps: X itself
__global__ __launch_bounds__(kThreads) void emit_kernel(OrthParams p)
{
    const uint32_t b = blockIdx.z, i = blockIdx.y;
    for (uint32_t j = threadIdx.x; j < static_cast<uint32_t>(p.n); j += kThreads) {
        const uint64_t xt = (static_cast<uint64_t>(b) * p.np + j) * p.mp + i;
        const float v = p.s.xt_full ? p.s.xt_full[xt] : static_cast<float>(p.s.xt[xt]) + static_cast<float>(p.s.xt_lo[xt]);
        store_any(p.out, b * p.out_batch + i * p.out_row + j * p.out_col, v * (1.0f / kScaleX), p.out_dtype);
    }
}

// ---- products

// A workgroup's tile: SIDE x SIDE of C by 2 x WN waves; padded sizes are
// multiples of it.  Larger tiles read less of their factors per product
// (from LDS above all); smaller ones give small matrices more workgroups.
template <int SIDE_, bool SPLIT_>
struct Shape {
    static constexpr int SIDE = SIDE_;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int WN = SIDE == 256 ? 4 : 2;
    static constexpr int WAVES = 2 * WN, THREADS = 64 * WAVES;
    static constexpr int FM = SIDE / 64, FN = SIDE / (32 * WN);   // accumulators of a wave
    static constexpr int FACTORS = SPLIT ? 4 : 2;             // P, Q, and their low parts
    static constexpr int ROWS = SIDE * static_cast<int>(kStepBytes);
    static constexpr int BUFFER = FACTORS * ROWS;
    static constexpr int LOADS = BUFFER / (1024 * WAVES);     // of a wave, a step
    static constexpr int BUFFERS = SIDE == 64 ? 4 : 2;
    static constexpr int PER_SIMD = SIDE == 256 || 2 * BUFFERS * BUFFER <= 160 * 1024 ? 2 : 1;    // waves
};

// A tile of 32 x 32 of a symmetric product by four waves, which take its steps in
// turn, each in LDS of its own, and add up: for matrices whose larger tiles
// would leave CUs idle.
template <bool SPLIT_>
struct Narrow {
    static constexpr int SIDE = 32;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int WAVES = 4, THREADS = 64 * WAVES, FM = 1, FN = 1;
    static constexpr int FACTORS = SPLIT ? 4 : 2;
    static constexpr int ROWS = SIDE * static_cast<int>(kStepBytes);
    static constexpr int STEP = FACTORS * ROWS;               // bytes of a wave's step
    static constexpr int BUFFER = WAVES * STEP, BUFFERS = 2;
    static constexpr int LOADS = STEP / 1024;
    static constexpr int PER_SIMD = 2 * BUFFERS * BUFFER <= 160 * 1024 ? 2 : 1;
};

struct Factor {
    const char *hi, *lo;     // the tile's first row
    uint32_t row_bytes;
};

template <typename S>
__device__ __forceinline__ void bring_rows(const char* p, uint32_t row_bytes, uint32_t step, char* to)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // a wave's groups of 8 rows have its own parity
    const uint32_t mine = (8 * wave + (lane >> 3)) * row_bytes + brought_piece(lane, wave) * kSlot;
    p += static_cast<uint64_t>(step) * kStepBytes;
#pragma unroll
    for (int i = 0; i < S::SIDE / (8 * S::WAVES); ++i)
        bring(p + static_cast<uint64_t>(8 * S::WAVES * i) * row_bytes + mine, to + (S::WAVES * i + wave) * 1024);
}

template <typename S>
__device__ __forceinline__ void bring_step(const Factor& p, const Factor& q, uint32_t step, char* buffer)
{
    bring_rows<S>(p.hi, p.row_bytes, step, buffer);
    bring_rows<S>(q.hi, q.row_bytes, step, buffer + S::ROWS);
    if constexpr (S::SPLIT) {
        bring_rows<S>(p.lo, p.row_bytes, step, buffer + 2 * S::ROWS);
        bring_rows<S>(q.lo, q.row_bytes, step, buffer + 3 * S::ROWS);
    }
    // the loads stay ahead of the products that hide them
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ float16v multiply(half8 a, half8 b, float16v acc)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc, 0, 0, 0);
}

template <typename S>
using Acc = float16v[S::FM][S::FN];

template <typename S>
__device__ __forceinline__ void clear(Acc<S>& acc)
{
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t)
            acc[s][t] = float16v{};
}

template <typename S>
__device__ __forceinline__ void add(Acc<S>& acc, const Acc<S>& more)
{
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t)
            acc[s][t] += more[s][t];
}

// One instruction depth's share of the factors.
template <typename S>
struct Fragments {
    half8 a[S::FM], b[S::FN], a_lo[S::SPLIT ? S::FM : 1], b_lo[S::SPLIT ? S::FN : 1];
};

template <typename S>
__device__ __forceinline__ void read_fragments(Fragments<S>& f, const char* buffer, uint32_t o)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const char* p = buffer + (wave & 1) * (S::FM * kBlockBytes) + piece_at(lane, o);
    const char* q = buffer + S::ROWS + (wave >> 1) * (S::FN * kBlockBytes) + piece_at(lane, o);
#pragma unroll
    for (int s = 0; s < S::FM; ++s) {
        f.a[s] = *reinterpret_cast<const half8*>(p + s * kBlockBytes);
        if constexpr (S::SPLIT)
            f.a_lo[s] = *reinterpret_cast<const half8*>(p + 2 * S::ROWS + s * kBlockBytes);
    }
#pragma unroll
    for (int t = 0; t < S::FN; ++t) {
        f.b[t] = *reinterpret_cast<const half8*>(q + t * kBlockBytes);
        if constexpr (S::SPLIT)
            f.b_lo[t] = *reinterpret_cast<const half8*>(q + 2 * S::ROWS + t * kBlockBytes);
    }
}

// With SPLIT, `acc` takes the products of the high parts and `small` those of a
// high and a low part.  The reads issued before go between the products.
template <typename S>
__device__ __forceinline__ void multiply_fragments(const Fragments<S>& f, Acc<S>& acc, Acc<S>& small)
{
    constexpr int READS = (S::FM + S::FN) * (S::SPLIT ? 2 : 1), PRODUCTS = S::FM * S::FN * (S::SPLIT ? 3 : 1);
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t) {
            acc[s][t] = multiply(f.a[s], f.b[t], acc[s][t]);
            if constexpr (S::SPLIT) {
                small[s][t] = multiply(f.a[s], f.b_lo[t], small[s][t]);
                small[s][t] = multiply(f.a_lo[s], f.b[t], small[s][t]);
            }
        }
    constexpr int EACH = (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
    for (int k = 0; k < PRODUCTS; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);
    }
}

// The tile's sums over `steps` steps.  With SPLIT the products of the high
// parts are summed over 128 elements and added up outside the matrix cores, and
// the small ones apart from them: in one running sum the error of an update of
// low rank is 3.3e-5 of the result, a plain binary32 product's own is 1.2e-5.
template <typename S>
__device__ __forceinline__ void products(const Factor& p, const Factor& q, uint32_t steps,
                                         char* (&buffers)[S::BUFFERS], Acc<S>& acc)
{
    Acc<S> part, small;
    clear<S>(acc);
    clear<S>(small);
    pipeline<S::LOADS, Fragments<S>>(
        steps, buffers, [](uint32_t, int) {}, [&](uint32_t k, char* buffer) { bring_step<S>(p, q, k, buffer); },
        [&](Fragments<S>& f, const char* buffer, uint32_t o) { read_fragments<S>(f, buffer, o); },
        [&](const Fragments<S>& f, int depth) {
            if constexpr (S::SPLIT) {
                if (depth % 8 == 0)
                    clear<S>(part);
                multiply_fragments<S>(f, part, small);
                if (depth % 8 == 7)
                    add<S>(acc, part);
            } else {
                multiply_fragments<S>(f, acc, small);
            }
        });
    if constexpr (S::SPLIT) {
        if (steps % 2)
            add<S>(acc, part);
        add<S>(acc, small);
    }
}

// The same of a narrow tile, in the first wave.
template <typename S>
__device__ __forceinline__ void products_in_turn(const Factor& p, const Factor& q, uint32_t steps, char* (&buffers)[2],
                                                 Acc<S>& acc)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Acc<S> part, small;
    clear<S>(acc);
    clear<S>(small);
    auto rows = [&](const char* from, uint32_t row_bytes, uint32_t step, char* to) {
        from += static_cast<uint64_t>(step) * kStepBytes;
#pragma unroll
        for (uint32_t i = 0; i < S::SIDE / 8; ++i)
            bring(from + (8 * i + (lane >> 3)) * row_bytes + brought_piece(lane, i) * kSlot, to + i * 1024);
    };
    auto bring_own = [&](uint32_t step, char* to) {
        rows(p.hi, p.row_bytes, step, to);
        rows(q.hi, q.row_bytes, step, to + S::ROWS);
        if constexpr (S::SPLIT) {
            rows(p.lo, p.row_bytes, step, to + 2 * S::ROWS);
            rows(q.lo, q.row_bytes, step, to + 3 * S::ROWS);
        }
    };
    auto work = [&](uint32_t step, char* own) {
        // its loads have landed but those of the wave's next step
        if (step + S::WAVES < steps)
            landed_own<S::LOADS>();
        else
            landed_own<0>();
        Fragments<S> f[kDepths];
#pragma unroll
        for (int o = 0; o < kDepths; ++o) {
            const char* at = own + piece_at(lane, o);
            f[o].a[0] = *reinterpret_cast<const half8*>(at);
            f[o].b[0] = *reinterpret_cast<const half8*>(at + S::ROWS);
            if constexpr (S::SPLIT) {
                f[o].a_lo[0] = *reinterpret_cast<const half8*>(at + 2 * S::ROWS);
                f[o].b_lo[0] = *reinterpret_cast<const half8*>(at + 3 * S::ROWS);
            }
        }
        reads_done();
        if (step + 2 * S::WAVES < steps)
            bring_own(step + 2 * S::WAVES, own);
        if constexpr (S::SPLIT)
            clear<S>(part);
#pragma unroll
        for (int o = 0; o < kDepths; ++o) {
            if constexpr (S::SPLIT) {
                part[0][0] = multiply(f[o].a[0], f[o].b[0], part[0][0]);
                small[0][0] = multiply(f[o].a[0], f[o].b_lo[0], small[0][0]);
                small[0][0] = multiply(f[o].a_lo[0], f[o].b[0], small[0][0]);
            } else {
                acc[0][0] = multiply(f[o].a[0], f[o].b[0], acc[0][0]);
            }
        }
        if constexpr (S::SPLIT)
            add<S>(acc, part);
    };
    char* own0 = buffers[0] + wave * S::STEP;
    char* own1 = buffers[1] + wave * S::STEP;
    if (wave < steps)
        bring_own(wave, own0);
    if (wave + S::WAVES < steps)
        bring_own(wave + S::WAVES, own1);
    for (uint32_t k = wave; k < steps; k += 2 * S::WAVES) {
        work(k, own0);
        if (k + S::WAVES < steps)
            work(k + S::WAVES, own1);
    }
    if constexpr (S::SPLIT)
        add<S>(acc, small);
    __syncthreads();
    float16v* sums = reinterpret_cast<float16v*>(buffers[1]);
    if (wave > 0)
        sums[(wave - 1) * 64 + lane] = acc[0][0];
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int w = 0; w < S::WAVES - 1; ++w)
            acc[0][0] += sums[w * 64 + lane];
    }
}

// A symmetric product's tile (ti, tj); false for the waves that have no part of it.
template <typename S>
__device__ __forceinline__ bool symmetric(const Factor& p, const Factor& q, uint32_t steps, char* (&buffers)[S::BUFFERS],
                                          Acc<S>& acc)
{
    if constexpr (S::SIDE == 32) {
        products_in_turn<S>(p, q, steps, buffers, acc);
        return threadIdx.x < 64;
    } else {
        products<S>(p, q, steps, buffers, acc);
        return true;
    }
}

__device__ __forceinline__ Factor factor(const _Float16* hi, const _Float16* lo, uint64_t row, uint32_t cols)
{
    Factor f;
    f.hi = reinterpret_cast<const char*>(hi + row * cols);
    f.lo = reinterpret_cast<const char*>(lo + row * cols);
    f.row_bytes = 2 * cols;
    return f;
}

// The k-th tile on or below the diagonal, row by row.
__device__ __forceinline__ void lower_tile(uint32_t k, uint32_t& ti, uint32_t& tj)
{
    uint32_t i = static_cast<uint32_t>((sqrtf(8.0f * k + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > k)
        --i;
    while ((i + 1) * (i + 2) / 2 <= k)
        ++i;
    ti = i;
    tj = k - i * (i + 1) / 2;
}

// A wave's part of tile (ti, tj): its first row and column.
template <typename S>
struct Place {
    uint32_t row, col;

    __device__ __forceinline__ Place(uint32_t ti, uint32_t tj)
    {
        const uint32_t wave = threadIdx.x >> 6;
        row = ti * S::SIDE + (wave & 1) * (32 * S::FM);
        col = tj * S::SIDE + (wave >> 1) * (32 * S::FN);
    }
};

// Between two ways out of C: no conversion of it is kept from the one to the
// other, which would take as many registers again.
template <typename S>
__device__ __forceinline__ void forget(Acc<S>& acc)
{
#pragma unroll
    for (int s = 0; s < S::FM; ++s)
#pragma unroll
        for (int t = 0; t < S::FN; ++t)
            asm volatile("" : "+v"(acc[s][t]));
}

__device__ __forceinline__ _Float16 high(float v) { return static_cast<_Float16>(v); }
__device__ __forceinline__ _Float16 low(float v) { return static_cast<_Float16>(v - static_cast<float>(high(v))); }

// The wave's part to rows of `ld` binary16, high parts and, where wanted, low ones.
template <typename S>
__device__ __forceinline__ void store_rows(_Float16* hi, _Float16* lo, uint32_t ld, const Place<S>& at, Acc<S>& acc,
                                           char* own)
{
    auto to = [&](_Float16* x) {
        return [=](uint32_t i, uint32_t j, const uint4& run) {
            *reinterpret_cast<uint4*>(x + static_cast<uint64_t>(at.row + i) * ld + at.col + j) = run;
        };
    };
    forget<S>(acc);
    rows_out<_Float16>(acc, own, high, to(hi));
    if constexpr (S::SPLIT) {
        forget<S>(acc);
        rows_out<_Float16>(acc, own, low, to(lo));
    }
}

// ... and turned, to columns as rows.
template <typename T, typename S, typename C>
__device__ __forceinline__ void store_turned(T* x, uint32_t ld, const Place<S>& at, Acc<S>& acc, char* own, C convert)
{
    forget<S>(acc);
    columns_out<T>(acc, own, convert, [=](uint32_t j, uint32_t i, const uint4& run) {
        *reinterpret_cast<uint4*>(x + static_cast<uint64_t>(at.col + j) * ld + at.row + i) = run;
    });
}

// A block's elements of a turned matrix, four a load.
__device__ __forceinline__ void load_turned(const _Float16* x, uint64_t at, float v[16])
{
    typedef _Float16 half4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const half4 h = *reinterpret_cast<const half4*>(x + at + 8 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r)
            v[4 * g + r] = static_cast<float>(h[r]);
    }
}

__device__ __forceinline__ void load_turned(const float* x, uint64_t at, float v[16])
{
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4 f = *reinterpret_cast<const float4*>(x + at + 8 * g);
        v[4 * g] = f.x;
        v[4 * g + 1] = f.y;
        v[4 * g + 2] = f.z;
        v[4 * g + 3] = f.w;
    }
}

template <typename S>
__global__ __launch_bounds__(S::THREADS, S::PER_SIMD) void gram_kernel(OrthParams p)
{
    BUFFERS_IN_LDS(S)
    uint32_t ti, tj;
    lower_tile(blockIdx.x, ti, tj);
    const uint64_t x = static_cast<uint64_t>(blockIdx.y) * p.mp * p.np, o = static_cast<uint64_t>(blockIdx.y) * p.mp * p.mp;
    Acc<S> acc;
    if (!symmetric<S>(factor(p.s.x + x, p.s.x_lo + x, ti * S::SIDE, p.np),
                      factor(p.s.x + x, p.s.x_lo + x, tj * S::SIDE, p.np), p.steps_n, buffers, acc))
        return;
    _Float16* hi = p.s.o + o;
    _Float16* lo = p.s.o_lo + o;
    float* d = p.s.d + blockIdx.y * p.mp;
    const Place<S> at(ti, tj);
    char* own = own_part<S::FM, S::BUFFER>(buffers[0], buffers[1], threadIdx.x >> 6);
    each_block(acc, [&](uint32_t i, uint32_t j, float16v& v) {
        v *= kScaleA / (kScaleX * kScaleX);
        if (ti == tj) {
#pragma unroll
            for (int q = 0; q < 16; ++q)
                if (at.row + i + row_of(q) == at.col + j) {
                    d[at.col + j] = v[q] * (1.0f / kScaleA);
                    v[q] = 0.0f;
                }
        }
    });
    store_rows<S>(hi, lo, p.mp, at, acc, own);
    if (ti != tj) {
        store_turned(hi, p.mp, at, acc, own, high);
        if constexpr (S::SPLIT)
            store_turned(lo, p.mp, at, acc, own, low);
    }
}

template <typename S>
__global__ __launch_bounds__(S::THREADS, S::PER_SIMD) void square_kernel(OrthParams p)
{
    BUFFERS_IN_LDS(S)
    uint32_t ti, tj;
    lower_tile(blockIdx.x, ti, tj);
    const uint64_t o = static_cast<uint64_t>(blockIdx.y) * p.mp * p.mp;
    const _Float16* o_hi = p.s.o + o;
    const _Float16* o_lo = p.s.o_lo + o;
    Acc<S> acc;
    if (!symmetric<S>(factor(o_hi, o_lo, ti * S::SIDE, p.mp), factor(o_hi, o_lo, tj * S::SIDE, p.mp), p.steps_m, buffers,
                      acc))
        return;
    _Float16* hi = p.s.b + o;
    _Float16* lo = p.s.b_lo + o;
    const float* d = p.s.d + blockIdx.y * p.mp;
    float* d_b = p.s.d_b + blockIdx.y * p.mp;
    const Place<S> at(ti, tj);
    char* own = own_part<S::FM, S::BUFFER>(buffers[0], buffers[1], threadIdx.x >> 6);
    each_block(acc, [&](uint32_t bi, uint32_t bj, float16v& v) {
        const uint32_t i = at.row + bi, j = at.col + bj;
        // O is symmetric: its row j has the block's column
        float e[16], more[16], di[16];
        const uint64_t turned = static_cast<uint64_t>(j) * p.mp + i;
        load_turned(o_hi, turned, e);
        if constexpr (S::SPLIT)
            load_turned(o_lo, turned, more);
        load_turned(d, i, di);
        const float dj = d[j];
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const float square = v[q] * (1.0f / (kScaleA * kScaleA));
            const float a = (S::SPLIT ? e[q] + more[q] : e[q]) * (1.0f / kScaleA);
            v[q] = kScaleB * (p.b * a + p.c * (square + (di[q] + dj) * a));
            if (ti == tj && i + row_of(q) == j) {
                d_b[j] = p.a + p.b * dj + p.c * (dj * dj + square);
                v[q] = 0.0f;
            }
        }
    });
    store_rows<S>(hi, lo, p.mp, at, acc, own);
    if (ti != tj) {
        store_turned(hi, p.mp, at, acc, own, high);
        if constexpr (S::SPLIT)
            store_turned(lo, p.mp, at, acc, own, low);
    }
}

// The result of a wave's part in the layout of `out`: along or down it where
// either side is contiguous.
template <typename T, typename S>
__device__ __forceinline__ void store_result(const OrthParams& p, uint32_t b, const Place<S>& at, Acc<S>& acc, char* own)
{
    forget<S>(acc);
    T* out = static_cast<T*>(p.out) + b * p.out_batch;
    if (p.out_col == 1) {
        rows_out<T>(acc, own, from_f32<T>, [&](uint32_t i, uint32_t j, const uint4& run) {
            if (at.row + i < static_cast<uint32_t>(p.m))
                store_inside(out + (at.row + i) * p.out_row + at.col + j, static_cast<int64_t>(p.n) - at.col - j, run);
        });
    } else {
        columns_out<T>(acc, own, from_f32<T>, [&](uint32_t j, uint32_t i, const uint4& run) {
            if (at.col + j >= static_cast<uint32_t>(p.n))
                return;
            T* to = out + (at.col + j) * p.out_col + (at.row + i) * p.out_row;
            const int64_t left = static_cast<int64_t>(p.m) - at.row - i;
            if (p.out_row == 1) {
                store_inside(to, left, run);
            } else {
                T e[16 / sizeof(T)];
                __builtin_memcpy(e, &run, 16);
#pragma unroll
                for (uint32_t k = 0; k < 16 / sizeof(T); ++k)
                    if (k < left)
                        to[k * p.out_row] = e[k];
            }
        });
    }
}

template <typename S, bool LAST>
__global__ __launch_bounds__(S::THREADS, S::PER_SIMD) void step_kernel(OrthParams p)
{
    BUFFERS_IN_LDS(S)
    const uint32_t b = blockIdx.z, ti = blockIdx.y, tj = blockIdx.x;
    const uint64_t x = static_cast<uint64_t>(b) * p.mp * p.np, o = static_cast<uint64_t>(b) * p.mp * p.mp;
    Acc<S> acc;
    products<S>(factor(p.s.b + o, p.s.b_lo + o, ti * S::SIDE, p.mp),
                factor(p.s.xt + x, p.s.xt_lo + x, tj * S::SIDE, p.mp), p.steps_m, buffers, acc);
    const float* d_b = p.s.d_b + b * p.mp;
    const Place<S> at(ti, tj);
    char* own = own_part<S::FM, S::BUFFER>(buffers[0], buffers[1], threadIdx.x >> 6);
    each_block(acc, [&](uint32_t bi, uint32_t bj, float16v& v) {
        const uint64_t turned = x + static_cast<uint64_t>(at.col + bj) * p.mp + at.row + bi;
        float old[16], more[16], d[16];
        if constexpr (S::SPLIT) {
            load_turned(p.s.xt_full, turned, old);
        } else {
            load_turned(p.s.xt, turned, old);
            load_turned(p.s.xt_lo, turned, more);
        }
        load_turned(d_b, at.row + bi, d);
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            v[q] = __builtin_fmaf(d[q], S::SPLIT ? old[q] : old[q] + more[q], v[q] * (1.0f / kScaleB));
            if constexpr (LAST)
                v[q] *= 1.0f / kScaleX;
        }
    });
    if constexpr (LAST && !S::SPLIT) {
        store_result<__bf16>(p, b, at, acc, own);
    } else if constexpr (LAST) {
        if (p.out_dtype == SQN_F32)
            store_result<float>(p, b, at, acc, own);
        else
            store_result<_Float16>(p, b, at, acc, own);
    } else {
        store_rows<S>(p.s.x + x, p.s.x_lo + x, p.np, at, acc, own);
        store_turned(p.s.xt_to + x, p.mp, at, acc, own, high);
        store_turned(p.s.xt_to_lo + x, p.mp, at, acc, own, low);
        if constexpr (S::SPLIT)
            store_turned(p.s.xt_full + x, p.mp, at, acc, own, [](float v) { return v; });
    }
}

// ---- small matrices: one workgroup each, all steps in one launch
//
// X stays in registers, in binary32, as the accumulators of its blocks; LDS
// holds the factor that a product reads: X, then O, then X^T in X's place and B
// in O's.  The launches of the tiles take 17 times 4 us whatever the size.

constexpr int kSmallThreads = 512;
constexpr int kSmallWaves = kSmallThreads / 64;

// M x N blocks of 32 x 32.
template <int M_, int N_, bool SPLIT_>
struct Small {
    static constexpr int M = M_, N = N_;
    static constexpr bool SPLIT = SPLIT_;
    static constexpr int XB = (M * N + kSmallWaves - 1) / kSmallWaves;    // blocks of X a wave
    static constexpr int OB = (M * M + kSmallWaves - 1) / kSmallWaves;    // of O and B
    // bytes of a row of a factor: its elements, of at least 128, so that 16 rows differ in their slots
    static constexpr uint32_t PITCH_N = (N > 4 ? N : 4) * 64, PITCH_M = 4 * 64;
    static constexpr uint32_t X_BYTES = M * 32 * PITCH_N > N * 32 * PITCH_M ? M * 32 * PITCH_N : N * 32 * PITCH_M;
    static constexpr uint32_t O_BYTES = M * 32 * PITCH_M;
};

// Element k of row r of a factor lies in the piece of 16 bytes (k / 8) ^ (r % 16)
// of the row, so 16 rows' pieces are in slots of their own.  Rows and elements
// of a lane are a part that the lane fixes and one that the code does, in
// different bits: the slots are one exclusive or of both.

// A block's elements to rows of a factor: element q at (i + row_of(q), j), i a
// multiple of 32 plus 0 or 4.
__device__ __forceinline__ void small_store(char* hi, char* lo, uint32_t pitch, uint32_t i, uint32_t j, const float16v& v)
{
    const uint32_t slot = ((j >> 3) ^ (i & 4)) * 16 + (j & 7) * 2;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
        const uint32_t at = i * pitch + (slot ^ (row_of(q) & 15) * 16) + row_of(q) * pitch;
        *reinterpret_cast<_Float16*>(hi + at) = high(v[q]);
        if (lo)
            *reinterpret_cast<_Float16*>(lo + at) = low(v[q]);
    }
}

// ... turned, element q at (j, i + row_of(q)).
__device__ __forceinline__ void small_store_turned(char* hi, char* lo, uint32_t pitch, uint32_t i, uint32_t j,
                                                   const float16v& v)
{
    typedef _Float16 half4 __attribute__((ext_vector_type(4)));
    const uint32_t slot = ((i >> 3) ^ (j & 15)) * 16 + (i & 4) * 2;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        half4 h, l;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            h[r] = high(v[4 * g + r]);
            l[r] = low(v[4 * g + r]);
        }
        const uint32_t at = j * pitch + (slot ^ g * 16);
        *reinterpret_cast<half4*>(hi + at) = h;
        if (lo)
            *reinterpret_cast<half4*>(lo + at) = l;
    }
}

// Blocks of P Q^T over `depth` elements: rows i of P on, and j, j + apart, ...
// of Q.  P's fragment serves all of them.
template <bool SPLIT, int B>
__device__ __forceinline__ void small_products(const char* p, const char* p_lo, uint32_t i, const char* q, const char* q_lo,
                                               uint32_t j, uint32_t apart, uint32_t pitch, uint32_t depth,
                                               float16v (&acc)[B])
{
    const uint32_t lane = threadIdx.x & 63, row = lane & 31, slot = ((lane >> 5) ^ (row & 15)) * 16;
    auto read = [&](const char* x, uint32_t r, uint32_t k) {
        return *reinterpret_cast<const half8*>(x + r * pitch + (row * pitch + (slot ^ 2 * k)));
    };
    float16v small[B];
#pragma unroll
    for (int c = 0; c < B; ++c)
        acc[c] = small[c] = float16v{};
#pragma unroll 4
    for (uint32_t k = 0; k < depth; k += 16) {
        const half8 a = read(p, i, k);
        half8 b[B];
#pragma unroll
        for (int c = 0; c < B; ++c)
            b[c] = read(q, j + c * apart, k);
        if constexpr (SPLIT) {
            const half8 a_lo = read(p_lo, i, k);
#pragma unroll
            for (int c = 0; c < B; ++c) {
                small[c] = multiply(a, read(q_lo, j + c * apart, k), small[c]);
                small[c] = multiply(a_lo, b[c], small[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < B; ++c)
            acc[c] = multiply(a, b[c], acc[c]);
    }
    if constexpr (SPLIT) {
#pragma unroll
        for (int c = 0; c < B; ++c)
            acc[c] += small[c];
    }
}

template <typename S, typename T, typename O>
__global__ __launch_bounds__(kSmallThreads) void small_kernel(OrthParams p, int32_t steps)
{
    constexpr int M = S::M, N = S::N;
    __shared__ __align__(16) char x[(S::SPLIT ? 2 : 1) * S::X_BYTES];
    __shared__ __align__(16) char o[(S::SPLIT ? 2 : 1) * S::O_BYTES];
    __shared__ float d[32 * M], d_b[32 * M];
    __shared__ double sums[kSmallWaves];
    char* const x_lo = S::SPLIT ? x + S::X_BYTES : nullptr;
    char* const o_lo = S::SPLIT ? o + S::O_BYTES : nullptr;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t m = p.m, n = p.n, di = 4 * (lane >> 5), dj = lane & 31;
    // The wave's blocks are in one row of blocks, their columns `apart`; of O's
    // and B's a wave has OB or none.
    static_assert(kSmallWaves % M == 0 && (M * N) % kSmallWaves == 0, "whole rounds of waves");
    constexpr uint32_t apart = 32 * kSmallWaves / M;
    const uint32_t bi = 32 * (wave % M), bj = 32 * (wave / M);
    const bool has_o = wave < M * M;
    // f(c, i, j) over the wave's first `count` blocks: the c-th, whose element q of
    // this lane is (i + row_of(q), j)
    auto blocks = [&](int count, auto f) {
#pragma unroll
        for (int c = 0; c < count; ++c)
            f(c, bi + di, bj + c * apart + dj);
    };

    float16v v[S::XB];
    double sum = 0.0;
    const T* in = static_cast<const T*>(p.in) + blockIdx.x * p.in_batch;
    blocks(S::XB, [&](int c, uint32_t i, uint32_t j) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint32_t r = i + row_of(q);
            v[c][q] = r < m && j < n ? to_f32(in[r * p.in_row + j * p.in_col]) : 0.0f;
        }
#pragma unroll
        for (int q = 0; q < 16; ++q)
            sum = __builtin_fma(static_cast<double>(v[c][q]), static_cast<double>(v[c][q]), sum);
    });
    for (int s = 32; s; s /= 2)
        sum += __shfl_xor(sum, s);
    if (lane == 0)
        sums[wave] = sum;
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kSmallWaves; ++w)
        sum += sums[w];
    const double norm = sqrt(sum) + static_cast<double>(p.eps);
    const double scale = norm > 0.0 ? kScaleX / norm : 0.0;
    // a NaN or an infinity anywhere gives NaN everywhere
    const float nan = isfinite(norm) ? 0.0f : __builtin_nanf("");
    blocks(S::XB, [&](int c, uint32_t, uint32_t) {
#pragma unroll
        for (int q = 0; q < 16; ++q)
            v[c][q] = static_cast<float>(v[c][q] * scale) + nan;
    });

    for (int32_t step = 0; step < steps; ++step) {
        blocks(S::XB, [&](int c, uint32_t i, uint32_t j) { small_store(x, x_lo, S::PITCH_N, i, j, v[c]); });
        __syncthreads();
        float16v a[S::OB];
        if (has_o) {
            small_products<S::SPLIT, S::OB>(x, x_lo, bi, x, x_lo, bj, apart, S::PITCH_N, 32 * N, a);
            blocks(S::OB, [&](int c, uint32_t i, uint32_t j) {
                a[c] *= kScaleA / (kScaleX * kScaleX);
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    if (i + row_of(q) == j) {
                        d[j] = a[c][q] * (1.0f / kScaleA);
                        a[c][q] = 0.0f;
                    }
                small_store_turned(o, o_lo, S::PITCH_M, i, j, a[c]);
            });
        }
        __syncthreads();
        blocks(S::XB, [&](int c, uint32_t i, uint32_t j) { small_store_turned(x, x_lo, S::PITCH_M, i, j, v[c]); });
        if (has_o) {
            float16v square[S::OB];
            small_products<S::SPLIT, S::OB>(o, o_lo, bi, o, o_lo, bj, apart, S::PITCH_M, 32 * M, square);
            blocks(S::OB, [&](int c, uint32_t i, uint32_t j) {
                const float dcol = d[j];
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const float s = square[c][q] * (1.0f / (kScaleA * kScaleA)), e = a[c][q] * (1.0f / kScaleA);
                    a[c][q] = kScaleB * (p.b * e + p.c * (s + (d[i + row_of(q)] + dcol) * e));
                    if (i + row_of(q) == j) {
                        d_b[j] = p.a + p.b * dcol + p.c * (dcol * dcol + s);
                        a[c][q] = 0.0f;
                    }
                }
            });
        }
        __syncthreads();
        if (has_o)
            blocks(S::OB, [&](int c, uint32_t i, uint32_t j) { small_store_turned(o, o_lo, S::PITCH_M, i, j, a[c]); });
        __syncthreads();
        float16v more[S::XB];
        small_products<S::SPLIT, S::XB>(o, o_lo, bi, x, x_lo, bj, apart, S::PITCH_M, 32 * M, more);
        blocks(S::XB, [&](int c, uint32_t i, uint32_t) {
#pragma unroll
            for (int q = 0; q < 16; ++q)
                v[c][q] = __builtin_fmaf(d_b[i + row_of(q)], v[c][q], more[c][q] * (1.0f / kScaleB));
        });
        __syncthreads();
    }

    O* out = static_cast<O*>(p.out) + blockIdx.x * p.out_batch;
    blocks(S::XB, [&](int c, uint32_t i, uint32_t j) {
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const uint32_t r = i + row_of(q);
            if (r < m && j < n)
                out[r * p.out_row + j * p.out_col] = from_f32<O>(v[c][q] * (1.0f / kScaleX));
        }
    });
}

// ---- layout and launches

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Whether one workgroup does a matrix of m <= n: its factors, and their low
// parts where they are split, lie in the 160 KB of a CU.
bool is_small(int32_t m, int32_t n, bool split_all) { return m <= 128 && n <= (split_all ? 128 : 256); }

template <typename S, typename T>
void launch_small_to(const OrthParams& p, int32_t batch, int32_t steps, hipStream_t stream)
{
    if constexpr (!S::SPLIT)
        small_kernel<S, T, __bf16><<<batch, kSmallThreads, 0, stream>>>(p, steps);
    else if (p.out_dtype == SQN_F32)
        small_kernel<S, T, float><<<batch, kSmallThreads, 0, stream>>>(p, steps);
    else
        small_kernel<S, T, _Float16><<<batch, kSmallThreads, 0, stream>>>(p, steps);
}

template <typename T>
hipError_t launch_small(const OrthParams& p, int32_t batch, int32_t steps, bool split_all, hipStream_t stream)
{
    const bool low = p.m <= 64;
    if (split_all) {
        if (low)
            launch_small_to<Small<2, 4, true>, T>(p, batch, steps, stream);
        else
            launch_small_to<Small<4, 4, true>, T>(p, batch, steps, stream);
    } else if (p.n <= 128) {
        if (low)
            launch_small_to<Small<2, 4, false>, T>(p, batch, steps, stream);
        else
            launch_small_to<Small<4, 4, false>, T>(p, batch, steps, stream);
    } else {
        if (low)
            launch_small_to<Small<2, 8, false>, T>(p, batch, steps, stream);
        else
            launch_small_to<Small<4, 8, false>, T>(p, batch, steps, stream);
    }
    return hipGetLastError();
}

int32_t up_to(int32_t v, int32_t side) { return (v + side - 1) / side * side; }

// Side of the tiles of a batch of matrices: the largest whose tiles fill the chip
// and whose rows and columns past the matrix add at most half to the products
// that tiles of 64 take, and to their scratch.  (Larger tiles and those of 64, us
// to bfloat16: 64 of 390 x 390 534 and 736, products 1.49 times as large; 24 of 520
// x 520 470 and 500, 1.37; 16 of 257 x 900 244 and 213, 1.54; 24 of 130 x 1300 293
// and 199, 1.86; 1000 of 16 x 4096 14,560 and 4,629, with 8.7 and 2.1 GB.)
int32_t tile_side(int32_t batch, int32_t m, int32_t n, bool split_all)
{
    auto taken = [&](int32_t side) {
        const int64_t mp = up_to(m, side), np = up_to(n, side);
        return batch * (mp / side) * (np / side) >= 200
               && 2 * mp * mp * np <= 3 * int64_t{up_to(m, 64)} * up_to(m, 64) * up_to(n, 64);
    };
    if (!split_all && taken(256))
        return 256;
    return taken(128) ? 128 : 64;
}

// Narrow tiles take the symmetric products where tiles of 64 would and each CU
// has one narrow tile at most.  (The call with them and without, us: 701 x 1100
// to binary32, 253 narrow tiles, 147 and 178, to bfloat16 108 and 120; 300 x 400
// to binary32, 55 of them, 104 and 124; 900 x 900, 465 of them, 227 and 202.)
constexpr int64_t kCus = 256;

size_t layout(int32_t batch, int32_t rows, int32_t cols, bool split_all, char* base, Scratch* s)
{
    const int32_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    if (is_small(m, n, split_all))
        return 0;
    const int32_t side = tile_side(batch, m, n, split_all);
    const size_t mp = up_to(m, side), np = up_to(n, side);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char* here = base + at;
        at += padded(bytes * batch);
        return here;
    };
    auto halves = [&](size_t count, bool wanted) {
        return wanted ? reinterpret_cast<_Float16*>(take(2 * count)) : nullptr;
    };
    Scratch t;
    t.x = halves(mp * np, true);
    t.x_lo = halves(mp * np, split_all);
    t.xt = halves(mp * np, true);
    t.xt_to = halves(mp * np, true);
    t.xt_lo = halves(mp * np, true);
    t.xt_to_lo = split_all ? halves(mp * np, true) : t.xt_lo;
    t.xt_full = split_all ? reinterpret_cast<float*>(take(4 * mp * np)) : nullptr;
    t.o = halves(mp * mp, true);
    t.b = halves(mp * mp, true);
    t.o_lo = halves(mp * mp, split_all);
    t.b_lo = halves(mp * mp, split_all);
    t.d = reinterpret_cast<float*>(take(4 * mp));
    t.d_b = reinterpret_cast<float*>(take(4 * mp));
    t.norms = reinterpret_cast<double*>(take(8 * kNormBlocks));
    if (s)
        *s = t;
    return at;
}

template <typename T>
void launch_start(const OrthParams& p, int32_t batch, hipStream_t stream)
{
    norm_kernel<T><<<dim3(kNormBlocks, batch), kThreads, 0, stream>>>(p);
    start_kernel<T><<<dim3(p.np / 64, p.mp / 64, batch), kThreads, 0, stream>>>(p);
}

// The symmetric products in tiles of G, B X in tiles of S.
template <typename S, typename G = S>
hipError_t run_steps(OrthParams p, int32_t batch, int32_t steps, hipStream_t stream)
{
    const uint32_t tg = p.mp / G::SIDE;
    const dim3 lower(tg * (tg + 1) / 2, batch), all(p.np / S::SIDE, p.mp / S::SIDE, batch);
    for (int32_t k = 0; k < steps; ++k) {
        gram_kernel<G><<<lower, G::THREADS, 0, stream>>>(p);
        square_kernel<G><<<lower, G::THREADS, 0, stream>>>(p);
        if (k + 1 == steps) {
            step_kernel<S, true><<<all, S::THREADS, 0, stream>>>(p);
            break;
        }
        step_kernel<S, false><<<all, S::THREADS, 0, stream>>>(p);
        _Float16* t = p.s.xt;
        p.s.xt = p.s.xt_to;
        p.s.xt_to = t;
        t = p.s.xt_lo;
        p.s.xt_lo = p.s.xt_to_lo;
        p.s.xt_to_lo = t;
    }
    return hipGetLastError();
}

}  // namespace

size_t orthogonalise_bytes(int32_t batch, int32_t rows, int32_t cols, int32_t out_dtype)
{
    return layout(batch, rows, cols, out_dtype != SQN_BF16, nullptr, nullptr);
}

hipError_t launch_orthogonalise(const sqn_batch& updates, int32_t steps, const float coefficients[3], float eps,
                                const sqn_batch& out, void* workspace, hipStream_t stream)
{
    const bool tall = updates.rows > updates.cols;
    const bool split_all = out.dtype != SQN_BF16;
    OrthParams p;
    layout(updates.batch, updates.rows, updates.cols, split_all, static_cast<char*>(workspace), &p.s);
    p.in = updates.data;
    p.out = out.data;
    p.in_batch = updates.batch_stride;
    p.in_row = tall ? updates.col_stride : updates.row_stride;
    p.in_col = tall ? updates.row_stride : updates.col_stride;
    p.out_batch = out.batch_stride;
    p.out_row = tall ? out.col_stride : out.row_stride;
    p.out_col = tall ? out.row_stride : out.col_stride;
    p.m = tall ? updates.cols : updates.rows;
    p.n = tall ? updates.rows : updates.cols;
    const int32_t side = tile_side(updates.batch, p.m, p.n, split_all);
    p.mp = up_to(p.m, side);
    p.np = up_to(p.n, side);
    p.steps_m = (2 * p.m + kStepBytes - 1) / kStepBytes;
    p.steps_n = (2 * p.n + kStepBytes - 1) / kStepBytes;
    p.out_dtype = out.dtype;
    p.a = coefficients[0];
    p.b = coefficients[1];
    p.c = coefficients[2];
    p.eps = eps;
    if (is_small(p.m, p.n, split_all)) {
        if (updates.dtype == SQN_F32)
            return launch_small<float>(p, updates.batch, steps, split_all, stream);
        if (updates.dtype == SQN_F16)
            return launch_small<_Float16>(p, updates.batch, steps, split_all, stream);
        return launch_small<__bf16>(p, updates.batch, steps, split_all, stream);
    }
    if (updates.dtype == SQN_F32)
        launch_start<float>(p, updates.batch, stream);
    else if (updates.dtype == SQN_F16)
        launch_start<_Float16>(p, updates.batch, stream);
    else
        launch_start<__bf16>(p, updates.batch, stream);
    if (steps == 0) {
        emit_kernel<<<dim3(1, p.m, updates.batch), kThreads, 0, stream>>>(p);
        return hipGetLastError();
    }
    const int64_t along = p.mp / Narrow<true>::SIDE;
    const bool narrow = updates.batch * (along * (along + 1) / 2) <= kCus;
    if (split_all) {
        if (side == 128)
            return run_steps<Shape<128, true>>(p, updates.batch, steps, stream);
        return narrow ? run_steps<Shape<64, true>, Narrow<true>>(p, updates.batch, steps, stream)
                      : run_steps<Shape<64, true>>(p, updates.batch, steps, stream);
    }
    if (side == 256)
        return run_steps<Shape<256, false>>(p, updates.batch, steps, stream);
    if (side == 128)
        return run_steps<Shape<128, false>>(p, updates.batch, steps, stream);
    return narrow ? run_steps<Shape<64, false>, Narrow<false>>(p, updates.batch, steps, stream)
                  : run_steps<Shape<64, false>>(p, updates.batch, steps, stream);
}

}  // namespace sqn
