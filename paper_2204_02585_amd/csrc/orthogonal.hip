// Update matrices orthogonalised by Newton-Schulz products.
//
//   X <- G / (||G||_F + eps);  `steps` times:  A = X X^T,
//   X <- a X + (b A + c A A) X
//
// X is held with its shorter side as rows (m <= n), so the square products
// are m x m.  All products are of the form C = P Q^T with rows of P and Q
// contiguous along the sum, on v_mfma_f32_16x16x32_f16:
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
// 256 x 256 update falls from 1.4e-3 to 6e-4 of its norm).  And updates of low
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

namespace sqn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPad = 64;                 // rows, columns and sums are padded to this
constexpr int kNormBlocks = 64;          // workgroups per matrix that sum squares

constexpr float kScaleX = 4096.0f;       // hi + lo = 2^12 X
constexpr float kScaleA = 4096.0f;       // 2^12 O
constexpr float kScaleB = 2048.0f;       // 2^11 (b A + c A A) off the diagonal

// One matrix's scratch; the matrices of a batch follow each other.
struct Scratch {
    _Float16 *x, *x_lo;                  // [mp][np]
    float* x_full;                       // [mp][np], where factors are split
    _Float16 *xt, *xt_lo;                // [np][mp], read by the step
    _Float16 *xt_to, *xt_to_lo;          // [np][mp], written by it
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
    int32_t m, n, mp, np;
    int32_t in_dtype, out_dtype;
    float a, b, c, eps;
    int32_t last;                        // the step writes `out`
};

__device__ __forceinline__ float load_any(const void* p, int64_t i, int32_t dtype)
{
    if (dtype == SQN_F32)
        return static_cast<const float*>(p)[i];
    if (dtype == SQN_F16)
        return static_cast<float>(static_cast<const _Float16*>(p)[i]);
    return static_cast<float>(static_cast<const __bf16*>(p)[i]);
}

__device__ __forceinline__ void store_any(void* p, int64_t i, float v, int32_t dtype)
{
    if (dtype == SQN_F32)
        static_cast<float*>(p)[i] = v;
    else if (dtype == SQN_F16)
        static_cast<_Float16*>(p)[i] = static_cast<_Float16>(v);
    else
        static_cast<__bf16*>(p)[i] = static_cast<__bf16>(v);
}

// Sums of squares of a matrix, kNormBlocks of them, in binary64: gradients may
// be small enough for their squares to vanish in binary32.
__global__ __launch_bounds__(kThreads) void norm_kernel(OrthParams p)
{
    const int64_t base = blockIdx.y * p.in_batch;
    // along the contiguous side
    const bool rows_inner = p.in_row < p.in_col;
    const uint32_t inner = rows_inner ? p.m : p.n, outer = rows_inner ? p.n : p.m;
    const int64_t si = rows_inner ? p.in_row : p.in_col, so = rows_inner ? p.in_col : p.in_row;
    double sum = 0.0;
    const uint64_t total = static_cast<uint64_t>(inner) * outer;
    for (uint64_t k = blockIdx.x * kThreads + threadIdx.x; k < total; k += kNormBlocks * kThreads) {
        const uint32_t j = static_cast<uint32_t>(k / inner), i = static_cast<uint32_t>(k - static_cast<uint64_t>(j) * inner);
        const double v = load_any(p.in, base + i * si + j * so, p.in_dtype);
        sum = __builtin_fma(v, v, sum);
    }
    for (int d = 32; d; d /= 2)
        sum += __shfl_xor(sum, d);
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

// X and X^T of 64 x 64 elements a workgroup, zeros past m and n.
__global__ __launch_bounds__(kThreads) void start_kernel(OrthParams p)
{
    __shared__ float tile[64][65];
    const uint32_t b = blockIdx.z;
    double sum = 0.0;
    for (int k = 0; k < kNormBlocks; ++k)
        sum += p.s.norms[b * kNormBlocks + k];
    const double norm = sqrt(sum) + static_cast<double>(p.eps);
    // a NaN or an infinity anywhere gives NaN everywhere
    const double scale = norm > 0.0 ? kScaleX / norm : 0.0;
    const float inv_nan = isfinite(norm) ? 0.0f : __builtin_nanf("");
    const uint32_t i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
    const bool rows_inner = p.in_row < p.in_col;
    for (uint32_t k = threadIdx.x; k < 64 * 64; k += kThreads) {
        const uint32_t fast = k & 63, slow = k >> 6;
        const uint32_t i = rows_inner ? fast : slow, j = rows_inner ? slow : fast;
        float v = 0.0f;
        if (i0 + i < static_cast<uint32_t>(p.m) && j0 + j < static_cast<uint32_t>(p.n))
            v = static_cast<float>(load_any(p.in, b * p.in_batch + (i0 + i) * p.in_row + (j0 + j) * p.in_col, p.in_dtype)
                                   * scale)
                + inv_nan;
        tile[i][j] = v;
    }
    __syncthreads();
    const uint64_t at = static_cast<uint64_t>(b) * p.mp * p.np;
    for (uint32_t k = threadIdx.x; k < 64 * 64; k += kThreads) {
        const uint32_t fast = k & 63, slow = k >> 6;
        _Float16 hi, lo;
        split(tile[slow][fast], hi, lo);
        const uint64_t x = at + static_cast<uint64_t>(i0 + slow) * p.np + j0 + fast;
        p.s.x[x] = hi;
        p.s.x_lo[x] = lo;
        if (p.s.x_full)
            p.s.x_full[x] = tile[slow][fast];
        split(tile[fast][slow], hi, lo);
        const uint64_t xt = at + static_cast<uint64_t>(j0 + slow) * p.mp + i0 + fast;
        p.s.xt[xt] = hi;
        if (p.s.xt_lo)
            p.s.xt_lo[xt] = lo;
    }
}

// no steps: X itself
__global__ __launch_bounds__(kThreads) void emit_kernel(OrthParams p)
{
    const uint32_t b = blockIdx.z, i = blockIdx.y;
    for (uint32_t j = threadIdx.x; j < static_cast<uint32_t>(p.n); j += kThreads) {
        const uint64_t x = (static_cast<uint64_t>(b) * p.mp + i) * p.np + j;
        const float v = p.s.x_full ? p.s.x_full[x] : static_cast<float>(p.s.x[x]) + static_cast<float>(p.s.x_lo[x]);
        store_any(p.out, b * p.out_batch + i * p.out_row + j * p.out_col, v * (1.0f / kScaleX), p.out_dtype);
    }
}

// ---- products: 64 x 64 of C a workgroup, 32 x 32 a wave

// acc[s][t]: rows 16 s + 4 (lane / 16) + q, column 16 t + lane % 16 of the wave's part.
struct Part {
    float4v acc[2][2];
    uint32_t row, col;      // of acc[0][0][0]
};

__device__ __forceinline__ half8 fragment(const _Float16* p) { return *reinterpret_cast<const half8*>(p); }

__device__ __forceinline__ float4v multiply(half8 a, half8 b, float4v acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, acc, 0, 0, 0);
}

// The sums over all of `sum`.  With SPLIT the products of the high parts are
// formed over stretches of 128 and added up outside the matrix cores, and the
// small ones apart from them: in one running sum the error of an update of
// low rank is 3.3e-5 of the result, a plain binary32 product's own is 1.2e-5.
template <bool SPLIT>
__device__ __forceinline__ void products(Part& c, const _Float16* p, const _Float16* p_lo, const _Float16* q,
                                         const _Float16* q_lo, uint32_t ld_p, uint32_t ld_q, uint32_t sum,
                                         uint32_t tile_row, uint32_t tile_col)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t row = tile_row + (wave & 1) * 32, col = tile_col + (wave >> 1) * 32;
    const uint64_t pf = static_cast<uint64_t>(row + (lane & 15)) * ld_p + 8 * (lane >> 4);
    const uint64_t qf = static_cast<uint64_t>(col + (lane & 15)) * ld_q + 8 * (lane >> 4);
    c.row = row + 4 * (lane >> 4);
    c.col = col + (lane & 15);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
            c.acc[s][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    float4v small[2][2] = {};
    for (uint32_t k0 = 0; k0 < sum; k0 += 128) {
        float4v part[2][2];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                part[s][t] = SPLIT ? float4v{0.0f, 0.0f, 0.0f, 0.0f} : c.acc[s][t];
        const uint32_t end = min(sum, k0 + 128);
        for (uint32_t k = k0; k < end; k += 32) {
            half8 a[2], b[2], a_lo[2], b_lo[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                a[s] = fragment(p + pf + static_cast<uint64_t>(16 * s) * ld_p + k);
                b[s] = fragment(q + qf + static_cast<uint64_t>(16 * s) * ld_q + k);
                if constexpr (SPLIT) {
                    a_lo[s] = fragment(p_lo + pf + static_cast<uint64_t>(16 * s) * ld_p + k);
                    b_lo[s] = fragment(q_lo + qf + static_cast<uint64_t>(16 * s) * ld_q + k);
                }
            }
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if constexpr (SPLIT) {
                        small[s][t] = multiply(a[s], b_lo[t], small[s][t]);
                        small[s][t] = multiply(a_lo[s], b[t], small[s][t]);
                    }
                    part[s][t] = multiply(a[s], b[t], part[s][t]);
                }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                c.acc[s][t] = SPLIT ? c.acc[s][t] + part[s][t] : part[s][t];
    }
    if constexpr (SPLIT) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                c.acc[s][t] += small[s][t];
    }
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

// f(i, j, value, mirror) over the workgroup's elements
template <typename F>
__device__ __forceinline__ void each(const Part& c, F f)
{
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                f(c.row + 16 * s + q, c.col + 16 * t, c.acc[s][t][q]);
}

template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void gram_kernel(OrthParams p)
{
    uint32_t ti, tj;
    lower_tile(blockIdx.x, ti, tj);
    const uint64_t x = static_cast<uint64_t>(blockIdx.y) * p.mp * p.np, o = static_cast<uint64_t>(blockIdx.y) * p.mp * p.mp;
    Part c;
    products<SPLIT>(c, p.s.x + x, p.s.x_lo + x, p.s.x + x, p.s.x_lo + x, p.np, p.np, p.np, ti * 64, tj * 64);
    each(c, [&](uint32_t i, uint32_t j, float v) {
        if (i == j) {
            p.s.d[blockIdx.y * p.mp + i] = v * (1.0f / (kScaleX * kScaleX));
            v = 0.0f;
        }
        _Float16 hi, lo;
        split(v * (kScaleA / (kScaleX * kScaleX)), hi, lo);
        const uint64_t at = o + static_cast<uint64_t>(i) * p.mp + j, mirror = o + static_cast<uint64_t>(j) * p.mp + i;
        p.s.o[at] = hi;
        if (ti != tj)
            p.s.o[mirror] = hi;
        if constexpr (SPLIT) {
            p.s.o_lo[at] = lo;
            if (ti != tj)
                p.s.o_lo[mirror] = lo;
        }
    });
}

template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void square_kernel(OrthParams p)
{
    uint32_t ti, tj;
    lower_tile(blockIdx.x, ti, tj);
    const uint64_t o = static_cast<uint64_t>(blockIdx.y) * p.mp * p.mp;
    const float* d = p.s.d + blockIdx.y * p.mp;
    Part c;
    products<SPLIT>(c, p.s.o + o, p.s.o_lo + o, p.s.o + o, p.s.o_lo + o, p.mp, p.mp, p.mp, ti * 64, tj * 64);
    each(c, [&](uint32_t i, uint32_t j, float v) {
        const uint64_t at = o + static_cast<uint64_t>(i) * p.mp + j, mirror = o + static_cast<uint64_t>(j) * p.mp + i;
        v *= 1.0f / (kScaleA * kScaleA);
        if (i == j) {
            p.s.d_b[blockIdx.y * p.mp + i] = p.a + p.b * d[i] + p.c * (d[i] * d[i] + v);
            v = 0.0f;
        } else {
            float e = static_cast<float>(p.s.o[at]);
            if constexpr (SPLIT)
                e += static_cast<float>(p.s.o_lo[at]);
            e *= 1.0f / kScaleA;
            v = p.b * e + p.c * (v + (d[i] + d[j]) * e);
        }
        _Float16 hi, lo;
        split(v * kScaleB, hi, lo);
        p.s.b[at] = hi;
        if (ti != tj)
            p.s.b[mirror] = hi;
        if constexpr (SPLIT) {
            p.s.b_lo[at] = lo;
            if (ti != tj)
                p.s.b_lo[mirror] = lo;
        }
    });
}

template <bool SPLIT>
__global__ __launch_bounds__(kThreads) void step_kernel(OrthParams p)
{
    const uint32_t b = blockIdx.z;
    const uint64_t x = static_cast<uint64_t>(b) * p.mp * p.np, o = static_cast<uint64_t>(b) * p.mp * p.mp;
    Part c;
    products<SPLIT>(c, p.s.b + o, p.s.b_lo + o, p.s.xt + x, p.s.xt_lo + x, p.mp, p.mp, p.mp, blockIdx.y * 64,
                    blockIdx.x * 64);
    each(c, [&](uint32_t i, uint32_t j, float v) {
        const uint64_t at = x + static_cast<uint64_t>(i) * p.np + j;
        const float old = SPLIT ? p.s.x_full[at] : static_cast<float>(p.s.x[at]) + static_cast<float>(p.s.x_lo[at]);
        v = __builtin_fmaf(p.s.d_b[b * p.mp + i], old, v * (1.0f / kScaleB));
        if (p.last) {
            if (i < static_cast<uint32_t>(p.m) && j < static_cast<uint32_t>(p.n))
                store_any(p.out, b * p.out_batch + i * p.out_row + j * p.out_col, v * (1.0f / kScaleX), p.out_dtype);
            return;
        }
        _Float16 hi, lo;
        split(v, hi, lo);
        p.s.x[at] = hi;
        p.s.x_lo[at] = lo;
        if constexpr (SPLIT)
            p.s.x_full[at] = v;
        const uint64_t to = x + static_cast<uint64_t>(j) * p.mp + i;
        p.s.xt_to[to] = hi;
        if constexpr (SPLIT)
            p.s.xt_to_lo[to] = lo;
    });
}

// ---- layout and launches

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

size_t layout(int32_t batch, int32_t rows, int32_t cols, bool split_all, char* base, Scratch* s)
{
    const size_t m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
    const size_t mp = (m + kPad - 1) / kPad * kPad, np = (n + kPad - 1) / kPad * kPad;
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
    t.x_lo = halves(mp * np, true);
    t.x_full = split_all ? reinterpret_cast<float*>(take(4 * mp * np)) : nullptr;
    t.xt = halves(mp * np, true);
    t.xt_to = halves(mp * np, true);
    t.xt_lo = halves(mp * np, split_all);
    t.xt_to_lo = halves(mp * np, split_all);
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

template <bool SPLIT>
hipError_t run_steps(OrthParams p, int32_t batch, int32_t steps, hipStream_t stream)
{
    const uint32_t tm = p.mp / 64, tn = p.np / 64;
    const uint32_t lower = tm * (tm + 1) / 2;
    for (int32_t k = 0; k < steps; ++k) {
        p.last = k + 1 == steps;
        gram_kernel<SPLIT><<<dim3(lower, batch), kThreads, 0, stream>>>(p);
        square_kernel<SPLIT><<<dim3(lower, batch), kThreads, 0, stream>>>(p);
        step_kernel<SPLIT><<<dim3(tn, tm, batch), kThreads, 0, stream>>>(p);
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
    p.mp = (p.m + kPad - 1) / kPad * kPad;
    p.np = (p.n + kPad - 1) / kPad * kPad;
    p.in_dtype = updates.dtype;
    p.out_dtype = out.dtype;
    p.a = coefficients[0];
    p.b = coefficients[1];
    p.c = coefficients[2];
    p.eps = eps;
    p.last = 0;
    norm_kernel<<<dim3(kNormBlocks, updates.batch), kThreads, 0, stream>>>(p);
    start_kernel<<<dim3(p.np / 64, p.mp / 64, updates.batch), kThreads, 0, stream>>>(p);
    if (steps == 0) {
        emit_kernel<<<dim3(1, p.m, updates.batch), kThreads, 0, stream>>>(p);
        return hipGetLastError();
    }
    return split_all ? run_steps<true>(p, updates.batch, steps, stream)
                     : run_steps<false>(p, updates.batch, steps, stream);
}

}  // namespace sqn
