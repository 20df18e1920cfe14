// A layer while it is trained and asked, and its gradient:
//
//   z = x w^T + b,  y = D(act(z)) + residual
//   dz = D(dy) act'(z),  dx = dz w,  dw = dz^T x,  db = sum of dz's rows
//
// All three products are C = P Q^T, stored with the rows of P along the memory of
// C's rows: P = w, Q = x;  P = w^T, Q = dz;  P = x^T, Q = dz^T.  A factor whose
// rows are contiguous along the sum ("along") or across it ("across") is read as
// it lies in memory: the tiles of tile.h, whose steps bring 128 bytes of the sum
// of every row, or as many elements of the sum across, and the LDS reads that
// turn 16-bit elements on their way to the registers.  Nothing is transposed in
// memory.  Three kernels share the work: tiles; narrow layers of many points, whose
// bytes are all that counts, with their weights in registers; and layers of few
// points, with nothing but the weights' bytes.  Which, goes by sizes and alignment
// (plan_of, layer_plan, GradientPlan, narrow_of, launch_layer_typed).
//
// Rounding.  Sums and epilogues are binary32.  Matrix instructions take dz in 16 bits
// beside 16-bit factors: as it is where it is grad's own values and zeros, else in two
// parts (terms_of), so that a gradient's error is that of its own rounding.  The mask's
// share is applied to the sums, before which dz stays in grad's range.  The bias's sums
// take it in binary32.
#include <math.h>
#include <algorithm>
#include <type_traits>

#include "learn.h"
#include "mask.h"
#include "numeric.h"
#include "sqn_internal.h"
#include "tile.h"

namespace sqn {
namespace {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kThreads = 256;

// ---- what a product's sums go through on their way out

struct Finish {
    const void* bias;            // [units] or null
    const void* residual;        // of the output's type, or null
    void* pre;                   // z of the factors' type, or null
    void* out;
    int64_t residual_stride, pre_stride, out_stride;      // elements
    uint32_t bias_f32, act, units;
    float scale;                 // of a gradient's product
    Mask mask;
};

// The normal distribution: its share Phi below z, and exp(-z^2 / 2).
//
// Phi(-a) = exp(-a^2 / 2) q(a) for a >= 0, and t = 1 / (1 + 0.35 a) takes q to the
// whole of (0, 1]: a polynomial of degree 9 in t, fitted for the least relative
// error (3.2e-8), so that the values far below zero keep their digits.  22 operations
// a value, with the exponential that the slope shares (erfcf and expf take some 80: 8192
// x 8192 outputs with a mask and z kept took 691 us of a layer, with the loads of the
// bias that left with them 545).  With binary32's roundings Phi is off by 5e-7 and
// 5e-8 z^2 of itself, the latter from the exponent's: less than a hundredth of half a
// step of the 16-bit values that are made of it.
//
// FINE, for values of binary32: the exponent and t keep their low parts, and below
// |z| = 1 Phi is 1/2 + z p(z^2), p of degree 6: z Phi is off by 3.0e-7 of itself at most
// for -12 < z < 12 (7.3e-6 without), its slope by 2.0e-7 of what it is the sum of (7.1e-6).
// Some 40 operations: 50,001 points of 42 by 256 with z kept 45 us, 37 without.
template <bool FINE>
__device__ __forceinline__ float normal_share(float z, float& bell)
{
    constexpr float kHalf = -0.72134752f, kHalfLow = -9.6298149e-09f;    // -1 / (2 ln 2)
    float a = fabsf(z);
    if constexpr (FINE) {
        a = fminf(a, 64.0f);     // whose exponential is 0
        const float square = a * a, exponent = square * kHalf;
        const float low = __builtin_fmaf(__builtin_fmaf(a, a, -square), kHalf,
                                         __builtin_fmaf(square, kHalfLow, __builtin_fmaf(square, kHalf, -exponent)));
        bell = __builtin_amdgcn_exp2f(exponent);
        bell = __builtin_fmaf(bell, low * 0.69314718f, bell);
    } else {
        bell = __builtin_amdgcn_exp2f(z * z * kHalf);
    }
    const float below = __builtin_fmaf(0.35f, a, 1.0f);
    float t = __builtin_amdgcn_rcpf(below);
    if constexpr (FINE) {
        const float lost = __builtin_fmaf(0.35f, a, 1.0f - below);
        t = __builtin_fmaf(__builtin_fmaf(-lost, t, __builtin_fmaf(-below, t, 1.0f)), t, t);
    }
    float q = -0.029125869f;
    q = __builtin_fmaf(q, t, 0.14387225f);
    q = __builtin_fmaf(q, t, -0.25550461f);
    q = __builtin_fmaf(q, t, 0.15892933f);
    q = __builtin_fmaf(q, t, -0.022937165f);
    q = __builtin_fmaf(q, t, 0.10543295f);
    q = __builtin_fmaf(q, t, 0.11985243f);
    q = __builtin_fmaf(q, t, 0.13985908f);
    q = __builtin_fmaf(q, t, 0.13962157f);
    q *= t * bell;
    const float share = z < 0.0f ? q : 1.0f - q;
    if constexpr (FINE) {
        const float square = a * a;
        float p = 5.373781e-07f;
        p = __builtin_fmaf(p, square, -9.274743e-06f);
        p = __builtin_fmaf(p, square, 0.000115321134f);
        p = __builtin_fmaf(p, square, -0.0011872889f);
        p = __builtin_fmaf(p, square, 0.00997355f);
        p = __builtin_fmaf(p, square, -0.06649038f);
        p = __builtin_fmaf(p, square, 0.3989423f);
        return a < 1.0f ? __builtin_fmaf(z, p, 0.5f) : share;
    }
    return share;
}

// 1 / (1 + exp(-z)), off by 3e-7 and 6e-8 |z| of itself; FINE, z times it by 2.2e-7.
template <bool FINE>
__device__ __forceinline__ float logistic(float z)
{
    constexpr float kLog = -1.442695f, kLogLow = -1.9259630e-08f;    // -1 / ln 2
    if constexpr (FINE) {
        const float near = __builtin_amdgcn_fmed3f(z, -128.0f, 128.0f);     // infinity and 0 beyond
        const float exponent = near * kLog;
        const float low = __builtin_fmaf(near, kLogLow, __builtin_fmaf(near, kLog, -exponent));
        return 1.0f / __builtin_fmaf(__builtin_amdgcn_exp2f(exponent), __builtin_fmaf(low, 0.69314718f, 1.0f), 1.0f);
    } else {
        return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * kLog));
    }
}

// The choice stands outside the loops over a run, whose values then go through
// the long chains side by side.
template <bool FINE, int V>
__device__ __forceinline__ void activate(uint32_t act, float (&v)[V])
{
    float bell;
    if (act == SQN_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] = v[k] < 0.0f ? 0.0f : v[k];
    } else if (act == SQN_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] *= normal_share<FINE>(v[k], bell);
    } else if (act == SQN_ACT_SILU) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] *= logistic<FINE>(v[k]);
    }
}

// v times the activation's slopes at z.
template <bool FINE, int V>
__device__ __forceinline__ void times_slope(uint32_t act, const float (&z)[V], float (&v)[V])
{
    if (act == SQN_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] = z[k] <= 0.0f ? 0.0f : v[k];
    } else if (act == SQN_ACT_GELU) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float bell;
            const float share = normal_share<FINE>(z[k], bell);
            v[k] *= __builtin_fmaf(z[k] * 0.39894228f, bell, share);
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float s = logistic<FINE>(z[k]);
            v[k] *= s * __builtin_fmaf(z[k], 1.0f - s, 1.0f);
        }
    }
}

// The ragged run's address by an offset of zero that the compiler does not know: its
// accesses were merged with the whole run's where they share one, and a store of 16
// bytes went out as two of 4 and one of 8, or as two of 2 and one of 12.
template <typename T>
__device__ __forceinline__ T* ragged(T* p)
{
    uint32_t zero = 0;
    asm("" : "+v"(zero));
    return p + zero;
}

// A run of V elements of which `left` are inside the row.
template <typename T, int V>
__device__ __forceinline__ void load_inside(const T* p, uint32_t left, float (&v)[V])
{
    if (left >= V) {
        load_run<T, V>(p, v);
    } else {
        const T* q = ragged(p);
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] = k < static_cast<int>(left) ? to_f32(q[k]) : 0.0f;
    }
}

template <typename T, int V>
__device__ __forceinline__ void store_values(T* p, uint32_t left, const float (&v)[V])
{
    if (left >= V) {
        store_run<T, V>(p, v);
    } else {
        T* q = ragged(p);
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k < static_cast<int>(left))
                q[k] = from_f32<T>(v[k]);
    }
}

// A run as it is loaded, turned into values later, so that many are under way
// together.
template <typename T, int V>
struct Raw {
    T e[V];

    __device__ __forceinline__ void load(const T* p, uint32_t left)
    {
        if (left >= V) {
            const Run<T, V> r = *reinterpret_cast<const Run<T, V>*>(p);
            __builtin_memcpy(e, &r, sizeof(e));
        } else {
            const T* q = ragged(p);
#pragma unroll
            for (int k = 0; k < V; ++k)
                e[k] = k < static_cast<int>(left) ? q[k] : T(0.0f);
        }
    }
};

// The bias of units unit..unit + V, zeros of none.
template <typename X, int V>
__device__ __forceinline__ void load_bias(const Finish& f, uint32_t unit, float (&b)[V])
{
    const uint32_t left = f.units - min(unit, f.units);
#pragma unroll
    for (int k = 0; k < V; ++k)
        b[k] = 0.0f;
    if (f.bias && left) {
        if (f.bias_f32)
            load_inside<float, V>(static_cast<const float*>(f.bias) + unit, left, b);
        else
            load_inside<X, V>(static_cast<const X*>(f.bias) + unit, left, b);
    }
}

template <typename T, int V>
__device__ __forceinline__ void load_residual(const Finish& f, uint64_t row, uint32_t unit, Raw<T, V>& r)
{
    if (f.residual)
        r.load(static_cast<const T*>(f.residual) + row * f.residual_stride + unit, f.units - unit);
}

// Elements unit..unit + V of row `row` of an output of type T, from factors of
// type X; all of a layer's epilogue, or a gradient's scale.
template <typename X, typename T, bool LAYER, int V>
__device__ __forceinline__ void finish(const Finish& f, uint64_t key, uint64_t row, uint32_t unit, const float (&bias)[V],
                                       const Raw<T, V>& residual, float (&v)[V])
{
    const uint32_t left = f.units - unit;
    if constexpr (LAYER) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] += bias[k];
        if (f.pre)
            store_values<X, V>(static_cast<X*>(f.pre) + row * f.pre_stride + unit, left, v);
        activate<sizeof(T) == 4, V>(f.act, v);
        if (f.mask.on)
            apply_mask<V>(f.mask, key, row, unit, f.mask.scale, v);
        if (f.residual)
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] += to_f32(residual.e[k]);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            v[k] *= f.scale;
    }
    store_values<T, V>(static_cast<T*>(f.out) + row * f.out_stride + unit, left, v);
}

// ---- factors

struct Operand {
    const char* data;            // 16-byte aligned
    uint64_t pitch;              // bytes from row to row in memory, a multiple of 16
    uint32_t rows;               // of the factor: along, rows in memory; across, elements of one, in whole 16 bytes
    uint32_t valid;              // of the sum: along, bytes of a row, whole 16; across, rows in memory
    uint64_t apart;              // bytes from the high parts of the elements to their low ones
    uint32_t low;                // bit t: term t of the product takes the low parts
};

// A product of factors in parts: every step of the sum comes once for each term,
// whose parts the operands name.  Terms of a step follow each other, so that what
// they share is in the caches.
struct Terms {
    uint32_t count, inverse, whole;      // 2^32 / count rounded up, 0 of one; 1 of one

    Terms(uint32_t n = 1) : count(n), inverse(n == 1 ? 0 : n == 2 ? 0x80000000u : 0x55555556u), whole(n == 1) {}

    // the step that step k of all is a term of: exact below 2^31
    __device__ __forceinline__ uint32_t step(uint32_t k) const { return __umulhi(k, inverse) + k * whole; }
};

template <typename X>
struct Elements {
    static constexpr uint32_t STEP = kStepBytes / sizeof(X);     // of the sum
    static constexpr uint32_t PIECE = kSlot / sizeof(X);
};

// The slots of a row of an across factor in LDS are permuted by its place in the
// step, so that the lanes that LDS serves together reach all banks once: 16
// lanes of a turning read take four rows, 32 consecutive bytes of each.
template <typename X, int SIDE>
__device__ __forceinline__ uint32_t across_key(uint32_t k)
{
    if constexpr (sizeof(X) == 4)
        return 8 * (k >> 4 & 1);
    else
        return SIDE >= 128 ? 4 * (k & 3) : 4 * (k >> 1 & 1);
}

// What a lane brings of a factor's steps, through a buffer descriptor of the
// tile's rows: pieces past the sum's end lie past the descriptor's, and come as
// zeros without an access.  PARTED: of a product in terms, whose few scalar operations
// a step took tiles of 64 a tenth of their time (65,536 points of 256 by 256 in
// binary16, dw 21.5 us for 19.3).
template <typename X, int SIDE, int WAVES, bool ACROSS, bool PARTED>
struct Bringer {
    static constexpr int COUNT = SIDE * static_cast<int>(kStepBytes) / (1024 * WAVES);
    static constexpr uint32_t SLOTS = SIDE * sizeof(X) / kSlot;  // of a row across
    static constexpr uint32_t LINES = 64 / (SLOTS < 64 ? SLOTS : 64);            // of an instruction, across
    static constexpr uint32_t OUTSIDE = 0x80000000u;             // a tile's rows span less (in_place)
    const char* from;
    uint32_t at[COUNT], place[ACROSS ? COUNT : 1];
    uint32_t valid;
    uint64_t on;                 // bytes from step to step
    uint64_t apart;              // with PARTED, as the next two
    uint32_t low;
    Terms terms;

    __device__ __forceinline__ Bringer(const Operand& o, uint32_t row0, const Terms& t)
        : apart(o.apart), low(o.low), terms(t)
    {
        const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        valid = o.valid;
        if constexpr (ACROSS) {
            static_assert(SLOTS <= 64, "a row of a step is one instruction's at most");
            from = o.data + static_cast<uint64_t>(row0) * sizeof(X);
            on = o.pitch * Elements<X>::STEP;
            const uint32_t pieces = (o.rows - row0) / Elements<X>::PIECE;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const uint32_t k = (WAVES * i + wave) * LINES + lane / SLOTS;
                const uint32_t piece = lane % SLOTS ^ across_key<X, SIDE>(k);
                place[i] = k;
                at[i] = piece < pieces ? k * static_cast<uint32_t>(o.pitch) + piece * kSlot : OUTSIDE;
            }
        } else {
            from = o.data + row0 * o.pitch;
            on = kStepBytes;
            place[0] = brought_piece(lane, wave) * kSlot;
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const uint32_t row = 8 * (WAVES * i + wave) + (lane >> 3);
                at[i] = row < o.rows - row0 ? row * static_cast<uint32_t>(o.pitch) + place[0] : OUTSIDE;
            }
        }
    }

    // the rows of a step, and how much of the sum is left from it on
    struct Step {
        __amdgpu_buffer_rsrc_t rows;
        uint32_t left;
    };

    __device__ __forceinline__ Step step(uint32_t k) const
    {
        uint64_t part = 0;
        if constexpr (PARTED) {
            const uint32_t term = k;
            k = terms.step(term);
            part = low >> (term - k * terms.count) & 1 ? apart : 0;
        }
        // raw bytes, OUTSIDE of them
        return {__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from + part + k * on), 0, OUTSIDE, 0x00020000),
                valid - k * (ACROSS ? Elements<X>::STEP : kStepBytes)};
    }

    __device__ __forceinline__ void bring(const Step& s, int i, char* to) const
    {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(s.rows, (lds_void*)(to + (WAVES * i + wave) * 1024), kSlot,
                                                 place[ACROSS ? i : 0] < s.left ? at[i] : OUTSIDE, 0, 0, 0);
    }
};

// A lane's 16 bytes of a block of 32 rows at one depth: eight elements of the sum
// (four of binary32) of row lane % 32, places 32 g + 8 o (16 g + 4 o) on, g =
// lane / 32, of the step.
template <typename X, int SIDE, bool ACROSS, int F>
struct Reader {
    uint32_t at[F];

    __device__ __forceinline__ explicit Reader(uint32_t first)
    {
        const uint32_t lane = threadIdx.x & 63, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < F; ++s) {
            const uint32_t row = first + 32 * s;
            if constexpr (!ACROSS) {
                at[s] = row * kStepBytes;
            } else if constexpr (sizeof(X) == 4) {
                const uint32_t r = row + (lane & 31), k = 16 * half;
                at[s] = k * SIDE * 4 + ((r >> 2) ^ across_key<X, SIDE>(k)) * kSlot + (r & 3) * 4;
            } else {
                // lane 4 a + b of 16 takes elements 4 b .. 4 b + 3 of row a, and gets
                // element 4 a + b of the four rows
                const uint32_t k = 32 * half + (lane >> 2 & 3);
                const uint32_t piece = row / 8 + 2 * (lane >> 4 & 1) + (lane >> 1 & 1);
                at[s] = k * SIDE * 2 + (piece ^ across_key<X, SIDE>(k)) * kSlot + (lane & 1) * 8;
            }
        }
    }

    // block s at depth o
    __device__ __forceinline__ uint4 read(const char* buffer, int s, uint32_t o) const
    {
        uint4 f;
        if constexpr (!ACROSS) {
            f = *reinterpret_cast<const uint4*>(buffer + at[s] + piece_at(threadIdx.x & 63, o));
        } else if constexpr (sizeof(X) == 4) {
            const char* p = buffer + at[s] + 4 * o * SIDE * 4;
            auto word = [&](int k) { return *reinterpret_cast<const uint32_t*>(p + k * SIDE * 4); };
            f = uint4{word(0), word(1), word(2), word(3)};
        } else {
            // places 8 o and 8 o + 4 on: rows a of each four keep their key
            const char* p = buffer + at[s] + 8 * o * SIDE * 2;
            short4v e[2];
#pragma unroll
            for (int k = 0; k < 2; ++k)
                e[k] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4*)(p + 4 * k * SIDE * 2));
            __builtin_memcpy(&f, e, 16);
        }
        return f;
    }
};

// Element `e` of binary32 pieces, whose instructions take one of a lane; all of
// 16-bit ones.
template <typename X>
__device__ __forceinline__ float16v multiply(const uint4& a, const uint4& b, int e, float16v acc)
{
    if constexpr (sizeof(X) == 4) {
        float4v u, v;
        __builtin_memcpy(&u, &a, 16);
        __builtin_memcpy(&v, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], v[e], acc, 0, 0, 0);
    } else if constexpr (std::is_same_v<X, __bf16>) {
        bhalf8 u, v;
        __builtin_memcpy(&u, &a, 16);
        __builtin_memcpy(&v, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(u, v, acc, 0, 0, 0);
    } else {
        half8 u, v;
        __builtin_memcpy(&u, &a, 16);
        __builtin_memcpy(&v, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(u, v, acc, 0, 0, 0);
    }
}

// ---- tiles

// A workgroup's tile: SIDE x SIDE of C by 2 x 2 waves.  The wide accumulators of
// the largest tile (128 x 128 a wave, one wave a SIMD) spare LDS: of the 128 bytes a
// cycle it moves, reads and loads take 96 beside matrix cores that never wait; with
// eight waves of 128 x 64 they would take all, in tiles of 128 they would take 192.
template <int SIDE_>
struct Shape {
    static constexpr int SIDE = SIDE_;
    static constexpr int WAVES = 4, THREADS = 64 * WAVES;
    static constexpr int F = SIDE / 64;                          // blocks of a wave, either way
    static constexpr int ROWS = SIDE * static_cast<int>(kStepBytes);
    static constexpr int BUFFER = 2 * ROWS;
    static constexpr int LOADS = BUFFER / (1024 * WAVES);
    static constexpr int BUFFERS = SIDE == 64 ? 4 : 2;
    static constexpr int PER_SIMD = SIDE == 256 ? 1 : 2;         // waves
};

struct ProductParams {
    Operand p, q;
    uint32_t rows;               // of C
    uint32_t tiles_p, tiles_q;   // of C
    uint32_t steps, part_steps;  // of the sum, all terms of it, and of a part of it
    Terms terms;
    uint32_t parts;              // 1: the sums are finished here
    float* partial;              // [parts][rows][partial_pitch]
    uint32_t partial_pitch;
    Finish f;
};

template <typename S>
struct Fragments {
    uint4 f[2 * S::F];           // of P, then of Q
};

// The steps of a tile's sum, in the order of tile.h's, with every instruction in
// its place: behind each product stand a share of the next depth's reads and,
// at a step's last depth, of the loads into the buffer that it leaves.  With one
// wave a SIMD whatever stands in a block of its own leaves the matrix cores idle
// (the compiler's order: 1,040 TFLOP/s of 8192 x 8192 by 4096 in bfloat16).
// (T, the output's type, is here for the host's pass, which has none of the builtins
// and takes a function whose body it could not read only once.)
template <typename S, typename X, typename T, typename BP, typename BQ, typename RP, typename RQ>
__device__ __forceinline__ void sum_steps(const BP& bring_p, const BQ& bring_q, const RP& read_p, const RQ& read_q, uint32_t first,
                                          uint32_t steps, char* (&buffers)[S::BUFFERS], float16v (&acc)[S::F][S::F])
{
    constexpr int F = S::F, BUFFERS = S::BUFFERS, LOADS = S::LOADS;
    constexpr int PRODUCTS = F * F * (sizeof(X) == 4 ? 4 : 1);   // of a depth
    const uint32_t end = first + steps - 1;
    Fragments<S> f0, f1;
    auto read_block = [&](Fragments<S>& f, const char* buffer, int k, uint32_t o) {
        f.f[k] = k < F ? read_p.read(buffer, k, o) : read_q.read(buffer + S::ROWS, k - F, o);
    };
    auto bring = [&](const typename BP::Step& p, const typename BQ::Step& q, int i, char* buffer) {
        if (i < BP::COUNT)
            bring_p.bring(p, i, buffer);
        else
            bring_q.bring(q, i - BP::COUNT, buffer + S::ROWS);
    };
    // the products of a depth; `next` of `from` at depth o is read behind them, and
    // with LOAD step k comes into `to`
    auto depth = [&](const Fragments<S>& f, Fragments<S>& next, const char* from, uint32_t o, auto load, uint32_t k, char* to) {
        constexpr bool LOAD = decltype(load)::value;
        const auto step_p = bring_p.step(k);
        const auto step_q = bring_q.step(k);
        int reads = 0, loads = 0;
#pragma unroll
        for (int m = 0; m < PRODUCTS; ++m) {
            const int s = m / F % F, t = m % F;
            acc[s][t] = multiply<X>(f.f[s], f.f[F + t], m / (F * F), acc[s][t]);
            // the reads are done by the middle of the depth
#pragma unroll
            for (; reads < 2 * F && reads * PRODUCTS < (m + 1) * 4 * F; ++reads)
                read_block(next, from, reads, o);
            if constexpr (LOAD) {
#pragma unroll
                for (; loads * PRODUCTS < (m + 1) * LOADS; ++loads)
                    bring(step_p, step_q, loads, to);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
#pragma unroll
    for (int b = 0; b < BUFFERS; ++b) {
        const uint32_t k = min(first + b, end);
        const auto step_p = bring_p.step(k);
        const auto step_q = bring_q.step(k);
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            bring(step_p, step_q, i, buffers[b]);
    }
    landed<(BUFFERS - 1) * LOADS>();
#pragma unroll
    for (int k = 0; k < 2 * F; ++k)
        read_block(f0, buffers[0], k, 0);
    constexpr std::false_type no{};
    constexpr std::true_type yes{};
    // buffer b holds step k and will hold k + BUFFERS; past the end the last step
    // comes once more and is not used
    auto work = [&](uint32_t k, int b) {
        depth(f0, f1, buffers[b], 1, no, 0, nullptr);
        depth(f1, f0, buffers[b], 2, no, 0, nullptr);
        depth(f0, f1, buffers[b], 3, no, 0, nullptr);
        landed<(BUFFERS - 2) * LOADS>();
        depth(f1, f0, buffers[(b + 1) % BUFFERS], 0, yes, min(k + BUFFERS, end), buffers[b]);
    };
    uint32_t k = first;
    for (; k + BUFFERS <= end + 1; k += BUFFERS) {
#pragma unroll
        for (int b = 0; b < BUFFERS; ++b)
            work(k + b, b);
    }
#pragma unroll
    for (int b = 0; b < BUFFERS - 1; ++b)
        if (k + b <= end)
            work(k + b, b);
    // the loads still under way end before their buffers do
    landed<0>();
}

// Workgroups that follow each other go to the eight XCDs in turn: each takes a
// run of the parts' tiles, in columns of 8 tiles of Q, so that what its CUs work
// on at a time shares rows of both factors in the XCD's cache.
__device__ __forceinline__ void tile_of(uint32_t group, uint32_t groups, uint32_t tiles_p, uint32_t tiles_q, uint32_t& part,
                                        uint32_t& tp, uint32_t& tq)
{
    constexpr uint32_t kXcds = 8, kBand = 8;
    const uint32_t each = groups / kXcds, more = groups % kXcds;
    const uint32_t xcd = group % kXcds, nth = group / kXcds;
    const uint32_t all = xcd * each + min(xcd, more) + nth;
    part = all / (tiles_p * tiles_q);
    const uint32_t t = all - part * tiles_p * tiles_q;
    const uint32_t band = t / (kBand * tiles_p), in_band = t - band * kBand * tiles_p;
    const uint32_t width = min(kBand, tiles_q - band * kBand);
    tp = in_band / width;
    tq = band * kBand + in_band - tp * width;
}

template <typename S, typename X, typename T, bool LAYER, bool PA, bool QA, bool PARTED>
__device__ __forceinline__ void tile_share(const ProductParams& p, uint32_t group, uint32_t groups, char* (&buffers)[S::BUFFERS])
{
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t part, tp, tq;
    tile_of(group, groups, p.tiles_p, p.tiles_q, part, tp, tq);
    const uint32_t p0 = tp * S::SIDE, q0 = tq * S::SIDE;
    const Bringer<X, S::SIDE, S::WAVES, PA, PARTED> bring_p(p.p, p0, p.terms);
    const Bringer<X, S::SIDE, S::WAVES, QA, PARTED> bring_q(p.q, q0, p.terms);
    const uint32_t wave_p = (wave & 1) * (S::SIDE / 2), wave_q = (wave >> 1) * (S::SIDE / 2);
    const Reader<X, S::SIDE, PA, S::F> read_p(wave_p);
    const Reader<X, S::SIDE, QA, S::F> read_q(wave_q);
    // a lane's units of the output, and how many rows a wave finishes at once
    constexpr int V = 16 / sizeof(T);
    constexpr uint32_t RUNS = S::F * 32 / V, ROUNDS = RUNS / 2, TOGETHER = ROUNDS < 4 ? ROUNDS : 4;
    const uint32_t unit = p0 + wave_p + V * (lane % RUNS);
    float bias[V];
    if constexpr (LAYER)
        load_bias<X, V>(p.f, unit, bias);
    float16v acc[S::F][S::F];
#pragma unroll
    for (int s = 0; s < S::F; ++s)
#pragma unroll
        for (int t = 0; t < S::F; ++t)
            acc[s][t] = float16v{};
    const uint32_t first = part * p.part_steps, count = min(p.part_steps, p.steps - first);
    sum_steps<S, X, T>(bring_p, bring_q, read_p, read_q, first, count, buffers, acc);
    // out through LDS in binary32, a column of blocks at a time, so that a lane
    // finishes runs of rows, always of the same units
    constexpr uint32_t PITCH = S::F * 32 * 4, PIECES = PITCH / 16;
    char* own = own_part<S::F, S::BUFFER>(buffers[0], buffers[1], wave);
    const uint32_t half = lane >> 5, mine = lane & 31;
    const uint64_t key = LAYER && p.f.mask.on ? mask_key(p.f.mask) : 0;
    auto slot = [](uint32_t column, uint32_t piece) { return column * PITCH + (piece ^ (column & (PIECES - 1))) * 16; };
#pragma unroll
    for (int t = 0; t < S::F; ++t) {
        const uint32_t row0 = q0 + wave_q + 32 * t + lane / RUNS;
#pragma unroll
        for (int s = 0; s < S::F; ++s)
#pragma unroll
            for (uint32_t g = 0; g < 4; ++g)
                *reinterpret_cast<float4v*>(own + slot(mine, 8 * s + 2 * g + half))
                    = float4v{acc[s][t][4 * g], acc[s][t][4 * g + 1], acc[s][t][4 * g + 2], acc[s][t][4 * g + 3]};
        wave_fence();
        if (p.parts > 1) {
#pragma unroll 2
            for (uint32_t i = 0; i < PIECES / 2; ++i) {
                const uint32_t column = (64 * i + lane) / PIECES, piece = lane & (PIECES - 1);
                const uint32_t row = q0 + wave_q + 32 * t + column, at = p0 + wave_p + 4 * piece;
                if (row < p.rows && at < p.partial_pitch)
                    *reinterpret_cast<float4v*>(p.partial + (static_cast<uint64_t>(part) * p.rows + row) * p.partial_pitch + at)
                        = *reinterpret_cast<const float4v*>(own + slot(column, piece));
            }
        } else {
#pragma unroll 1
            for (uint32_t i0 = 0; i0 < ROUNDS; i0 += TOGETHER) {
                Raw<T, V> residual[TOGETHER];
                if constexpr (LAYER)
#pragma unroll
                    for (uint32_t i = 0; i < TOGETHER; ++i)
                        if (row0 + (i0 + i) * (64 / RUNS) < p.rows && unit < p.f.units)
                            load_residual<T, V>(p.f, row0 + (i0 + i) * (64 / RUNS), unit, residual[i]);
#pragma unroll
                for (uint32_t i = 0; i < TOGETHER; ++i) {
                    const uint32_t row = row0 + (i0 + i) * (64 / RUNS), column = (64 * (i0 + i) + lane) / RUNS;
                    float v[V];
#pragma unroll
                    for (int k = 0; k < V / 4; ++k) {
                        const float4v e = *reinterpret_cast<const float4v*>(own + slot(column, V / 4 * (lane % RUNS) + k));
                        __builtin_memcpy(v + 4 * k, &e, 16);
                    }
                    if (row < p.rows && unit < p.f.units)
                        finish<X, T, LAYER, V>(p.f, key, row, unit, bias, residual[i], v);
                }
            }
        }
        wave_fence();
    }
}

template <typename S, typename X, typename T, bool LAYER, bool PA, bool QA, bool PARTED>
__global__ __launch_bounds__(S::THREADS, S::PER_SIMD) void tile_kernel(ProductParams p)
{
    BUFFERS_IN_LDS(S)
    tile_share<S, X, T, LAYER, PA, QA, PARTED>(p, blockIdx.x, gridDim.x, buffers);
}

// Both products of a gradient side by side, the points' first.
template <typename S, typename X, typename T, bool PARTED>
__global__ __launch_bounds__(S::THREADS, S::PER_SIMD) void pair_kernel(ProductParams x, ProductParams w, uint32_t groups_x)
{
    BUFFERS_IN_LDS(S)
    if (blockIdx.x < groups_x)
        tile_share<S, X, T, false, true, false, PARTED>(x, blockIdx.x, groups_x, buffers);
    else
        tile_share<S, X, T, false, true, true, PARTED>(w, blockIdx.x - groups_x, gridDim.x - groups_x, buffers);
}

// The parts of the sums added up, in their order, and finished; zeros of no parts.
// The threads of a run (a power of two, more where there are many parts of few
// runs) take every slices-th part, so that their loads are under way together.
struct PartsParams {
    const float* partial;
    uint64_t rows, runs;         // runs: rows * per_row
    uint32_t parts, pitch, per_row;
    uint32_t slices;
    Finish f;
};

template <typename X, typename T, bool LAYER>
__device__ __forceinline__ void parts_share(const PartsParams& p, uint32_t group, uint32_t groups)
{
    constexpr int V = 4;
    __shared__ float4v shared[kThreads];
    const uint64_t key = LAYER && p.f.mask.on ? mask_key(p.f.mask) : 0;
    const uint32_t width = kThreads / p.slices, tx = threadIdx.x % width, ty = threadIdx.x / width;
    for (uint64_t first = static_cast<uint64_t>(group) * width; first < p.runs; first += static_cast<uint64_t>(groups) * width) {
        const uint64_t i = first + tx;
        const bool inside = i < p.runs;
        const uint64_t row = inside ? i / p.per_row : 0;
        const uint32_t unit = inside ? static_cast<uint32_t>(i - row * p.per_row) * V : 0;
        float bias[V];
        Raw<T, V> residual;
        if (LAYER && inside && ty == 0) {
            load_bias<X, V>(p.f, unit, bias);
            load_residual<T, V>(p.f, row, unit, residual);
        }
        float4v total = {};
        if (inside) {
#pragma unroll 8
            for (uint32_t k = ty; k < p.parts; k += p.slices)
                total += *reinterpret_cast<const float4v*>(p.partial + (k * p.rows + row) * p.pitch + unit);
        }
        if (p.slices > 1) {
            __syncthreads();
            shared[threadIdx.x] = total;
            __syncthreads();
            if (ty == 0)
                for (uint32_t k = 1; k < p.slices; ++k)
                    total += shared[k * width + tx];
        }
        if (inside && ty == 0) {
            float v[V];
            __builtin_memcpy(v, &total, 16);
            finish<X, T, LAYER, V>(p.f, key, row, unit, bias, residual, v);
        }
    }
}

template <typename X, typename T>
__global__ __launch_bounds__(kThreads) void parts_kernel(PartsParams p)
{
    parts_share<X, T, true>(p, blockIdx.x, gridDim.x);
}

// ---- layers of few points
//
// For one token's points the weights' bytes are all that takes time.  A
// workgroup computes 16 units of all points, or 64 where there are many units (its
// waves read the points' elements once for each: 16 points of 4096 by 16,384 in
// bfloat16 29 us, 43 with 16 units; one of 4096 by 4096 8, 17 with 64), on the
// 16 x 16 instructions; its waves take the sum's pieces in turn, straight from memory to
// registers at any alignment, and add up in LDS, in the order of the waves.

constexpr int kFewPoints = 16, kFewWaves = 8;

struct FewParams {
    const void *x, *w;
    int64_t x_stride, w_stride;  // elements
    uint32_t points, cols;
    Finish f;
};

// A lane's elements of an instruction's 16 rows: 16 bytes of row lane % 16, those
// of piece lane / 16 of four.
template <typename X>
struct Sixteen {
    static constexpr uint32_t N = 16 / sizeof(X), ALL = 4 * N;

    static __device__ __forceinline__ uint4 whole(const X* p)
    {
        const Run<X, N> r = *reinterpret_cast<const Run<X, N>*>(p);
        uint4 v;
        __builtin_memcpy(&v, &r, 16);
        return v;
    }

    static __device__ __forceinline__ uint4 ragged(const X* p, uint32_t left)
    {
        X e[N];
#pragma unroll
        for (uint32_t k = 0; k < N; ++k)
            e[k] = k < left ? p[k] : X(0.0f);
        uint4 v;
        __builtin_memcpy(&v, e, 16);
        return v;
    }

    static __device__ __forceinline__ float4v multiply(const uint4& a, const uint4& b, float4v acc)
    {
        if constexpr (sizeof(X) == 4) {
            float4v u, v;
            __builtin_memcpy(&u, &a, 16);
            __builtin_memcpy(&v, &b, 16);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[k], v[k], acc, 0, 0, 0);
            return acc;
        } else if constexpr (std::is_same_v<X, __bf16>) {
            bhalf8 u, v;
            __builtin_memcpy(&u, &a, 16);
            __builtin_memcpy(&v, &b, 16);
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(u, v, acc, 0, 0, 0);
        } else {
            half8 u, v;
            __builtin_memcpy(&u, &a, 16);
            __builtin_memcpy(&v, &b, 16);
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(u, v, acc, 0, 0, 0);
        }
    }
};

template <typename X, typename T, int BLOCKS>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(FewParams p)
{
    typedef Sixteen<X> S;
    constexpr int UNITS = 16 * BLOCKS, V = 4, TOGETHER = 8 / BLOCKS;
    __shared__ __align__(16) float part[kFewWaves][kFewPoints][UNITS + 4];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const uint32_t unit0 = blockIdx.x * UNITS, mine = lane & 15, at = lane / 16 * S::N;
    // rows past the ends read the last one, and are not stored
    const X* x = static_cast<const X*>(p.x) + min(mine, p.points - 1) * p.x_stride + at;
    const X* w[BLOCKS];
    float4v acc[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        w[b] = static_cast<const X*>(p.w) + min(unit0 + 16 * b + mine, p.f.units - 1) * p.w_stride + at;
        acc[b] = float4v{};
    }
    // two pieces that follow each other, lines of the rows, are one wave's
    const uint32_t full = p.cols / S::ALL;
    uint32_t k = 2 * wave;
    auto piece = [&](int i) { return k + i / 2 * 2 * waves + i % 2; };
    for (; piece(TOGETHER - 1) < full; k += TOGETHER * waves) {
        uint4 of_x[TOGETHER], of_w[TOGETHER][BLOCKS];
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i) {
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                of_w[i][b] = S::whole(w[b] + piece(i) * S::ALL);
            of_x[i] = S::whole(x + piece(i) * S::ALL);
        }
#pragma unroll
        for (int i = 0; i < TOGETHER; ++i)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                acc[b] = S::multiply(of_w[i][b], of_x[i], acc[b]);
    }
    for (; k <= full; k += 2 * waves)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t from = (k + i) * S::ALL;
            if (k + i < full) {
                const uint4 of_x = S::whole(x + from);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    acc[b] = S::multiply(S::whole(w[b] + from), of_x, acc[b]);
            } else if (k + i == full && from < p.cols) {
                const uint32_t left = from + at < p.cols ? p.cols - from - at : 0;
                const uint4 of_x = S::ragged(x + from, left);
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    acc[b] = S::multiply(S::ragged(w[b] + from, left), of_x, acc[b]);
            }
        }
    // a lane holds units 4 (lane / 16) .. + 3 of point lane % 16
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b)
        *reinterpret_cast<float4v*>(&part[wave][mine][16 * b + lane / 16 * 4]) = acc[b];
    const uint32_t row = threadIdx.x / (UNITS / V), run = threadIdx.x % (UNITS / V) * V;
    const bool inside = row < p.points && unit0 + run < p.f.units;
    float bias[V];
    Raw<T, V> residual;
    uint64_t key = 0;
    if (inside) {
        load_bias<X, V>(p.f, unit0 + run, bias);
        load_residual<T, V>(p.f, row, unit0 + run, residual);
        key = p.f.mask.on ? mask_key(p.f.mask) : 0;
    }
    __syncthreads();
    if (!inside)
        return;
    float4v total = *reinterpret_cast<const float4v*>(&part[0][row][run]);
    for (uint32_t i = 1; i < waves; ++i)
        total += *reinterpret_cast<const float4v*>(&part[i][row][run]);
    float v[V];
    __builtin_memcpy(v, &total, 16);
    finish<X, T, true, V>(p.f, key, row, unit0 + run, bias, residual, v);
}

template <typename X, typename T>
void launch_few(const sqn_matrix& x, const sqn_matrix& w, const Finish& f, hipStream_t stream)
{
    FewParams p;
    p.x = x.data;
    p.w = w.data;
    p.x_stride = x.row_stride;
    p.w_stride = w.row_stride;
    p.points = static_cast<uint32_t>(x.rows);
    p.cols = static_cast<uint32_t>(x.cols);
    p.f = f;
    // a wave for every four pieces of the sum; 64 threads finish each 16 units, so
    // larger workgroups have as many waves at least
    const uint32_t blocks = f.units >= 64 * 256 ? 4 : 1;
    const uint32_t waves = std::clamp<uint32_t>((p.cols + 4 * Sixteen<X>::ALL - 1) / (4 * Sixteen<X>::ALL), blocks, kFewWaves);
    const uint32_t groups = (f.units + 16 * blocks - 1) / (16 * blocks);
    if (blocks == 4)
        few_kernel<X, T, 4><<<groups, 64 * waves, 0, stream>>>(p);
    else
        few_kernel<X, T, 1><<<groups, 64 * waves, 0, stream>>>(p);
}

// ---- factors that do not lie on 16-byte boundaries, copied to where they do

struct PackParams {
    const void* from;
    char* to;
    int64_t stride;              // elements
    uint64_t pieces;             // rows * per_row
    uint32_t cols, per_row;      // pieces of 16 bytes in a row, zeros past its end
};

template <typename U>
__global__ __launch_bounds__(kThreads) void pack_kernel(PackParams p)
{
    constexpr uint32_t N = 16 / sizeof(U);
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.pieces;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t row = p.pieces >> 32 ? i / p.per_row : static_cast<uint32_t>(i) / p.per_row;
        const uint32_t col = static_cast<uint32_t>(i - row * p.per_row) * N;
        const U* from = static_cast<const U*>(p.from) + row * p.stride + col;
        U e[N];
        if (col + N <= p.cols) {
            const Run<U, N> r = *reinterpret_cast<const Run<U, N>*>(from);
            __builtin_memcpy(e, &r, 16);
        } else {
#pragma unroll
            for (uint32_t k = 0; k < N; ++k)
                e[k] = col + k < p.cols ? from[k] : U{0};
        }
        uint4 piece;
        __builtin_memcpy(&piece, e, 16);
        *reinterpret_cast<uint4*>(p.to + i * 16) = piece;
    }
}

// ---- factors in two parts of 16 bits

// v as the sum of two values of bfloat16, to 2^-15 of itself, and a binary16 exactly.
// Unless v is 0 both have its sign and are not 0 (the high part is the last value
// before v), and both are v where it is not finite: so their products with an
// infinite factor, or of an infinite v, are what v's own is.
__device__ __forceinline__ void two_parts(float v, __bf16& high, __bf16& low)
{
    const uint32_t bits = __float_as_uint(v);
    const bool finite = fabsf(v) < HUGE_VALF;
    const float h = finite && v != 0.0f ? __uint_as_float((bits - 1) & 0xffff0000u) : v;
    high = from_f32<__bf16>(h);
    low = from_f32<__bf16>(finite ? v - h : v);
}

// A matrix of binary16 as two of bfloat16, `apart` bytes from each other.
__global__ __launch_bounds__(kThreads) void part_kernel(PackParams p, uint64_t apart)
{
    constexpr int N = 8;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.pieces;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t row = p.pieces >> 32 ? i / p.per_row : static_cast<uint32_t>(i) / p.per_row;
        const uint32_t col = static_cast<uint32_t>(i - row * p.per_row) * N;
        float v[N];
        load_inside<_Float16, N>(static_cast<const _Float16*>(p.from) + row * p.stride + col, p.cols - col, v);
        __bf16 high[N], low[N];
#pragma unroll
        for (int k = 0; k < N; ++k)
            two_parts(v[k], high[k], low[k]);
        uint4 piece;
        __builtin_memcpy(&piece, high, 16);
        *reinterpret_cast<uint4*>(p.to + i * 16) = piece;
        __builtin_memcpy(&piece, low, 16);
        *reinterpret_cast<uint4*>(p.to + apart + i * 16) = piece;
    }
}

// ---- the gradient before a layer's activation, and its sums

struct SlopeParams {
    const void *grad, *pre;      // pre: null without an activation
    void* dz;                    // [points][pitch] of the products' type, zeros past the units, or null
    uint64_t apart;              // bytes to its low parts
    float* sums;                 // [groups down][units] or null
    void* bias;                  // the sums themselves, where there is one group
    int32_t bias_dtype;
    int64_t grad_stride, pre_stride;
    uint32_t points, units, pitch, rows, act;     // rows: of a workgroup
    uint32_t across;             // threads along a row: a power of two
    Mask mask;                   // its scale is applied to the products and sums: dz stays in grad's range
};

__device__ __forceinline__ void store_bias(void* out, uint32_t u, float v, int32_t dtype)
{
    if (dtype == SQN_F32)
        static_cast<float*>(out)[u] = v;
    else if (dtype == SQN_F16)
        static_cast<_Float16*>(out)[u] = from_f32<_Float16>(v);
    else
        static_cast<__bf16*>(out)[u] = from_f32<__bf16>(v);
}

// PARTED: dz in two parts of bfloat16.
template <typename X, typename G, bool PARTED>
__global__ __launch_bounds__(kThreads) void slope_kernel(SlopeParams p)
{
    constexpr int V = 8;
    typedef std::conditional_t<PARTED, __bf16, X> D;
    __shared__ float part[kThreads][V + 1];
    const uint32_t tx = threadIdx.x & (p.across - 1), ty = threadIdx.x / p.across, down = kThreads / p.across;
    const uint32_t unit = (blockIdx.x * p.across + tx) * V;
    const uint64_t row0 = static_cast<uint64_t>(blockIdx.y) * p.rows;
    const uint64_t end = min(row0 + p.rows, static_cast<uint64_t>(p.points));
    const uint64_t key = p.mask.on ? mask_key(p.mask) : 0;
    const uint32_t left = unit < p.units ? p.units - unit : 0;
    float sum[V] = {};
    // where the run is inside the row there is no branch between its loads and the
    // next rows'
    auto rows = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        constexpr int TOGETHER = WHOLE ? 2 : 1;
        for (uint64_t row = row0 + ty; row < end; row += TOGETHER * down) {
            Raw<G, V> of_grad[TOGETHER];
            Raw<X, V> of_pre[TOGETHER];
#pragma unroll
            for (int i = 0; i < TOGETHER; ++i) {
                // rows past the end read the last one, and take part in nothing
                const uint64_t at = std::min(row + i * down, end - 1);
                of_grad[i].load(static_cast<const G*>(p.grad) + at * p.grad_stride + unit, WHOLE ? V : left);
                if (p.pre)
                    of_pre[i].load(static_cast<const X*>(p.pre) + at * p.pre_stride + unit, WHOLE ? V : left);
            }
#pragma unroll
            for (int i = 0; i < TOGETHER; ++i) {
                const uint64_t at = row + i * down;
                if (at >= end)
                    break;
                float v[V], z[V];
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    v[k] = to_f32(of_grad[i].e[k]);
                    z[k] = p.pre ? to_f32(of_pre[i].e[k]) : 0.0f;
                }
                if (p.mask.on)
                    apply_mask<V>(p.mask, key, at, unit, 1.0f, v);
                if (p.pre)
                    times_slope<sizeof(X) == 4, V>(p.act, z, v);
                if (p.dz) {
                    D* to = static_cast<D*>(p.dz) + at * p.pitch + unit;
                    const uint32_t room = WHOLE ? V : p.pitch - unit;
                    if constexpr (PARTED) {
                        float high[V], low[V];
#pragma unroll
                        for (int k = 0; k < V; ++k) {
                            D h, l;
                            two_parts(v[k], h, l);
                            high[k] = to_f32(h);
                            low[k] = to_f32(l);
                        }
                        store_values<D, V>(to, room, high);
                        store_values<D, V>(to + p.apart / sizeof(D), room, low);
                    } else {
                        store_values<D, V>(to, room, v);
                    }
                }
#pragma unroll
                for (int k = 0; k < V; ++k)
                    sum[k] += v[k];
            }
        }
    };
    if (left >= V)
        rows(std::true_type{});
    else if (unit < p.pitch)
        rows(std::false_type{});
    if (!p.sums && !p.bias)
        return;
#pragma unroll
    for (int k = 0; k < V; ++k)
        part[threadIdx.x][k] = sum[k];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < p.across * V; c += kThreads) {
        float total = 0.0f;
#pragma unroll 8
        for (uint32_t k = 0; k < down; ++k)
            total += part[k * p.across + c / V][c % V];
        const uint32_t u = blockIdx.x * p.across * V + c;
        if (u >= p.units)
            continue;
        if (p.bias)
            store_bias(p.bias, u, total * p.mask.scale, p.bias_dtype);
        else
            p.sums[static_cast<uint64_t>(blockIdx.y) * p.units + u] = total;
    }
}

// The sums of slope_kernel's workgroups added up: 4 units a workgroup, 64 threads
// each, whose loads are under way together (8 threads each, one load after another,
// took 17 us of 512 sums).
struct BiasParams {
    const float* sums;           // [groups][units]
    void* bias;
    uint32_t groups, units;
    int32_t dtype;
    float scale;
};

constexpr uint32_t kSumUnits = 4, kSumSlices = kThreads / kSumUnits;

__device__ __forceinline__ void bias_share(const BiasParams& p, uint32_t group)
{
    __shared__ float part[kSumSlices][kSumUnits + 1];
    const uint32_t tx = threadIdx.x % kSumUnits, ty = threadIdx.x / kSumUnits, u = group * kSumUnits + tx;
    float total = 0.0f;
    if (u < p.units) {
#pragma unroll 8
        for (uint32_t k = ty; k < p.groups; k += kSumSlices)
            total += p.sums[static_cast<uint64_t>(k) * p.units + u];
    }
    part[ty][tx] = total;
    __syncthreads();
    if (ty || u >= p.units)
        return;
#pragma unroll 8
    for (uint32_t k = 1; k < kSumSlices; ++k)
        total += part[k][tx];
    store_bias(p.bias, u, total * p.scale, p.dtype);
}

// What is left of a gradient's sums in one launch: of the points, of the weights and
// of the bias, each of some workgroups or none.
template <typename X>
__global__ __launch_bounds__(kThreads) void sums_kernel(PartsParams x, PartsParams w, BiasParams bias, uint32_t groups_x,
                                                        uint32_t groups_w)
{
    if (blockIdx.x < groups_x)
        parts_share<X, X, false>(x, blockIdx.x, groups_x);
    else if (blockIdx.x < groups_x + groups_w)
        parts_share<X, X, false>(w, blockIdx.x - groups_x, groups_w);
    else
        bias_share(bias, blockIdx.x - groups_x - groups_w);
}

// ---- choices

constexpr int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// A matrix whose pieces can be brought as they lie: on 16-byte boundaries in whole
// pieces, a tile's rows within 32-bit offsets.
bool in_place(const sqn_matrix& m)
{
    const int64_t size = static_cast<int64_t>(element_size(m.dtype));
    return reinterpret_cast<uintptr_t>(m.data) % kSlot == 0 && m.row_stride * size % kSlot == 0 && m.cols * size % kSlot == 0
        && m.row_stride * size < (int64_t{1} << 23);
}

int64_t packed_cols(const sqn_matrix& m) { return round_up(m.cols, kSlot / static_cast<int64_t>(element_size(m.dtype))); }

size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

size_t pack_bytes(const sqn_matrix& m)
{
    return in_place(m) ? 0 : aligned(static_cast<size_t>(m.rows) * packed_cols(m) * element_size(m.dtype));
}

// What a launch moves at most in one go; threads take more past it.
constexpr uint64_t kMaxGroups = 1u << 22;

uint32_t groups_of(uint64_t items)
{
    return static_cast<uint32_t>(std::min((items + kThreads - 1) / kThreads, kMaxGroups));
}

// The matrix, or a copy of it at `to`, whose rows are filled up.
sqn_matrix packed(const sqn_matrix& m, char*& to, hipStream_t stream)
{
    if (in_place(m))
        return m;
    sqn_matrix c = m;
    c.data = to;
    c.cols = c.row_stride = packed_cols(m);
    to += pack_bytes(m);
    if (m.rows == 0)
        return c;
    PackParams p;
    p.from = m.data;
    p.to = static_cast<char*>(c.data);
    p.stride = m.row_stride;
    p.cols = static_cast<uint32_t>(m.cols);
    p.per_row = static_cast<uint32_t>(c.cols * static_cast<int64_t>(element_size(m.dtype)) / kSlot);
    p.pieces = static_cast<uint64_t>(m.rows) * p.per_row;
    if (m.dtype == SQN_F32)
        pack_kernel<uint32_t><<<groups_of(p.pieces), kThreads, 0, stream>>>(p);
    else
        pack_kernel<uint16_t><<<groups_of(p.pieces), kThreads, 0, stream>>>(p);
    return c;
}

// ---- narrow layers of many points
//
// Bound by the points' bytes, which move once while the weights stay where they
// are used: a wave keeps its 32 rows of P (up to four steps) in registers, as
// fragments, and the workgroups go through the points in slabs that stream into
// one of four LDS buffers, the next three under way.  Of UB blocks of P the
// workgroup's waves take one each, SUBS times, with 32 points of the slab each.
// (Tiles read the points' rows once for every 128 units and wait for their loads a
// round at a time: 500,000 points of 256 by 256 in binary16 154 us, 116 so.)

constexpr int kNarrowRows = 256;
constexpr int64_t kNarrowPoints = 16384;

struct NarrowParams {
    const void *p, *q;           // the weights, [units][cols] either way; the points' rows
    int64_t p_stride;            // elements
    uint64_t q_pitch;            // bytes
    uint32_t p_lines, p_cols;    // of the weights in memory
    uint32_t points, valid;      // valid: bytes of a point's row
    Finish f;                    // units: rows of P
    // with SLOPE, whose points' rows are grad's and become dz's on their way
    const void* pre;             // or null
    uint64_t pre_pitch;          // bytes
    void* dz;                    // [points][dz_pitch elements], or null
    uint64_t dz_apart;           // bytes to its low parts
    float* sums;                 // [gridDim.x][sum], or null
    uint32_t sum, dz_pitch, act;
    uint32_t parted;             // bfloat16 with pre: dz's low parts, where pre's rows were, multiply too
    Mask mask;                   // its scale is the finish's
};

// A piece of 16 bytes at any alignment, of whose elements `left` are there.
template <typename X>
__device__ __forceinline__ uint4 piece_of(const X* p, int32_t left)
{
    constexpr int N = Elements<X>::PIECE;
    if (left >= N) {
        const Run<X, N> r = *reinterpret_cast<const Run<X, N>*>(p);
        uint4 v;
        __builtin_memcpy(&v, &r, 16);
        return v;
    }
    const X* q = ragged(p);
    X e[N];
#pragma unroll
    for (int k = 0; k < N; ++k)
        e[k] = k < left ? q[k] : X(0.0f);
    uint4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// UB blocks of 32 rows of P, STEPS steps of the sum; a lane brings LOAD bytes at once.
template <int UB_, int STEPS_, int LOAD_, bool SLOPE_ = false>
struct Narrow {
    static constexpr int UB = UB_, STEPS = STEPS_, LOAD = LOAD_;
    static constexpr bool SLOPE = SLOPE_;
    static constexpr int SUBS = UB == 8 ? 1 : UB == 4 || STEPS == 4 ? 2 : 4;
    static constexpr int WAVES = UB * SUBS, THREADS = 64 * WAVES;     // that multiply
    static constexpr int BRINGERS = LOAD == 4 ? 4 : 1;                // waves that bring the points
    static constexpr int SIDE = 32 * UB, POINTS = 32 * SUBS;
    static constexpr int BUFFERS = 4;
    static constexpr int STEP = POINTS * static_cast<int>(kStepBytes), ROWS = STEPS * STEP;
    static constexpr int BUFFER = SLOPE ? 2 * ROWS : ROWS;            // grad's rows, and pre's
    static constexpr int LOADS = ROWS / (64 * LOAD) / BRINGERS;     // instructions of a slab, of a wave
    static constexpr int P_STEP = SIDE * static_cast<int>(kStepBytes);
    static constexpr int PIECES = P_STEP / (static_cast<int>(kSlot) * THREADS);    // of P, a thread and step
};

template <typename S, typename X, typename T, bool LAYER, bool PA>
__global__ __launch_bounds__(S::THREADS + 64 * S::BRINGERS) void narrow_kernel(NarrowParams p)
{
    BUFFERS_IN_LDS(S)
    constexpr int OWN = 32 * 128;
    constexpr int SHARED = std::max(S::WAVES * OWN, S::P_STEP);
    __shared__ __align__(16) char shared[SHARED];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t slabs = (p.points + S::POINTS - 1) / S::POINTS;
    // of this workgroup: slabs blockIdx.x, + gridDim.x, ...
    const uint32_t count = (slabs - blockIdx.x + gridDim.x - 1) / gridDim.x;

    if (wave >= S::WAVES) {
        // The waves that bring the points store nothing, so what they wait for is
        // the slab alone (where every wave brought a share, a slab waited for the
        // stores of the one before).
        constexpr uint32_t OUTSIDE = 0x80000000u, LANES = kStepBytes / S::LOAD;    // of a row's step
        constexpr uint32_t ROWS = 64 / LANES;                                     // of an instruction
        const uint32_t byte = lane % LANES * S::LOAD;
        auto bring_rows = [&](const void* q, uint64_t pitch, uint32_t nth, char* to) {
            const uint64_t row0 = (blockIdx.x + static_cast<uint64_t>(nth) * gridDim.x) * S::POINTS;
            const uint32_t left = nth < count ? p.points - static_cast<uint32_t>(row0) : 0;
            const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(
                const_cast<char*>(static_cast<const char*>(q) + row0 * pitch), 0, OUTSIDE, 0x00020000);
            // past the last slab and past a row's end nothing is read, and the loads count as ever
#pragma unroll 8
            for (uint32_t k = 0; k < S::LOADS; ++k) {
                const uint32_t i = (wave - S::WAVES) * S::LOADS + k;
                const uint32_t step = i * (64 * S::LOAD) / S::STEP, row = i * ROWS % S::POINTS + lane / LANES;
                const uint32_t at = step * kStepBytes + ((byte / kSlot) ^ (row >> 1 & 7)) * kSlot + byte % kSlot;
                const uint32_t from = row < left && at < p.valid ? row * static_cast<uint32_t>(pitch) + at : OUTSIDE;
                if constexpr (S::LOAD == kSlot)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void*)(to + i * (64 * S::LOAD)), kSlot, from, 0, 0, 0);
                else
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_void*)(to + i * (64 * S::LOAD)), 4, from, 0, 0, 0);
            }
        };
        auto bring_slab = [&](uint32_t nth, char* to) {
            bring_rows(p.q, p.q_pitch, nth, to);
            if (S::SLOPE && p.pre)
                bring_rows(p.pre, p.pre_pitch, nth, to + S::ROWS);
        };
#pragma unroll
        for (int b = 0; b < S::BUFFERS - 1; ++b)
            bring_slab(b, buffers[b]);
        for (int k = 0; k < 2 * S::STEPS; ++k)       // the weights' barriers
            __builtin_amdgcn_s_barrier();
        for (uint32_t n = 0; n < count; n += S::BUFFERS)
#pragma unroll
            for (int b = 0; b < S::BUFFERS; ++b)
                if (n + b < count) {
                    if (S::SLOPE && p.pre)
                        landed<std::min((S::BUFFERS - 2) * 2 * S::LOADS, 63)>();
                    else
                        landed<std::min((S::BUFFERS - 2) * S::LOADS, 63)>();
                    bring_slab(n + b + S::BUFFERS - 1, buffers[(b + S::BUFFERS - 1) % S::BUFFERS]);
                    if constexpr (S::SLOPE)          // dz's barrier
                        __builtin_amdgcn_s_barrier();
                }
        // the loads still under way end before their buffers do
        landed_own<0>();
        return;
    }

    const uint32_t block = wave % S::UB, sub = wave / S::UB, half = lane >> 5, mine = lane & 31;
    // the weights through LDS into the waves that use them, a step at a time
    uint4 w[S::STEPS * kDepths];
    {
        uint4 piece[S::STEPS][S::PIECES];
        uint32_t to[S::PIECES];
        const X* rows = static_cast<const X*>(p.p);
        constexpr uint32_t N = Elements<X>::PIECE, ACROSS = S::SIDE / N;
#pragma unroll
        for (int i = 0; i < S::PIECES; ++i) {
            const uint32_t id = S::THREADS * i + threadIdx.x;
            const uint32_t line = PA ? id / ACROSS : id / 8, col = PA ? id % ACROSS * N : id % 8 * N;
            to[i] = PA ? (line * ACROSS + ((id % ACROSS) ^ across_key<X, S::SIDE>(line))) * kSlot
                       : (line * 8 + ((id % 8) ^ (line >> 1 & 7))) * kSlot;
            auto of_step = [&](int k, auto load) {
                const uint32_t l = line + (PA ? k * Elements<X>::STEP : 0), c = col + (PA ? 0 : k * Elements<X>::STEP);
                return load(rows + l * p.p_stride + c, l < p.p_lines ? static_cast<int32_t>(p.p_cols) - static_cast<int32_t>(c) : 0);
            };
            // without a branch all of a thread's loads are under way together
            if (p.p_cols % N == 0) {
#pragma unroll
                for (int k = 0; k < S::STEPS; ++k)
                    piece[k][i] = of_step(k, [&](const X* from, int32_t left) {
                        const uint4 v = piece_of<X>(left > 0 ? from : rows, N);
                        return left > 0 ? v : uint4{0, 0, 0, 0};
                    });
            } else {
#pragma unroll
                for (int k = 0; k < S::STEPS; ++k)
                    piece[k][i] = of_step(k, piece_of<X>);
            }
        }
        const Reader<X, S::SIDE, PA, 1> read_p(32 * block);
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
#pragma unroll
            for (int i = 0; i < S::PIECES; ++i)
                *reinterpret_cast<uint4*>(shared + to[i]) = piece[k][i];
            landed<63>();
#pragma unroll
            for (int o = 0; o < kDepths; ++o)
                w[k * kDepths + o] = read_p.read(shared, 0, o);
            landed<63>();
        }
    }

    constexpr int V = 16 / sizeof(T);
    constexpr uint32_t RUNS = 32 / V, ROUNDS = RUNS / 2;
    const uint32_t unit = 32 * block + V * (lane % RUNS);
    float bias[V];
    if constexpr (LAYER)
        load_bias<X, V>(p.f, unit, bias);
    const uint64_t key = LAYER && p.f.mask.on ? mask_key(p.f.mask) : 0;
    const Reader<X, S::POINTS, false, 1> read_q(32 * sub);
    char* own = shared + wave * OWN;
    auto slot = [](uint32_t column, uint32_t piece) { return column * 128 + (piece ^ (column & 7)) * 16; };
    // With SLOPE a thread takes the same units of rows of every slab, so that their
    // sums stay with it.
    constexpr int N = Elements<X>::PIECE;
    constexpr uint32_t GROUPS = 8 * S::STEPS, DOWN = S::THREADS / GROUPS;
    const uint32_t of_step = threadIdx.x % GROUPS / 8, piece = threadIdx.x % 8, down = threadIdx.x / GROUPS;
    const uint32_t of_unit = of_step * Elements<X>::STEP + piece * N;
    const uint64_t slope_key = S::SLOPE && p.mask.on ? mask_key(p.mask) : 0;
    float sum[N] = {};
    auto slope_slab = [&](uint32_t nth, char* buffer) {
#pragma unroll
        for (uint32_t row = down; row < S::POINTS; row += DOWN) {
            char* at = buffer + of_step * S::STEP + row * kStepBytes + (piece ^ (row >> 1 & 7)) * kSlot;
            const uint64_t point = (blockIdx.x + static_cast<uint64_t>(nth) * gridDim.x) * S::POINTS + row;
            X e[N];
            float v[N], z[N];
            __builtin_memcpy(e, at, 16);
#pragma unroll
            for (int k = 0; k < N; ++k)
                v[k] = to_f32(e[k]);
            if (p.mask.on)
                apply_mask<N>(p.mask, slope_key, point, of_unit, 1.0f, v);
            if (p.pre) {
                __builtin_memcpy(e, at + S::ROWS, 16);
#pragma unroll
                for (int k = 0; k < N; ++k)
                    z[k] = to_f32(e[k]);
                times_slope<sizeof(X) == 4, N>(p.act, z, v);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                sum[k] += v[k];
                e[k] = from_f32<X>(v[k]);
            }
            X low[N];
            if constexpr (std::is_same_v<X, __bf16>)
                if (p.parted)
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        two_parts(v[k], e[k], low[k]);
            uint4 whole;
            __builtin_memcpy(&whole, e, 16);
            *reinterpret_cast<uint4*>(at) = whole;
            char* to = p.dz && point < p.points && of_unit < p.dz_pitch
                ? reinterpret_cast<char*>(static_cast<X*>(p.dz) + point * p.dz_pitch + of_unit) : nullptr;
            if (to)
                *reinterpret_cast<uint4*>(to) = whole;
            if constexpr (std::is_same_v<X, __bf16>)
                if (p.parted) {
                    __builtin_memcpy(&whole, low, 16);
                    *reinterpret_cast<uint4*>(at + S::ROWS) = whole;
                    if (to)
                        *reinterpret_cast<uint4*>(to + p.dz_apart) = whole;
                }
        }
    };
    auto work = [&](uint32_t nth, char* buffer) {
        // every wave has read the slab before, and this one has landed
        landed<63>();
        if constexpr (S::SLOPE) {
            if (down < static_cast<uint32_t>(S::POINTS))
                slope_slab(nth, buffer);
            landed<63>();
        }
        // two sums side by side, of every other depth
        float16v acc[2] = {};
#pragma unroll
        for (int k = 0; k < S::STEPS * kDepths; ++k) {
            const uint4 q = read_q.read(buffer + k / kDepths * S::STEP, 0, k % kDepths);
#pragma unroll
            for (int e = 0; e < (sizeof(X) == 4 ? 4 : 1); ++e)
                acc[(k + e) & 1] = multiply<X>(w[k], q, e, acc[(k + e) & 1]);
        }
        // (one loop for both, as a function of the rows, spilled registers)
        if constexpr (S::SLOPE && std::is_same_v<X, __bf16>)
            if (p.parted) {
#pragma unroll
                for (int k = 0; k < S::STEPS * kDepths; ++k) {
                    const uint4 q = read_q.read(buffer + S::ROWS + k / kDepths * S::STEP, 0, k % kDepths);
                    acc[k & 1] = multiply<X>(w[k], q, 0, acc[k & 1]);
                }
            }
        acc[0] += acc[1];
        const uint64_t row0 = (blockIdx.x + static_cast<uint64_t>(nth) * gridDim.x) * S::POINTS + 32 * sub + lane / RUNS;
        Raw<T, V> residual[ROUNDS];
        if constexpr (LAYER)
#pragma unroll
            for (uint32_t i = 0; i < ROUNDS; ++i)
                if (row0 + i * (64 / RUNS) < p.points && unit < p.f.units)
                    load_residual<T, V>(p.f, row0 + i * (64 / RUNS), unit, residual[i]);
#pragma unroll
        for (uint32_t g = 0; g < 4; ++g)
            *reinterpret_cast<float4v*>(own + slot(mine, 2 * g + half))
                = float4v{acc[0][4 * g], acc[0][4 * g + 1], acc[0][4 * g + 2], acc[0][4 * g + 3]};
        wave_fence();
#pragma unroll
        for (uint32_t i = 0; i < ROUNDS; ++i) {
            const uint32_t column = i * (64 / RUNS) + lane / RUNS;
            float v[V];
#pragma unroll
            for (int k = 0; k < V / 4; ++k) {
                const float4v e = *reinterpret_cast<const float4v*>(own + slot(column, V / 4 * (lane % RUNS) + k));
                __builtin_memcpy(v + 4 * k, &e, 16);
            }
            if (row0 + i * (64 / RUNS) < p.points && unit < p.f.units)
                finish<X, T, LAYER, V>(p.f, key, row0 + i * (64 / RUNS), unit, bias, residual[i], v);
        }
        wave_fence();
    };
    for (uint32_t n = 0; n < count; n += S::BUFFERS)
#pragma unroll
        for (int b = 0; b < S::BUFFERS; ++b)
            if (n + b < count)
                work(n + b, buffers[b]);
    if constexpr (S::SLOPE) {
        if (!p.sums)
            return;
        // the workgroup's sums, in the order of the rows
        float(*part)[N] = reinterpret_cast<float(*)[N]>(shared);
        landed<63>();
#pragma unroll
        for (int k = 0; k < N; ++k)
            part[threadIdx.x][k] = sum[k];
        landed<63>();
        for (uint32_t u = threadIdx.x; u < p.sum; u += S::THREADS) {
            const uint32_t group = u / Elements<X>::STEP * 8 + u % Elements<X>::STEP / N;
            float total = 0.0f;
#pragma unroll 8
            for (uint32_t k = 0; k < std::min<uint32_t>(DOWN, S::POINTS); ++k)
                total += part[k * GROUPS + group][u % N];
            p.sums[static_cast<uint64_t>(blockIdx.x) * p.sum + u] = total;
        }
    }
}

// Layers whose weights a workgroup's registers hold, of points enough for several
// slabs a CU, where tiles would need copies onto 16-byte boundaries or read the
// points twice; of binary16 and bfloat16 also where tiles of 64 and 128 are so many
// that their starts and ends are most of the time.  (us so and in tiles: 65,536
// points of 256 by 256 in binary16 19 and 20, the gradient of its points 17 and 18,
// of 500,000 116 and 154, of 20,000 11 and 10; of 64 by 64 of 65,536 8.0 and 7.7, of
// 131,072 12 and 13, of 500,000 25 and 46, in binary32 72 and 80; of 128 by 128 of
// 500,000 42 and 56, in binary32 187 and 176; of 50,001 points of 42 by 256 of
// binary32 31 and 46.)
bool narrow_of(const sqn_matrix& w, int64_t units, int64_t sum, int64_t points, bool points_in_place)
{
    if (units > kNarrowRows || sum * static_cast<int64_t>(element_size(w.dtype)) > 4 * kStepBytes || points < kNarrowPoints)
        return false;
    if (!in_place(w) || !points_in_place)
        return true;
    return units > kNarrowRows / 2 ? points >= 2 * kNarrowPoints : w.dtype != SQN_F32 && points >= 8 * kNarrowPoints;
}

// Whether the points' rows can be brought from where they lie: binary32 elements
// one at a time.
bool narrow_in_place(const sqn_matrix& q)
{
    return in_place(q) || (q.dtype == SQN_F32 && q.row_stride * 4 < (int64_t{1} << 23));
}

size_t narrow_pack_bytes(const sqn_matrix& q) { return narrow_in_place(q) ? 0 : pack_bytes(q); }

// The workgroups.
template <typename S, typename X, typename T, bool LAYER, bool PA>
uint32_t launch_narrow_shape(const NarrowParams& p, hipStream_t stream)
{
    const uint32_t slabs = (p.points + S::POINTS - 1) / S::POINTS, groups = std::min(slabs, S::WAVES == 8 ? 256u : 512u);
    narrow_kernel<S, X, T, LAYER, PA><<<groups, S::THREADS + 64 * S::BRINGERS, 0, stream>>>(p);
    return groups;
}

// wide: rows on 16-byte boundaries.
template <int UB, int STEPS, typename X, typename T, bool LAYER, bool PA>
void launch_narrow_steps(const NarrowParams& p, bool wide, hipStream_t stream)
{
    if constexpr (sizeof(X) == 4) {
        if (!wide) {
            launch_narrow_shape<Narrow<UB, STEPS, 4>, X, T, LAYER, PA>(p, stream);
            return;
        }
    }
    launch_narrow_shape<Narrow<UB, STEPS, 16>, X, T, LAYER, PA>(p, stream);
}

template <int UB, typename X, typename T, bool LAYER, bool PA>
void launch_narrow_blocks(const NarrowParams& p, int64_t sum, bool wide, hipStream_t stream)
{
    const int64_t steps = (sum * static_cast<int64_t>(sizeof(X)) + kStepBytes - 1) / kStepBytes;
    if (steps == 1)
        launch_narrow_steps<UB, 1, X, T, LAYER, PA>(p, wide, stream);
    else if (steps == 2)
        launch_narrow_steps<UB, 2, X, T, LAYER, PA>(p, wide, stream);
    else
        launch_narrow_steps<UB, 4, X, T, LAYER, PA>(p, wide, stream);
}

// w [lines][cols]: the units, or, PA, the sum.
NarrowParams narrow_params(const sqn_matrix& w, const sqn_matrix& q, const Finish& f)
{
    const int64_t size = static_cast<int64_t>(element_size(q.dtype));
    NarrowParams p{};
    p.p = w.data;
    p.q = q.data;
    p.p_stride = w.row_stride;
    p.q_pitch = static_cast<uint64_t>(q.row_stride * size);
    p.p_lines = static_cast<uint32_t>(w.rows);
    p.p_cols = static_cast<uint32_t>(w.cols);
    p.points = static_cast<uint32_t>(q.rows);
    p.valid = static_cast<uint32_t>(q.cols * size);
    p.f = f;
    return p;
}

template <typename X, typename T, bool LAYER, bool PA>
void launch_narrow(const sqn_matrix& w, const sqn_matrix& points, int64_t sum, const Finish& f, char* work, hipStream_t stream)
{
    const sqn_matrix q = narrow_in_place(points) ? points : packed(points, work, stream);
    const NarrowParams p = narrow_params(w, q, f);
    const bool wide = in_place(q);
    if (f.units <= 64)
        launch_narrow_blocks<2, X, T, LAYER, PA>(p, sum, wide, stream);
    else if (f.units <= 128)
        launch_narrow_blocks<4, X, T, LAYER, PA>(p, sum, wide, stream);
    else
        launch_narrow_blocks<8, X, T, LAYER, PA>(p, sum, wide, stream);
}

// The gradient of the points, and before it dz and the sums of its rows in groups,
// in one go over grad and pre (apart 65,536 points of 256 by 256 in binary16 took
// 42 us).
constexpr uint32_t kSlopedGroups = 256;

bool narrow_sloped(const sqn_matrix& grad, const sqn_matrix& x, const sqn_matrix& w, const sqn_matrix* pre)
{
    return x.cols > kNarrowRows / 2 && grad.dtype == x.dtype && narrow_of(w, x.cols, w.rows, x.rows, true) && narrow_in_place(grad)
        && (!pre || narrow_in_place(*pre));
}

template <int STEPS, typename X>
uint32_t launch_sloped_steps(const NarrowParams& p, bool wide, hipStream_t stream)
{
    if constexpr (sizeof(X) == 4) {
        if (!wide)
            return launch_narrow_shape<Narrow<8, STEPS, 4, true>, X, X, false, true>(p, stream);
    }
    return launch_narrow_shape<Narrow<8, STEPS, 16, true>, X, X, false, true>(p, stream);
}

// The groups of sums.
template <typename X>
uint32_t launch_sloped(const sqn_matrix& w, const sqn_matrix& grad, const sqn_matrix* pre, int32_t act, const Mask& m, void* dz,
                       int64_t dz_pitch, uint64_t dz_apart, bool parted, float* sums, const Finish& f, hipStream_t stream)
{
    NarrowParams p = narrow_params(w, grad, f);
    p.pre = pre ? pre->data : nullptr;
    p.pre_pitch = pre ? static_cast<uint64_t>(pre->row_stride) * sizeof(X) : 0;
    p.dz = dz;
    p.dz_pitch = static_cast<uint32_t>(dz_pitch);
    p.dz_apart = dz_apart;
    p.parted = parted ? 1 : 0;
    p.sums = sums;
    p.sum = static_cast<uint32_t>(w.rows);
    p.act = static_cast<uint32_t>(act);
    p.mask = m;
    const bool wide = in_place(grad) && (!pre || in_place(*pre));
    const int64_t steps = (w.rows * static_cast<int64_t>(sizeof(X)) + kStepBytes - 1) / kStepBytes;
    if (steps == 1)
        return launch_sloped_steps<1, X>(p, wide, stream);
    if (steps == 2)
        return launch_sloped_steps<2, X>(p, wide, stream);
    return launch_sloped_steps<4, X>(p, wide, stream);
}

Operand along(const sqn_matrix& m)
{
    const int64_t size = static_cast<int64_t>(element_size(m.dtype));
    return {static_cast<const char*>(m.data), static_cast<uint64_t>(m.row_stride * size), static_cast<uint32_t>(m.rows),
            static_cast<uint32_t>(m.cols * size), 0, 0};
}

Operand across(const sqn_matrix& m)
{
    const int64_t size = static_cast<int64_t>(element_size(m.dtype));
    return {static_cast<const char*>(m.data), static_cast<uint64_t>(m.row_stride * size), static_cast<uint32_t>(m.cols),
            static_cast<uint32_t>(m.rows), 0, 0};
}

// Tiles and parts of a product's sum.
struct Plan {
    int64_t side;
    int64_t steps, part_steps, parts;
    size_t bytes;                // of the parts' sums
    double time, work;           // alone, and of all CUs' time beside others
};

int64_t tiles_of(int64_t rows_p, int64_t rows_q, int64_t side) { return (rows_p + side - 1) / side * ((rows_q + side - 1) / side); }

// A step of tiles of 64, 128 and 256 (of 16 bits) and a tile's start and end, in us.
constexpr int64_t kSides[3] = {64, 128, 256}, kCus = 256;
constexpr double kStep[2][3] = {{0.26, 0.46, 1.45}, {0.51, 1.79}}, kEnds[3] = {1.5, 3.0, 18.0};

// Tiles and parts by what they take, in us: the rounds of workgroups on 256 CUs,
// each the steps of a part and a start and an end, and a launch and the bytes of the
// parts' sums behind them.  A step's time is the CU's matrix cores' in the largest
// tiles and for binary32, and what L2 and LDS deliver in the smaller ones, of which
// two workgroups share a CU.  (us by side, 64, 128 and 256, of bfloat16: 4096 points
// of 256 by 256 5, 7 and 19; 65,536 34, 21 and 25; 2048 of 4096 by 2048 54, 44 and 85;
// 8192 of 1024 by 1024 33, 23 and 36; of binary32: 65,536 of 256 by 256 84, 75 and 80,
// 1024 of 4096 by 1024 72, 237 and 919: four tiles of 128 never take more than one of
// 256, whose reads its matrix instructions outweigh.  By parts, 1, 4 and 16, 17 points
// of 4096 by 4096 16, 10 and 15; a gradient's 256 x 256 over 16,384 points 58, 20 and 14.)
Plan plan_of(int64_t rows_p, int64_t rows_q, int64_t sum, int32_t dtype, int64_t terms = 1, int64_t only = 0)
{
    constexpr int64_t kMostParts = 64;
    constexpr double kAlone = 0.12;      // a step in tiles of 128 takes more without another workgroup beside it
    constexpr double kJoin = 4.0, kJoinBytes = 3.5e6;            // a us
    const int f32 = dtype == SQN_F32 ? 1 : 0;
    const int64_t step = kStepBytes / static_cast<int64_t>(element_size(dtype));
    const int64_t steps = (sum + step - 1) / step * terms;
    Plan r{64, steps, std::max<int64_t>(1, steps), steps ? 1 : 0, 0, HUGE_VAL, 0.0};
    for (int s = 0; steps && s < (f32 ? 2 : 3); ++s) {
        if (only && kSides[s] != only)
            continue;
        const int64_t tiles = tiles_of(rows_p, rows_q, kSides[s]);
        for (int64_t parts = 1; parts <= std::min(kMostParts, steps); parts *= 2) {
            const int64_t each = (steps + parts - 1) / parts, used = (steps + each - 1) / each;
            const double sums = used > 1 ? 2.0 * used * 4.0 * rows_q * round_up(rows_p, 4) : 0.0;
            const int64_t rounds = (tiles * used + kCus - 1) / kCus;
            const double group = each * (kStep[f32][s] + (s == 1 && rounds == 1 ? kAlone : 0.0)) + kEnds[s];
            const double join = used > 1 ? kJoin + sums / kJoinBytes : 0.0;
            const double time = rounds * group + join;
            if (time < r.time) {
                r.time = time;
                r.work = static_cast<double>(tiles * used) / kCus * group + join;
                r.side = kSides[s];
                r.part_steps = each;
                r.parts = used;
            }
            // further parts only add rounds
            if (tiles * parts >= 2 * kCus)
                break;
        }
    }
    r.bytes = r.parts > 1 ? aligned(static_cast<size_t>(r.parts) * rows_q * round_up(rows_p, 4) * 4) : 0;
    return r;
}

// A layer's tiles: an epilogue that computes or moves more than the sums stands alone
// in tiles of 256 and beside another tile's products in those of 128.  (us in tiles of
// 128 and 256, 8192 by 8192 outputs in bfloat16: sums of 2048 elements with z kept 318
// and 276, with GELU and a mask 304 and 318, with a residual 338 and 357; with GELU, a
// mask and z kept, of 1024 227 and 238, of 2048 353 and 340 (on another card 324 and
// 330), of 4096 595 and 547.)
Plan layer_plan(const Finish& f, int64_t rows, int64_t sum, int32_t dtype)
{
    Plan plan = plan_of(f.units, rows, sum, dtype);
    if (plan.side != 256 || plan.parts != 1)
        return plan;
    constexpr double kCompute = 17.0, kKeep = 11.0, kAdd = 33.0, kBeside = 0.2;     // us of a tile of 256; of that in one of 128
    const double more = kCompute * ((f.act > SQN_ACT_RELU ? 1 : 0) + f.mask.on) + kKeep * (f.pre ? 1 : 0) + kAdd * (f.residual ? 1 : 0);
    auto time = [&](int s, double ends) {
        const int64_t rounds = (tiles_of(f.units, rows, kSides[s]) + kCus - 1) / kCus;
        return rounds * (plan.steps * kStep[0][s] + kEnds[s] + ends);
    };
    if (time(1, kBeside * more) < time(2, more))
        plan.side = 128;
    return plan;
}

// Both products of a gradient: in one launch where tiles of one side for both take
// less than each by itself and a launch between them.  (All of a gradient in bfloat16 in
// a graph, so and apart: 1000 points of 512 by 512 13 us and 17, 2048 of 2048 by 2048 47
// and 59, 16 of 4096 by 4096 26 and 28; with SiLU, whose dz has two parts, 21 and 28, 83
// and 98, 32 and 32.)
struct GradientPlan {
    Plan x, w;
    bool pair;

    GradientPlan(int64_t points, int64_t cols, int64_t units, int32_t dtype, int64_t terms)
        : x(plan_of(cols, points, units, dtype, terms)), w(plan_of(cols, units, points, dtype, terms)), pair(false)
    {
        constexpr double kLaunch = 3.0;
        double least = x.time + w.time + kLaunch;
        const Plan *best_x = nullptr, *best_w = nullptr;
        Plan of_x[2], of_w[2];
        for (int k = 0; points && k < 2; ++k) {
            of_x[k] = plan_of(cols, points, units, dtype, terms, 64 << k);
            of_w[k] = plan_of(cols, units, points, dtype, terms, 64 << k);
            const double time = std::max({of_x[k].time, of_w[k].time, of_x[k].work + of_w[k].work});
            if (time < least) {
                least = time;
                best_x = &of_x[k];
                best_w = &of_w[k];
            }
        }
        if (best_x) {
            x = *best_x;
            w = *best_w;
            pair = true;
        }
    }
};

// A product of `rows` rows of C; `partial` holds the plan's bytes.
ProductParams product_of(const Operand& a, const Operand& b, int64_t rows, const Plan& plan, const Finish& f, char* partial,
                         uint32_t terms = 1)
{
    ProductParams p{};
    p.p = a;
    p.q = b;
    p.rows = static_cast<uint32_t>(rows);
    p.tiles_p = static_cast<uint32_t>((f.units + plan.side - 1) / plan.side);
    p.tiles_q = static_cast<uint32_t>((rows + plan.side - 1) / plan.side);
    p.steps = static_cast<uint32_t>(plan.steps);
    p.part_steps = static_cast<uint32_t>(plan.part_steps);
    p.parts = static_cast<uint32_t>(plan.parts);
    p.terms = Terms(terms);
    p.partial = reinterpret_cast<float*>(partial);
    p.partial_pitch = static_cast<uint32_t>(round_up(f.units, 4));
    p.f = f;
    return p;
}

uint32_t groups_of(const ProductParams& p) { return p.tiles_p * p.tiles_q * p.parts; }

// What is left to add up of several parts, or none.
PartsParams parts_of(const ProductParams& p)
{
    PartsParams j{};
    j.partial = p.partial;
    j.rows = p.rows;
    j.parts = p.parts;
    j.pitch = p.partial_pitch;
    j.per_row = j.pitch / 4;
    j.runs = j.rows * j.per_row;
    j.f = p.f;
    // up to 16 threads a run, while that leaves all of them busy
    j.slices = 1;
    while (2 * j.slices <= std::min(j.parts, 16u) && j.runs * j.slices < 256 * kThreads)
        j.slices *= 2;
    return j;
}

uint32_t groups_of(const PartsParams& j) { return j.parts == 1 ? 0 : groups_of(j.runs * j.slices); }

template <typename X, typename T, bool LAYER, bool PA, bool QA, bool PARTED>
void launch_tiles(const ProductParams& p, int64_t side, hipStream_t stream)
{
    const uint32_t groups = groups_of(p);
    if (groups == 0)
        return;
    if constexpr (sizeof(X) == 2)
        if (side == 256) {
            tile_kernel<Shape<256>, X, T, LAYER, PA, QA, PARTED><<<groups, Shape<256>::THREADS, 0, stream>>>(p);
            return;
        }
    if (side == 128)
        tile_kernel<Shape<128>, X, T, LAYER, PA, QA, PARTED><<<groups, Shape<128>::THREADS, 0, stream>>>(p);
    else
        tile_kernel<Shape<64>, X, T, LAYER, PA, QA, PARTED><<<groups, Shape<64>::THREADS, 0, stream>>>(p);
}

template <typename X, typename T, bool PARTED>
void launch_pair(const ProductParams& x, const ProductParams& w, int64_t side, hipStream_t stream)
{
    const uint32_t of_x = groups_of(x), groups = of_x + groups_of(w);
    if (side == 128)
        pair_kernel<Shape<128>, X, T, PARTED><<<groups, Shape<128>::THREADS, 0, stream>>>(x, w, of_x);
    else
        pair_kernel<Shape<64>, X, T, PARTED><<<groups, Shape<64>::THREADS, 0, stream>>>(x, w, of_x);
}

template <typename X, typename T>
void launch_layer_typed(const sqn_matrix& x, const sqn_matrix& w, const Finish& f, char* work, hipStream_t stream)
{
    if (x.rows <= kFewPoints) {
        launch_few<X, T>(x, w, f, stream);
        return;
    }
    if (narrow_of(w, w.rows, x.cols, x.rows, in_place(x))) {
        launch_narrow<X, T, true, false>(w, x, x.cols, f, work, stream);
        return;
    }
    const sqn_matrix a = packed(w, work, stream), b = packed(x, work, stream);
    const Plan plan = layer_plan(f, x.rows, x.cols, x.dtype);
    const ProductParams p = product_of(along(a), along(b), x.rows, plan, f, work);
    launch_tiles<X, T, true, false, false, false>(p, plan.side, stream);
    const PartsParams j = parts_of(p);
    if (j.parts != 1)
        parts_kernel<X, T><<<groups_of(j), kThreads, 0, stream>>>(j);
}

// Workgroups of slope_kernel: `across` threads of one along a row, `rows` of it,
// `groups` down the points.  Few points are one group, whose sums are the bias's
// gradient; else some 1024 workgroups, whose sums a launch behind them adds up
// (65,536 points of 256 units, both launches: 28 us, of 512 workgroups 30, of 2048
// 31).
constexpr int64_t kSlopeGroups = 1024;

struct SlopePlan {
    uint32_t across, rows, groups;

    SlopePlan(int64_t points, int64_t units)
    {
        const int64_t runs = (units + 7) / 8;
        const bool few = points <= 256;
        across = 1;
        while (across < (few ? 4 : 32) && across < runs)
            across *= 2;
        const int64_t wide = (runs + across - 1) / across, down = kThreads / across;
        const int64_t most = few ? 1 : std::clamp<int64_t>(kSlopeGroups / wide, 1, kSlopeGroups);
        rows = static_cast<uint32_t>(std::max((points + most - 1) / most, std::min<int64_t>(points, 4 * down)));
        groups = rows ? static_cast<uint32_t>((points + rows - 1) / rows) : 0;
    }
};

// Terms of a gradient's products.  dz = D(grad) act'(z) is as good as the factors'
// type for one where it is grad's own values and zeros; else 16 bits would lose digits
// of binary32 that the sums keep (bfloat16: 2.3e-3 of a gradient's norm for its own
// rounding's 1.7e-3), and binary16 values out of its range.  It is held in two parts
// of bfloat16 then, to 2^-15 of itself and in binary32's range.  Against bfloat16
// factors that makes two terms; against binary16 ones, two parts of bfloat16
// themselves, three: low by low, 2^-14 of a product at most, is left out.
constexpr uint32_t kLowOfDz = 2, kLowOfFactor = 4;       // the terms that take them: dz's second, the factor's third

uint32_t terms_of(int32_t act, int32_t grad_dtype, int32_t dtype)
{
    if (dtype == SQN_F32 || (act <= SQN_ACT_RELU && grad_dtype == dtype))
        return 1;
    return dtype == SQN_BF16 ? 2 : 3;
}

// The other factor of a product in `terms`: as it lies, packed or in parts.
size_t factor_bytes(const sqn_matrix& m, uint32_t terms)
{
    return terms == 3 ? 2 * aligned(static_cast<size_t>(m.rows) * packed_cols(m) * 2) : pack_bytes(m);
}

Operand factor_across(const sqn_matrix& m, uint32_t terms, char*& to, hipStream_t stream)
{
    if (terms != 3)
        return across(packed(m, to, stream));
    sqn_matrix c = m;
    c.data = to;
    c.dtype = SQN_BF16;
    c.cols = c.row_stride = packed_cols(m);
    Operand o = across(c);
    o.apart = factor_bytes(m, terms) / 2;
    o.low = kLowOfFactor;
    to += factor_bytes(m, terms);
    if (m.rows == 0)
        return o;
    PackParams p;
    p.from = m.data;
    p.to = static_cast<char*>(c.data);
    p.stride = m.row_stride;
    p.cols = static_cast<uint32_t>(m.cols);
    p.per_row = static_cast<uint32_t>(c.cols / 8);
    p.pieces = static_cast<uint64_t>(m.rows) * p.per_row;
    part_kernel<<<groups_of(p.pieces), kThreads, 0, stream>>>(p, o.apart);
    return o;
}

// What a gradient keeps in its workspace, in this order.
struct GradientScratch {
    uint32_t terms;
    bool own_dz;                 // grad is dz as it lies otherwise
    bool narrow;                 // the points' gradient of a narrow layer
    size_t dz, sums, x, w, partial_x, partial_w;
    size_t dz_apart;             // bytes of dz to its low parts
    bool pair;                   // both products in one launch
    Plan plan_x, plan_w;

    GradientScratch(const sqn_matrix& grad, const sqn_matrix& x_, const sqn_matrix& w_, int32_t act, bool masked, bool for_x, bool for_w,
                    bool for_bias)
    {
        const int64_t points = x_.rows, units = w_.rows;
        terms = terms_of(act, grad.dtype, x_.dtype);
        own_dz = (for_x || for_w) && (act != SQN_ACT_NONE || masked || grad.dtype != x_.dtype || !in_place(grad));
        const int64_t piece = kSlot / static_cast<int64_t>(element_size(x_.dtype));
        dz_apart = aligned(static_cast<size_t>(points) * round_up(units, piece) * element_size(x_.dtype));
        dz = own_dz ? (terms > 1 ? 2 : 1) * dz_apart : 0;
        // dz in parts is multiplied in narrow kernels where it is made, and whether that
        // is so goes by pre's alignment too: there is room for either way
        narrow = for_x && terms < 3 && narrow_of(w_, x_.cols, units, points, true);
        const bool tiles = for_x && (!narrow || terms == 2);
        const uint32_t groups = std::max(SlopePlan(points, units).groups, narrow ? kSlopedGroups : 0);
        sums = for_bias && groups > 1 ? aligned(static_cast<size_t>(groups) * units * 4) : 0;
        x = for_w ? factor_bytes(x_, terms) : 0;
        w = tiles ? factor_bytes(w_, terms) : 0;
        const GradientPlan plan(points, x_.cols, units, x_.dtype, terms);
        pair = plan.pair && for_x && for_w && !narrow;
        plan_x = pair ? plan.x : plan_of(x_.cols, points, units, x_.dtype, terms);
        plan_w = pair ? plan.w : plan_of(x_.cols, units, points, x_.dtype, terms);
        partial_x = tiles ? plan_x.bytes : 0;
        partial_w = for_w ? plan_w.bytes : 0;
    }

    size_t bytes() const { return dz + sums + x + w + partial_x + partial_w; }
};

// The products of a gradient that tiles compute, from factors of type X.
template <typename X, typename T, bool PARTED>
void launch_products(const ProductParams* of_x, const ProductParams* of_w, const GradientScratch& scratch, hipStream_t stream)
{
    if (of_x && of_w && scratch.pair) {
        launch_pair<X, T, PARTED>(*of_x, *of_w, scratch.plan_w.side, stream);
        return;
    }
    if (of_x)
        launch_tiles<X, T, false, true, false, PARTED>(*of_x, scratch.plan_x.side, stream);
    if (of_w)
        launch_tiles<X, T, false, true, true, PARTED>(*of_w, scratch.plan_w.side, stream);
}

template <typename X>
void launch_slopes(const SlopeParams& p, bool grad_f32, bool parted, const dim3& grid, hipStream_t stream)
{
    if constexpr (sizeof(X) == 4)
        slope_kernel<X, X, false><<<grid, kThreads, 0, stream>>>(p);
    else if (grad_f32)
        slope_kernel<X, float, true><<<grid, kThreads, 0, stream>>>(p);
    else if (parted)
        slope_kernel<X, X, true><<<grid, kThreads, 0, stream>>>(p);
    else
        slope_kernel<X, X, false><<<grid, kThreads, 0, stream>>>(p);
}

template <typename X>
hipError_t launch_gradient_typed(const sqn_matrix& grad, const sqn_matrix& x, const sqn_matrix& w, const sqn_matrix* pre,
                                 int32_t act, const sqn_dropout_mask* mask, const LayerGradients& to, void* workspace,
                                 hipStream_t stream)
{
    const GradientScratch scratch(grad, x, w, act, mask && mask->p != 0.0, to.x, to.w, to.bias);
    const uint32_t terms = scratch.terms;
    char* work = static_cast<char*>(workspace);
    const int64_t points = x.rows, units = w.rows;
    const Mask m = mask_of(mask, units);
    sqn_matrix dz = grad;
    char* const dz_at = work;
    work += scratch.dz;
    float* const sums = scratch.sums ? reinterpret_cast<float*>(work) : nullptr;
    work += scratch.sums;
    if (scratch.own_dz) {
        dz.data = dz_at;
        dz.dtype = terms == 3 ? SQN_BF16 : x.dtype;
        dz.cols = dz.row_stride = round_up(units, Elements<X>::PIECE);
    }
    Finish f{};
    f.scale = m.scale;
    f.units = static_cast<uint32_t>(x.cols);
    if (to.x && points) {
        f.out = to.x->data;
        f.out_stride = to.x->row_stride;
    }
    const SlopePlan plan(points, units);
    uint32_t groups = plan.groups;       // of the bias's sums
    const bool sloped = scratch.narrow && (scratch.own_dz || to.bias) && narrow_sloped(grad, x, w, pre);
    if (sloped) {
        groups = launch_sloped<X>(w, grad, pre, act, m, scratch.own_dz && to.w ? dz.data : nullptr, dz.cols, scratch.dz_apart,
                                  terms == 2, to.bias ? sums : nullptr, f, stream);
    } else if (points && (scratch.own_dz || to.bias)) {
        SlopeParams p{};
        p.grad = grad.data;
        p.grad_stride = grad.row_stride;
        p.pre = pre ? pre->data : nullptr;
        p.pre_stride = pre ? pre->row_stride : 0;
        p.dz = scratch.own_dz ? dz.data : nullptr;
        p.apart = scratch.dz_apart;
        p.sums = sums;
        p.points = static_cast<uint32_t>(points);
        p.units = static_cast<uint32_t>(units);
        p.pitch = static_cast<uint32_t>(scratch.own_dz ? dz.cols : units);
        p.rows = plan.rows;
        p.across = plan.across;
        if (to.bias && plan.groups == 1) {
            p.bias = to.bias;
            p.bias_dtype = to.bias_dtype;
        }
        p.act = static_cast<uint32_t>(act);
        p.mask = m;
        const dim3 grid(((p.pitch + 7) / 8 + p.across - 1) / p.across, plan.groups);
        launch_slopes<X>(p, grad.dtype == SQN_F32, terms > 1, grid, stream);
    }
    auto parted = [&](Operand o) {
        o.apart = scratch.dz_apart;
        o.low = terms > 1 ? kLowOfDz : 0;
        return o;
    };
    ProductParams of_x{}, of_w{};
    PartsParams left_x{}, left_w{};
    left_x.parts = left_w.parts = 1;     // nothing
    bool tiles_x = false;
    if (sloped) {
        // the points' gradient came with dz
    } else if (scratch.narrow && terms == 1) {
        launch_narrow<X, X, false, true>(w, dz, units, f, work, stream);
    } else if (to.x && points) {
        tiles_x = true;
        const Operand a = factor_across(w, terms, work, stream);
        of_x = product_of(a, parted(along(dz)), points, scratch.plan_x, f, work, terms);
        work += scratch.partial_x;
        left_x = parts_of(of_x);
    }
    if (to.w) {
        const Operand a = factor_across(x, terms, work, stream);
        f.out = to.w->data;
        f.out_stride = to.w->row_stride;
        of_w = product_of(a, parted(across(dz)), units, scratch.plan_w, f, work, terms);
        left_w = parts_of(of_w);
    }
    const ProductParams *const dx = tiles_x ? &of_x : nullptr, *const dw = to.w ? &of_w : nullptr;
    if (terms == 1)
        launch_products<X, X, false>(dx, dw, scratch, stream);
    else if constexpr (sizeof(X) == 2)
        launch_products<__bf16, X, true>(dx, dw, scratch, stream);
    // the bias's sums of one group have been added up, of none they are zeros
    const BiasParams bias = {sums, to.bias, groups, static_cast<uint32_t>(units), to.bias_dtype, m.scale};
    const uint32_t bias_groups = to.bias && groups != 1 ? static_cast<uint32_t>((units + kSumUnits - 1) / kSumUnits) : 0;
    const uint32_t all = groups_of(left_x) + groups_of(left_w) + bias_groups;
    if (all)
        sums_kernel<X><<<all, kThreads, 0, stream>>>(left_x, left_w, bias, groups_of(left_x), groups_of(left_w));
    return hipGetLastError();
}

}  // namespace

size_t layer_bytes(const sqn_matrix& x, const sqn_matrix& w)
{
    if (x.rows <= kFewPoints)
        return 0;
    if (narrow_of(w, w.rows, x.cols, x.rows, in_place(x)))
        return narrow_pack_bytes(x);
    return pack_bytes(x) + pack_bytes(w) + plan_of(w.rows, x.rows, x.cols, x.dtype).bytes;
}

hipError_t launch_layer(const sqn_matrix& x, const sqn_matrix& w, const sqn_epilogue& e, const sqn_matrix& out, void* workspace,
                        hipStream_t stream)
{
    Finish f{};
    f.bias = e.bias;
    f.bias_f32 = e.bias_dtype == SQN_F32 ? 1 : 0;
    f.act = static_cast<uint32_t>(e.activation);
    f.units = static_cast<uint32_t>(w.rows);
    f.mask = mask_of(e.dropout, w.rows);
    if (e.residual) {
        f.residual = e.residual->data;
        f.residual_stride = e.residual->row_stride;
    }
    if (e.pre) {
        f.pre = e.pre->data;
        f.pre_stride = e.pre->row_stride;
    }
    f.out = out.data;
    f.out_stride = out.row_stride;
    char* work = static_cast<char*>(workspace);
    if (x.dtype == SQN_F32)
        launch_layer_typed<float, float>(x, w, f, work, stream);
    else if (x.dtype == SQN_F16 && out.dtype == SQN_F32)
        launch_layer_typed<_Float16, float>(x, w, f, work, stream);
    else if (x.dtype == SQN_F16)
        launch_layer_typed<_Float16, _Float16>(x, w, f, work, stream);
    else if (out.dtype == SQN_F32)
        launch_layer_typed<__bf16, float>(x, w, f, work, stream);
    else
        launch_layer_typed<__bf16, __bf16>(x, w, f, work, stream);
    return hipGetLastError();
}

size_t layer_gradient_bytes(const sqn_matrix& grad, const sqn_matrix& x, const sqn_matrix& w, int32_t act, bool masked, bool for_x,
                            bool for_w, bool for_bias)
{
    return GradientScratch(grad, x, w, act, masked, for_x, for_w, for_bias).bytes();
}

hipError_t launch_layer_gradient(const sqn_matrix& grad, const sqn_matrix& x, const sqn_matrix& w, const sqn_matrix* pre,
                                 int32_t act, const sqn_dropout_mask* mask, const LayerGradients& to, void* workspace,
                                 hipStream_t stream)
{
    if (x.dtype == SQN_F32)
        return launch_gradient_typed<float>(grad, x, w, pre, act, mask, to, workspace, stream);
    if (x.dtype == SQN_F16)
        return launch_gradient_typed<_Float16>(grad, x, w, pre, act, mask, to, workspace, stream);
    return launch_gradient_typed<__bf16>(grad, x, w, pre, act, mask, to, workspace, stream);
}

}  // namespace sqn
