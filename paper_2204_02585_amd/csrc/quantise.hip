// Matrices in 4-bit blocks (MXFP4: 32 E2M1 elements and an E8M0 scale) and
// the layers evaluated on them.
#include "learn.h"
#include "numeric.h"
#include "sqn_internal.h"

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

// The largest magnitude's exponent field (0 for subnormals and zero) to the
// block's scale byte; 255 marks a NaN or an infinity.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits)
{
    const uint32_t e = top_bits >> 23;
    return e == 255 ? 255u : e > 2 ? e - 2 : 0u;
}

// Eight elements over 2^(byte - 127), as codes.  The product is exact up to
// elements too small to matter; the conversion rounds to nearest even and
// stops at 6.
__device__ __forceinline__ uint32_t encode8(const float v[8], uint32_t byte)
{
    const float inv = byte == 255 ? 0.0f : __uint_as_float((254 - byte) << 23);
    uint32_t c = 0;
    float s[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
        s[k] = byte == 255 ? 0.0f : v[k] * inv;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[0], s[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[2], s[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[4], s[5], 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, s[6], s[7], 1.0f, 3);
    return c;
}

// Elements at..at+8 of a row, zeros past its end.
template <typename T>
__device__ __forceinline__ void load_eight(const T* row, uint32_t at, uint32_t cols, float v[8])
{
    if (at + 8 <= cols) {
        load_run<T, 8>(row + at, v);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = at + k < cols ? to_f32(row[at + k]) : 0.0f;
    }
}

// The scale byte of the four lanes' elements.
__device__ __forceinline__ uint32_t shared_scale(const float v[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 1)));
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 2)));
    return scale_byte(top);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void quantise_kernel(QuantParams p)
{
    const uint32_t per_row = 4 * p.blocks;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.items;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t r = i / per_row;
        const uint32_t q = static_cast<uint32_t>(i - r * per_row);
        float v[8];
        load_eight<T>(static_cast<const T*>(p.x) + r * p.stride, 8 * q, p.cols, v);
        const uint32_t byte = shared_scale(v);
        reinterpret_cast<uint32_t*>(p.codes)[i] = encode8(v, byte);
        if ((i & 3) == 0)
            p.scales[i >> 2] = static_cast<uint8_t>(byte);
    }
}

// the magnitude of a 3-bit code, from the bits of binary32: subnormal 0.5, then 1 + m / 2
__device__ __forceinline__ float decode1(uint32_t code)
{
    const uint32_t m = code & 7;
    const float mag = m < 2 ? 0.5f * m : __uint_as_float(((m >> 1) + 126) << 23 | (m & 1) << 22);
    return __uint_as_float(__float_as_uint(mag) | (code & 8) << 28);
}

// 2^(byte - 127); NaN for 255
__device__ __forceinline__ float decode_scale(uint32_t byte)
{
    return byte == 255 ? __builtin_nanf("") : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void values_kernel(QuantParams p)
{
    const uint32_t per_row = 4 * p.blocks;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * kThreads + threadIdx.x; i < p.items;
         i += static_cast<uint64_t>(gridDim.x) * kThreads) {
        const uint64_t r = i / per_row;
        const uint32_t at = 8 * static_cast<uint32_t>(i - r * per_row);
        const uint32_t c = reinterpret_cast<const uint32_t*>(p.codes)[i];
        const float scale = decode_scale(p.scales[i >> 2]);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = decode1(c >> (4 * k)) * scale;
        T* row = static_cast<T*>(p.values) + r * p.stride;
        if (at + 8 <= p.cols) {
            store_run<T, 8>(row + at, v);
        } else {
            for (uint32_t k = 0; at + k < p.cols; ++k)
                row[at + k] = from_f32<T>(v[k]);
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
// out^T = W x^T on v_mfma_scale_f32_16x16x128_f8f6f4: W is the first factor,
// so a lane ends with four consecutive units of one point.  A lane's share of
// a factor is one block of one row, 16 bytes, with its scale.

struct ProductParams {
    const uint8_t *x, *x_scales, *w, *w_scales;
    const float* bias;
    void* out;
    int64_t out_stride;
    uint32_t points, units, blocks;
    int32_t relu, dtype;
};

struct Fragment {
    int8v codes;
    int scale;
};

__device__ __forceinline__ Fragment load_fragment(const uint8_t* codes, const uint8_t* scales, uint32_t row,
                                                  uint32_t block, uint32_t blocks)
{
    Fragment f;
    int4v c = {0, 0, 0, 0};
    f.scale = kOne;
    if (block < blocks) {
        const uint64_t at = static_cast<uint64_t>(row) * blocks + block;
        c = *reinterpret_cast<const int4v*>(codes + 16 * at);
        f.scale = scales[at];
    }
    f.codes = int8v{c[0], c[1], c[2], c[3], 0, 0, 0, 0};
    return f;
}

__device__ __forceinline__ float4v multiply(const Fragment& a, const Fragment& b, float4v acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.codes, b.codes, acc, 4, 4, 0, a.scale, 0, b.scale);
}

// Bias and activation; the store is of the units inside the matrix.
__device__ __forceinline__ void finish4(const ProductParams& p, uint32_t unit, uint32_t point, float4v acc)
{
    if (point >= p.points)
        return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (unit + q >= p.units)
            return;
        float v = acc[q];
        if (p.bias)
            v += p.bias[unit + q];
        if (p.relu)
            v = v < 0.0f ? 0.0f : v;
        const int64_t at = point * p.out_stride + unit + q;
        if (p.dtype == SQN_F32)
            static_cast<float*>(p.out)[at] = v;
        else if (p.dtype == SQN_F16)
            static_cast<_Float16*>(p.out)[at] = static_cast<_Float16>(v);
        else
            static_cast<__bf16*>(p.out)[at] = static_cast<__bf16>(v);
    }
}

__global__ __launch_bounds__(kThreads) void product_kernel(ProductParams p)
{
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t point_tiles = (p.points + 63) / 64;
    const uint32_t ti = blockIdx.x / point_tiles, tj = blockIdx.x - ti * point_tiles;
    const uint32_t unit0 = ti * 64 + (wave & 1) * 32, point0 = tj * 64 + (wave >> 1) * 32;
    uint32_t unit[2], point[2];
    float4v acc[2][2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        // rows past the end read the last one, and are not stored
        unit[s] = min(unit0 + 16 * s + (lane & 15), p.units - 1);
        point[s] = min(point0 + 16 * s + (lane & 15), p.points - 1);
#pragma unroll
        for (int t = 0; t < 2; ++t)
            acc[s][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (uint32_t k = lane >> 4; k < (p.blocks + 3) / 4 * 4; k += 4) {
        Fragment a[2], b[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            a[s] = load_fragment(p.w, p.w_scales, unit[s], k, p.blocks);
            b[s] = load_fragment(p.x, p.x_scales, point[s], k, p.blocks);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 0; t < 2; ++t)
                acc[s][t] = multiply(a[s], b[t], acc[s][t]);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int t = 0; t < 2; ++t)
            finish4(p, unit0 + 16 * s + 4 * (lane >> 4), point0 + 16 * t + (lane & 15), acc[s][t]);
}

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

}  // namespace

hipError_t launch_quantise(const sqn_matrix& x, const sqn_quantised& out, hipStream_t stream)
{
    QuantParams p;
    p.x = x.data;
    p.values = nullptr;
    p.codes = static_cast<uint8_t*>(out.codes);
    p.scales = static_cast<uint8_t*>(out.scales);
    p.stride = x.row_stride;
    p.cols = static_cast<uint32_t>(x.cols);
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.items = static_cast<uint64_t>(x.rows) * p.blocks * 4;
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
                                    const sqn_matrix& out, hipStream_t stream)
{
    ProductParams p;
    p.x = static_cast<const uint8_t*>(x.codes);
    p.x_scales = static_cast<const uint8_t*>(x.scales);
    p.w = static_cast<const uint8_t*>(w.codes);
    p.w_scales = static_cast<const uint8_t*>(w.scales);
    p.bias = bias;
    p.out = out.data;
    p.out_stride = out.row_stride;
    p.points = static_cast<uint32_t>(x.rows);
    p.units = static_cast<uint32_t>(w.rows);
    p.blocks = static_cast<uint32_t>(quant_blocks(x.cols));
    p.relu = relu ? 1 : 0;
    p.dtype = out.dtype;
    product_kernel<<<(p.points + 63) / 64 * ((p.units + 63) / 64), kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

size_t quantised_layer_bytes(int64_t rows, int64_t cols)
{
    const size_t blocks = static_cast<size_t>(rows) * quant_blocks(cols);
    return padded(16 * blocks) + padded(blocks);
}

hipError_t launch_quantised_layer(const sqn_matrix& x, const sqn_quantised& w, const float* bias, bool relu,
                                  const sqn_matrix& out, void* workspace, hipStream_t stream)
{
    sqn_quantised q;
    q.rows = x.rows;
    q.cols = x.cols;
    q.codes = workspace;
    q.scales = static_cast<char*>(workspace) + padded(16 * static_cast<size_t>(x.rows) * quant_blocks(x.cols));
    const hipError_t e = launch_quantise(x, q, stream);
    if (e != hipSuccess)
        return e;
    return launch_quantised_product(q, w, bias, relu, out, stream);
}

}  // namespace sqn
