// Rows of a learned table by index, and the table's gradient.
//
//   lookup    out[t] = scale W[id_t]
//   gradient  dW[v] = scale sum over the t with id_t = v of g[t]
//
// Both move bytes and compute next to nothing.  The gradient's sums must not
// depend on the order in which the GPU gets to the rows, so the positions are
// sorted by index (a stable radix sort), cut into tiles of the sorted order,
// and each tile sums its runs of equal indices; runs that cross tiles leave
// partial sums that a second kernel joins in tile order.
#include "learn.h"
#include "numeric.h"
#include "sqn_internal.h"

namespace sqn {
namespace {

constexpr int kThreads = 256;

// ---- lookup

struct LookupParams {
    const void* table;
    const void* ids;
    void* out;
    uint64_t rows;                      // of the table
    int64_t table_stride, out_stride;   // elements
    uint64_t items;                     // runs in the output: n * runs
    uint32_t per_block;                 // runs a workgroup copies
    uint32_t runs, cols;                // runs per row
    float scale;
};

// A thread copies runs of V elements (16 bytes); the last run of a row ends
// with it and may overlap the one before, whose elements it writes again with
// the same values.
template <typename T, typename I, int V>
__global__ __launch_bounds__(kThreads) void lookup_kernel(LookupParams p)
{
    const uint64_t start = static_cast<uint64_t>(blockIdx.x) * p.per_block;
    const uint64_t t0 = start / p.runs;
    const uint32_t c0 = static_cast<uint32_t>(start - t0 * p.runs);
    const uint64_t left = p.items - start;
    const uint32_t n = left < p.per_block ? static_cast<uint32_t>(left) : p.per_block;
    const I* ids = static_cast<const I*>(p.ids) + t0;
    const T* table = static_cast<const T*>(p.table);
    T* out = static_cast<T*>(p.out) + t0 * p.out_stride;
    for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t r = (c0 + i) / p.runs;
        const uint32_t e = min((c0 + i - r * p.runs) * V, p.cols - V);
        const int64_t id = ids[r];
        float v[V];
        if (static_cast<uint64_t>(id) < p.rows) {
            load_run<T, V>(table + id * p.table_stride + e, v);
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] *= p.scale;
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] = 0.0f;
        }
        store_run<T, V>(out + r * p.out_stride + e, v);
    }
}

template <typename T>
hipError_t lookup(const LookupParams& base, bool ids64, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    LookupParams p = base;
    const bool wide = p.cols >= V;
    p.runs = wide ? (p.cols + V - 1) / V : p.cols;
    p.items *= p.runs;
    p.per_block = 1024;
    // rows < 2^31 and cols <= 2^20: at most 2^31 2^20 / 1024 workgroups is more
    // than a grid takes, so long outputs give each more
    while ((p.items + p.per_block - 1) / p.per_block > 0x400000u && p.per_block < (1u << 30))
        p.per_block *= 2;
    const dim3 grid(static_cast<uint32_t>((p.items + p.per_block - 1) / p.per_block));
    if (wide) {
        if (ids64)
            lookup_kernel<T, int64_t, V><<<grid, kThreads, 0, stream>>>(p);
        else
            lookup_kernel<T, int32_t, V><<<grid, kThreads, 0, stream>>>(p);
    } else {
        if (ids64)
            lookup_kernel<T, int64_t, 1><<<grid, kThreads, 0, stream>>>(p);
        else
            lookup_kernel<T, int32_t, 1><<<grid, kThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

// ---- gradient: sorting
//
// Least significant digit first, kDigitBits a pass; each pass counts the
// digits of every workgroup's stretch of keys, then places them.  Within a
// stretch a wave takes consecutive keys, 64 at a time; equal digits among the
// 64 find their order with one ballot per bit.  Indices outside the table
// sort as the key `rows`, behind all others.
//
// While it sorts the chip is nearly idle, so the rows of the gradient are
// cleared by further workgroups of the same launches.

constexpr int kDigitBits = 8;
constexpr int kBins = 1 << kDigitBits;
constexpr int kWaves = kThreads / 64;
constexpr int kKeysPerThread = 16;
constexpr int kStep = kThreads * kKeysPerThread;    // keys a workgroup places at a time
constexpr int kMaxStretches = 256;

struct Clear {
    char* data;
    uint64_t row_bytes, stride_bytes, rows;
    uint64_t first, last;               // 16-byte pieces of all rows, this launch's share
    uint32_t blocks;                    // workgroups that clear
};

struct SortParams {
    const void* ids;                    // first pass: the indices
    const uint32_t* keys_in;            // later passes
    const uint32_t* at_in;
    uint32_t* keys_out;
    uint32_t* at_out;
    uint32_t* counts;                   // [kBins][stretches]
    uint32_t n, rows;
    uint32_t stretch;                   // keys per workgroup, a multiple of kStep
    uint32_t stretches;
    int shift;
    Clear clear;
};

// Zeros over this workgroup's share of the pieces; a row's last piece ends
// with the row and may overlap the one before.
__device__ void clear_share(const Clear& c, uint32_t block)
{
    struct __attribute__((packed, aligned(2))) Piece { uint32_t w[4]; };
    const uint64_t per_row = (c.row_bytes + 15) / 16;
    for (uint64_t i = c.first + static_cast<uint64_t>(block) * kThreads + threadIdx.x; i < c.last;
         i += static_cast<uint64_t>(c.blocks) * kThreads) {
        const uint64_t r = c.rows == 1 ? 0 : i / per_row;
        const uint64_t at = (i - r * per_row) * 16;
        char* row = c.data + r * c.stride_bytes;
        if (c.row_bytes >= 16) {
            *reinterpret_cast<Piece*>(row + min(at, c.row_bytes - 16)) = Piece{{0, 0, 0, 0}};
        } else {
            for (uint64_t b = 0; b < c.row_bytes; b += 2)
                *reinterpret_cast<uint16_t*>(row + b) = 0;
        }
    }
}

template <typename I>
__device__ __forceinline__ uint32_t key_of(const SortParams& p, uint32_t i)
{
    if constexpr (sizeof(I) == 1) {      // later passes
        return p.keys_in[i];
    } else {
        const int64_t id = static_cast<const I*>(p.ids)[i];
        return static_cast<uint64_t>(id) < p.rows ? static_cast<uint32_t>(id) : p.rows;
    }
}

template <typename I>
__global__ __launch_bounds__(kThreads) void count_kernel(SortParams p)
{
    if (blockIdx.x >= p.stretches) {
        clear_share(p.clear, blockIdx.x - p.stretches);
        return;
    }
    __shared__ uint32_t bins[kBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * p.stretch;
    const uint32_t last = min(p.n, first + p.stretch);
    for (uint32_t i = first + threadIdx.x; i < last; i += kThreads)
        atomicAdd(&bins[(key_of<I>(p, i) >> p.shift) & (kBins - 1)], 1u);
    __syncthreads();
    p.counts[threadIdx.x * p.stretches + blockIdx.x] = bins[threadIdx.x];
}

template <typename I>
__global__ __launch_bounds__(kThreads) void place_kernel(SortParams p)
{
    if (blockIdx.x >= p.stretches) {
        clear_share(p.clear, blockIdx.x - p.stretches);
        return;
    }
    __shared__ uint32_t base[kBins];             // where the stretch's next key of a digit goes
    __shared__ uint32_t seen[kWaves][kBins];     // of a step, per wave
    __shared__ uint32_t sums[kBins];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // this digit's keys in all stretches, and in those before this one
    uint32_t total = 0, before = 0;
    for (uint32_t s = 0; s < p.stretches; ++s) {
        const uint32_t c = p.counts[tid * p.stretches + s];
        before += s < blockIdx.x ? c : 0;
        total += c;
    }
    sums[tid] = total;
    __syncthreads();
    for (int d = 1; d < kBins; d *= 2) {
        const uint32_t add = tid >= d ? sums[tid - d] : 0;
        __syncthreads();
        sums[tid] += add;
        __syncthreads();
    }
    base[tid] = sums[tid] - total + before;

    const uint32_t first = blockIdx.x * p.stretch;
    const uint32_t last = min(p.n, first + p.stretch);
    for (uint32_t step = first; step < last; step += kStep) {
        for (int w = 0; w < kWaves; ++w)
            seen[w][tid] = 0;
        __syncthreads();
        uint32_t key[kKeysPerThread], rank[kKeysPerThread];
        const uint32_t mine = step + wave * (64 * kKeysPerThread) + lane;
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k)
            key[k] = mine + 64 * k < last ? key_of<I>(p, mine + 64 * k) : 0;
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k) {
            const bool there = mine + 64 * k < last;
            const uint32_t digit = (key[k] >> p.shift) & (kBins - 1);
            uint64_t same = __ballot(there);
#pragma unroll
            for (int b = 0; b < kDigitBits; ++b) {
                const uint64_t set = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? set : ~set;
            }
            // the wave's LDS accesses stay in program order
            const uint32_t had = seen[wave][digit];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            const uint64_t lower = same & ((uint64_t{1} << lane) - 1);
            rank[k] = had + __popcll(lower);
            if (there && lower == 0)
                seen[wave][digit] = had + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        // counts of the step to starts, wave after wave
        uint32_t at = base[tid];
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = seen[w][tid];
            seen[w][tid] = at;
            at += c;
        }
        base[tid] = at;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kKeysPerThread; ++k) {
            const uint32_t i = mine + 64 * k;
            if (i < last) {
                const uint32_t to = seen[wave][(key[k] >> p.shift) & (kBins - 1)] + rank[k];
                p.keys_out[to] = key[k];
                p.at_out[to] = sizeof(I) == 1 ? p.at_in[i] : i;
            }
        }
        __syncthreads();
    }
}

// ---- gradient: sums

struct SumParams {
    const uint32_t* keys;      // sorted
    const uint32_t* at;
    const void* grad;
    void* out;
    float* head;               // [tiles][width]: a tile's part of a run begun before it
    float* tail;               // [tiles][width]: of a run begun in it that goes on after it
    int64_t grad_stride, out_stride;
    uint32_t n, rows, cols;
    uint32_t tile, tiles;      // sorted entries per tile
    uint32_t runs, width;      // runs of V elements per row; width = runs V
    uint32_t lanes;            // lanes per tile, a power of two up to 64
    float scale;
    int accumulate;
};

// The run's elements of the gradient's row: scaled, added where asked.
// Elements below `skip` belong to the run before, which writes them.
template <typename O, int V>
__device__ __forceinline__ void finish(const SumParams& p, uint32_t key, uint32_t e, uint32_t skip, const float acc[V])
{
    O* to = static_cast<O*>(p.out) + key * p.out_stride + e;
    float v[V];
    if (skip == 0) {
        if (p.accumulate) {
            load_run<O, V>(to, v);
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] = __builtin_fmaf(acc[k], p.scale, v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[k] = acc[k] * p.scale;
        }
        store_run<O, V>(to, v);
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (k >= static_cast<int>(skip))
                to[k] = from_f32<O>(p.accumulate ? __builtin_fmaf(acc[k], p.scale, to_f32(to[k])) : acc[k] * p.scale);
    }
}

template <typename T, typename O, int V>
__global__ __launch_bounds__(kThreads) void sum_kernel(SumParams p)
{
    const uint32_t group = (blockIdx.x * kThreads + threadIdx.x) / p.lanes;
    const uint32_t c = blockIdx.y * p.lanes + threadIdx.x % p.lanes;
    if (group >= p.tiles || c >= p.runs)
        return;
    const uint32_t e = min(c * V, p.cols - V), skip = c * V - e;
    const uint32_t first = group * p.tile, last = min(p.n, first + p.tile);
    const T* grad = static_cast<const T*>(p.grad) + e;
    uint32_t key = p.keys[first];
    bool before = first > 0 && p.keys[first - 1] == key;
    float acc[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        acc[k] = 0.0f;
    auto part = [&](float* to) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            to[static_cast<uint64_t>(group) * p.width + c * V + k] = acc[k];
    };
    for (uint32_t i = first; i < last; ++i) {
        const uint32_t next = p.keys[i];
        if (next != key) {
            if (before)
                part(p.head);
            else
                finish<O, V>(p, key, e, skip, acc);
            before = false;
            key = next;
#pragma unroll
            for (int k = 0; k < V; ++k)
                acc[k] = 0.0f;
        }
        if (key >= p.rows)
            return;                     // indices outside the table come last
        float v[V];
        load_run<T, V>(grad + p.at[i] * p.grad_stride, v);
#pragma unroll
        for (int k = 0; k < V; ++k)
            acc[k] += v[k];
    }
    if (before)
        part(p.head);
    else if (last < p.n && p.keys[last] == key)
        part(p.tail);
    else
        finish<O, V>(p, key, e, skip, acc);
}

// A tile whose last run began in it and goes on: that run's parts in order.
template <typename O, int V>
__global__ __launch_bounds__(kThreads) void join_kernel(SumParams p)
{
    const uint32_t group = (blockIdx.x * kThreads + threadIdx.x) / p.lanes;
    const uint32_t c = blockIdx.y * p.lanes + threadIdx.x % p.lanes;
    if (group + 1 >= p.tiles || c >= p.runs)
        return;
    const uint32_t first = group * p.tile, last = first + p.tile;
    const uint32_t key = p.keys[last - 1];
    if (p.keys[last] != key || key >= p.rows)
        return;
    if (first > 0 && p.keys[first - 1] == key)
        return;                         // begun in a tile before
    float acc[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        acc[k] = p.tail[static_cast<uint64_t>(group) * p.width + c * V + k];
    for (uint32_t t = group + 1; t < p.tiles && p.keys[t * p.tile] == key; ++t) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            acc[k] += p.head[static_cast<uint64_t>(t) * p.width + c * V + k];
    }
    const uint32_t e = min(c * V, p.cols - V);
    finish<O, V>(p, key, e, c * V - e, acc);
}

// ---- gradient: layout and launches

constexpr uint32_t kTile = 32;

struct Plan {
    uint32_t passes, stretch, stretches, tiles, width;
    size_t keys[2], at[2], counts, head, tail, bytes;
};

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

Plan plan_of(int64_t n, int64_t rows, int64_t cols)
{
    Plan q;
    int bits = 1;
    while ((rows >> bits) != 0)
        ++bits;                          // the largest key is `rows`
    q.passes = (bits + kDigitBits - 1) / kDigitBits;
    const int64_t steps = (n + kStep - 1) / kStep;
    q.stretch = static_cast<uint32_t>((steps + kMaxStretches - 1) / kMaxStretches * kStep);
    q.stretches = q.stretch ? static_cast<uint32_t>((n + q.stretch - 1) / q.stretch) : 0;
    q.tiles = static_cast<uint32_t>((n + kTile - 1) / kTile);
    q.width = static_cast<uint32_t>((cols + 7) / 8 * 8);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += padded(bytes);
        return here;
    };
    for (int k = 0; k < 2; ++k) {
        q.keys[k] = take(4 * static_cast<size_t>(n));
        q.at[k] = take(4 * static_cast<size_t>(n));
    }
    q.counts = take(4 * static_cast<size_t>(kBins) * q.stretches);
    q.head = take(4 * static_cast<size_t>(q.tiles) * q.width);
    q.tail = take(4 * static_cast<size_t>(q.tiles) * q.width);
    q.bytes = at;
    return q;
}

template <typename T, typename O, int V>
void launch_sums(SumParams p, hipStream_t stream)
{
    p.runs = (p.cols + V - 1) / V;
    p.width = p.runs * V;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < p.runs)
        p.lanes *= 2;
    const uint32_t per_block = kThreads / p.lanes;
    const dim3 grid((p.tiles + per_block - 1) / per_block, (p.runs + p.lanes - 1) / p.lanes);
    sum_kernel<T, O, V><<<grid, kThreads, 0, stream>>>(p);
    if (p.tiles > 1)
        join_kernel<O, V><<<grid, kThreads, 0, stream>>>(p);
}

template <typename T, typename O>
void launch_sums_of(const SumParams& p, hipStream_t stream)
{
    constexpr int V = sizeof(T) == 4 ? 4 : 8;
    if (p.cols >= V)
        launch_sums<T, O, V>(p, stream);
    else
        launch_sums<T, O, 1>(p, stream);
}

template <typename T>
void launch_sums_from(const SumParams& p, int32_t out_dtype, hipStream_t stream)
{
    if (out_dtype == SQN_F32)
        launch_sums_of<T, float>(p, stream);
    else if (out_dtype == SQN_F16)
        launch_sums_of<T, _Float16>(p, stream);
    else
        launch_sums_of<T, __bf16>(p, stream);
}

}  // namespace

hipError_t launch_lookup(const sqn_matrix& table, const void* ids, bool ids64, float scale, const sqn_matrix& out,
                         hipStream_t stream)
{
    LookupParams p;
    p.table = table.data;
    p.ids = ids;
    p.out = out.data;
    p.rows = static_cast<uint64_t>(table.rows);
    p.table_stride = table.row_stride;
    p.out_stride = out.row_stride;
    p.items = static_cast<uint64_t>(out.rows);
    p.cols = static_cast<uint32_t>(table.cols);
    p.scale = scale;
    if (table.dtype == SQN_F32)
        return lookup<float>(p, ids64, stream);
    if (table.dtype == SQN_F16)
        return lookup<_Float16>(p, ids64, stream);
    return lookup<__bf16>(p, ids64, stream);
}

size_t lookup_gradient_bytes(int64_t n, int64_t rows, int64_t cols) { return plan_of(n, rows, cols).bytes; }

hipError_t launch_lookup_gradient(const sqn_matrix& grad, const void* ids, bool ids64, float scale, bool accumulate,
                                  const sqn_matrix& table_grad, void* workspace, hipStream_t stream)
{
    const Plan q = plan_of(grad.rows, table_grad.rows, table_grad.cols);
    char* ws = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + q.keys[0]), reinterpret_cast<uint32_t*>(ws + q.keys[1])};
    uint32_t* at[2] = {reinterpret_cast<uint32_t*>(ws + q.at[0]), reinterpret_cast<uint32_t*>(ws + q.at[1])};

    SortParams s;
    s.ids = ids;
    s.counts = reinterpret_cast<uint32_t*>(ws + q.counts);
    s.n = static_cast<uint32_t>(grad.rows);
    s.rows = static_cast<uint32_t>(table_grad.rows);
    s.stretch = q.stretch;
    s.stretches = q.stretches;
    Clear c;
    const size_t es = element_size(table_grad.dtype);
    c.data = static_cast<char*>(table_grad.data);
    c.row_bytes = static_cast<uint64_t>(table_grad.cols) * es;
    c.stride_bytes = static_cast<uint64_t>(table_grad.row_stride) * es;
    c.rows = static_cast<uint64_t>(table_grad.rows);
    if (c.stride_bytes == c.row_bytes) {
        c.row_bytes *= c.rows;
        c.rows = 1;
    }
    const uint64_t pieces = accumulate ? 0 : c.rows * ((c.row_bytes + 15) / 16);
    const uint32_t launches = s.n ? 2 * q.passes : 1;
    uint32_t launch = 0;
    auto share = [&]() {
        c.first = pieces / launches * launch;
        c.last = ++launch == launches ? pieces : pieces / launches * launch;
        const uint64_t want = (c.last - c.first + kThreads - 1) / kThreads;
        c.blocks = static_cast<uint32_t>(want < 2048 ? want : 2048);
        s.clear = c;
        return dim3(q.stretches + c.blocks);
    };
    if (s.n == 0) {
        const dim3 grid = share();
        if (grid.x)
            count_kernel<uint8_t><<<grid, kThreads, 0, stream>>>(s);
        return hipGetLastError();
    }
    for (uint32_t pass = 0; pass < q.passes; ++pass) {
        s.shift = static_cast<int>(pass) * kDigitBits;
        s.keys_in = keys[(pass + 1) & 1];
        s.at_in = at[(pass + 1) & 1];
        s.keys_out = keys[pass & 1];
        s.at_out = at[pass & 1];
        const dim3 count_grid = share();
        if (pass > 0)
            count_kernel<uint8_t><<<count_grid, kThreads, 0, stream>>>(s);
        else if (ids64)
            count_kernel<int64_t><<<count_grid, kThreads, 0, stream>>>(s);
        else
            count_kernel<int32_t><<<count_grid, kThreads, 0, stream>>>(s);
        const dim3 place_grid = share();
        if (pass > 0)
            place_kernel<uint8_t><<<place_grid, kThreads, 0, stream>>>(s);
        else if (ids64)
            place_kernel<int64_t><<<place_grid, kThreads, 0, stream>>>(s);
        else
            place_kernel<int32_t><<<place_grid, kThreads, 0, stream>>>(s);
    }
    SumParams p;
    p.keys = s.keys_out;
    p.at = s.at_out;
    p.grad = grad.data;
    p.out = table_grad.data;
    p.head = reinterpret_cast<float*>(ws + q.head);
    p.tail = reinterpret_cast<float*>(ws + q.tail);
    p.grad_stride = grad.row_stride;
    p.out_stride = table_grad.row_stride;
    p.n = s.n;
    p.rows = s.rows;
    p.cols = static_cast<uint32_t>(grad.cols);
    p.tile = kTile;
    p.tiles = q.tiles;
    p.scale = scale;
    p.accumulate = accumulate ? 1 : 0;
    if (grad.dtype == SQN_F32)
        launch_sums_from<float>(p, table_grad.dtype, stream);
    else if (grad.dtype == SQN_F16)
        launch_sums_from<_Float16>(p, table_grad.dtype, stream);
    else
        launch_sums_from<__bf16>(p, table_grad.dtype, stream);
    return hipGetLastError();
}

}  // namespace sqn
