// Rows of a learned table by index, and the table's gradient.
//
//   lookup    out[t] = scale W[id_t]
//   gradient  dW[v] = scale sum over the t with id_t = v of g[t]
//
// Both move bytes and compute next to nothing.  The gradient's sums must not
// depend on the order in which the GPU gets to the rows, so the positions are
// sorted by index (keeping their order where it is the same: by radix passes, or
// of fewer by buckets of rows), cut into tiles of the sorted order, and each
// tile sums its runs of equal indices; runs that cross tiles leave partial sums
// that a second kernel joins in tile order.  Very few indices take one launch.
#include <type_traits>

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

constexpr int kAhead = 4;        // runs of a thread under way together

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
    for (uint32_t i0 = threadIdx.x; i0 < n; i0 += kAhead * kThreads) {
        // the loads of all runs first
        float v[kAhead][V];
        int64_t id[kAhead];
        uint32_t r[kAhead], e[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const uint32_t i = min(i0 + a * kThreads, n - 1);
            r[a] = (c0 + i) / p.runs;
            e[a] = min((c0 + i - r[a] * p.runs) * V, p.cols - V);
            id[a] = ids[r[a]];
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            load_run<T, V>(table + (static_cast<uint64_t>(id[a]) < p.rows ? id[a] : 0) * p.table_stride + e[a], v[a]);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const bool inside = static_cast<uint64_t>(id[a]) < p.rows;
#pragma unroll
            for (int k = 0; k < V; ++k)
                v[a][k] = inside ? v[a][k] * p.scale : 0.0f;
            if (i0 + a * kThreads < n)
                store_run<T, V>(out + r[a] * p.out_stride + e[a], v[a]);
        }
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
// Least significant digit first, as few digits as ten bits each allow.  A pass
// counts the digits of every workgroup's stretch of keys, then places them.
// Within a stretch a wave takes consecutive keys, 64 at a time; equal digits
// among the 64 find their order with one ballot per bit.  Indices outside the
// table sort as the key `rows`, behind all others.  Fewer keys are
// sorted in one launch instead, by buckets of rows.
//
// While it sorts the chip is nearly idle, so the rows of the gradient are
// cleared by further workgroups of the same launches.

constexpr int kMaxDigitBits = 10;
constexpr int kMaxBins = 1 << kMaxDigitBits;
constexpr int kSortThreads = 1024;
// Keys that a thread places of a stretch.  Longer stretches leave CUs idle,
// shorter ones are spent on the counts of the stretches before (640,000 keys, us
// a pass: 16 keys a thread 25, 8 keys 22).
constexpr int kPlaceKeys = 8;
constexpr int kPlaceStep = kSortThreads * kPlaceKeys;
constexpr int kMaxStretches = 128;
constexpr int kWaves = kSortThreads / 64;

// Of the counts of all stretches, which every stretch sums up: the threads that
// share a bin, and a thread's loads under way while it ranks a key.
constexpr uint32_t kMaxTurns = 8;
constexpr int kCountsAhead = 4;
static_assert(kPlaceKeys * kCountsAhead * (4 * kSortThreads / kMaxBins) >= kMaxStretches, "a step's keys see all counts");

struct __attribute__((aligned(8))) Pair {
    uint32_t key, at;
};

struct Clear {
    char* data;
    uint64_t row_bytes, stride_bytes, rows;
    uint64_t first, last;               // 16-byte pieces of all rows, this launch's share
    uint32_t blocks;                    // workgroups that clear
};

struct SortParams {
    const void* ids;                    // first pass: the indices
    const Pair* in;                     // later passes
    Pair* out;
    uint32_t* counts;                   // [stretches][bins]
    uint32_t n, rows;
    uint32_t stretch;                   // keys per workgroup, a multiple of kPlaceStep
    uint32_t stretches;
    int shift, bits;                    // of the digit
    Clear clear;
};

// Zeros over this workgroup's share of the pieces; a row's last piece ends
// with the row and may overlap the one before.
__device__ void clear_share(const Clear& c, uint32_t block)
{
    struct __attribute__((packed, aligned(2))) Piece { uint32_t w[4]; };
    const uint64_t per_row = (c.row_bytes + 15) / 16;
    for (uint64_t i = c.first + static_cast<uint64_t>(block) * blockDim.x + threadIdx.x; i < c.last;
         i += static_cast<uint64_t>(c.blocks) * blockDim.x) {
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

// the type of `ids` in the passes after the first
struct Sorted {};

template <typename I>
__device__ __forceinline__ uint32_t key_at(const void* ids, uint32_t i, uint32_t rows)
{
    const int64_t id = static_cast<const I*>(ids)[i];
    return static_cast<uint64_t>(id) < rows ? static_cast<uint32_t>(id) : rows;
}

template <typename I>
__device__ __forceinline__ Pair pair_at(const SortParams& p, uint32_t i)
{
    if constexpr (std::is_same<I, Sorted>::value)
        return p.in[i];
    else
        return Pair{key_at<I>(p.ids, i, p.rows), i};
}

// The number in its step of a thread's key k of KEYS: a wave's keys lie together.
template <int KEYS>
__device__ __forceinline__ uint32_t number_of(int k)
{
    return (threadIdx.x >> 6) * (64 * KEYS) + 64 * k + (threadIdx.x & 63);
}

// A step's digits, digit(k) a thread's k-th, ranked among the equal ones of their
// wave, which counts them in seen[digit]; keys from `n` on are not there.
// begin(k) and end(k) stand around the k-th key's ballots.
template <int KEYS, typename D, typename B, typename E>
__device__ __forceinline__ void rank_keys(D digit_of, uint32_t n, uint32_t* seen, uint32_t (&rank)[KEYS],
                                          B begin, E end)
{
    const uint64_t below = (uint64_t{1} << (threadIdx.x & 63)) - 1;
#pragma unroll
    for (int k = 0; k < KEYS; ++k) {
        begin(k);
        const bool there = number_of<KEYS>(k) < n;
        const uint32_t digit = digit_of(k);
        // lanes whose digit differs from this one's in some bit
        uint32_t other_low = 0, other_high = 0;
#pragma unroll
        for (int b = 0; b < kMaxDigitBits; ++b) {
            const uint32_t bit = static_cast<uint32_t>(static_cast<int32_t>(digit << (31 - b)) >> 31);   // 0 or all ones
            const uint64_t set = __ballot(bit != 0);
            other_low |= static_cast<uint32_t>(set) ^ bit;
            other_high |= static_cast<uint32_t>(set >> 32) ^ bit;
        }
        const uint64_t same = __ballot(there) & ~(static_cast<uint64_t>(other_high) << 32 | other_low);
        // the wave's LDS accesses stay in program order
        const uint32_t had = seen[digit];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        rank[k] = had + __popcll(same & below);
        if (there && (same & below) == 0)
            seen[digit] = had + __popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        end(k);
    }
}

// Exclusive sums over `bins` values, one a thread (0 from `bins` on).
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t v, uint32_t* wave_sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t t = __shfl_up(s, d);
        s += lane >= d ? t : 0;
    }
    __syncthreads();
    if (lane == 63)
        wave_sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w)
        before += wave_sums[w];
    return before + s - v;
}

// seen[wave][bin] from counts to where the wave's first key of the bin goes,
// given where the step's first goes; returns where the next step's does.
template <int BINS>
__device__ __forceinline__ uint32_t counts_to_starts(uint32_t (*seen)[BINS], uint32_t bin, uint32_t at)
{
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = seen[w][bin];
        seen[w][bin] = at;
        at += c;
    }
    return at;
}

template <typename I>
__global__ __launch_bounds__(kSortThreads) void count_kernel(SortParams p)
{
    if (blockIdx.x >= p.stretches) {
        clear_share(p.clear, blockIdx.x - p.stretches);
        return;
    }
    static_assert(kMaxBins == kSortThreads, "a bin a thread");
    __shared__ uint32_t bins[kMaxBins];
    bins[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t first = blockIdx.x * p.stretch;
    const uint32_t last = min(p.n, first + p.stretch);
    const uint32_t count = 1u << p.bits;
#pragma unroll 8
    for (uint32_t i = first + threadIdx.x; i < last; i += kSortThreads)
        atomicAdd(&bins[pair_at<I>(p, i).key >> p.shift & (count - 1)], 1u);
    __syncthreads();
    if (threadIdx.x < count)
        p.counts[blockIdx.x * count + threadIdx.x] = bins[threadIdx.x];
}

template <typename I>
__global__ __launch_bounds__(kSortThreads) void place_kernel(SortParams p)
{
    if (blockIdx.x >= p.stretches) {
        clear_share(p.clear, blockIdx.x - p.stretches);
        return;
    }
    __shared__ uint32_t seen[kWaves][kMaxBins];    // of a step, per wave
    __shared__ __align__(16) uint32_t sums[2][4 * kSortThreads];
    __shared__ uint32_t wave_sums[kWaves];
    const uint32_t bins = 1u << p.bits, tid = threadIdx.x, wave = tid >> 6;
    const uint32_t first = blockIdx.x * p.stretch;
    const uint32_t last = min(p.n, first + p.stretch);

    // All stretches' counts, for the keys of a bin in those before this one and
    // from it on: four bins a load, the stretches by the threads in turns, under
    // way while the first step's keys are ranked (640,000 keys: 22 us a pass with
    // the sums ahead of the ranks).
    const uint32_t quads = bins / 4, turns = min(kSortThreads / quads, kMaxTurns);
    const uint32_t turn = tid / quads, quad = tid % quads;
    const uint4* counts = reinterpret_cast<const uint4*>(p.counts) + quad;
    uint4 here[kCountsAhead], before{0, 0, 0, 0}, after{0, 0, 0, 0};
    auto add = [](uint4& to, const uint4& c) { to.x += c.x, to.y += c.y, to.z += c.z, to.w += c.w; };

    uint32_t base = 0;
    auto place = [&](uint32_t step, auto first_step) {
        constexpr bool sum = decltype(first_step)::value;
        uint32_t next = turn, added = turn;            // stretches whose counts to load and to add
        Pair pair[kPlaceKeys];
        uint32_t rank[kPlaceKeys];
#pragma unroll
        for (int k = 0; k < kPlaceKeys; ++k)
            pair[k] = number_of<kPlaceKeys>(k) < last - step ? pair_at<I>(p, step + number_of<kPlaceKeys>(k)) : Pair{0, 0};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            seen[w][tid] = 0;
        __syncthreads();
        rank_keys<kPlaceKeys>(
            [&](int k) { return pair[k].key >> p.shift & (bins - 1); }, last - step, seen[wave], rank,
            [&](int k) {
                if (sum && k * kCountsAhead * turns < p.stretches) {
#pragma unroll
                    for (int a = 0; a < kCountsAhead; ++a) {
                        here[a] = counts[min(next, p.stretches - 1) * quads];
                        next += turns;
                    }
                }
            },
            [&](int k) {
                if (sum && k * kCountsAhead * turns < p.stretches) {
#pragma unroll
                    for (int a = 0; a < kCountsAhead; ++a) {
                        if (added < blockIdx.x)
                            add(before, here[a]);
                        else if (added < p.stretches)
                            add(after, here[a]);
                        added += turns;
                    }
                }
            });
        if (sum && turn < turns) {
            *reinterpret_cast<uint4*>(&sums[0][turn * bins + 4 * quad]) = before;
            *reinterpret_cast<uint4*>(&sums[1][turn * bins + 4 * quad]) = after;
        }
        __syncthreads();
        if constexpr (sum) {
            uint32_t total = 0;
            if (tid < bins)
                for (uint32_t t = 0; t < turns; ++t) {
                    base += sums[0][t * bins + tid];
                    total += sums[1][t * bins + tid];
                }
            base += exclusive_sum(total + base, wave_sums);
        }
        base = counts_to_starts(seen, tid, base);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlaceKeys; ++k)
            if (number_of<kPlaceKeys>(k) < last - step)
                p.out[seen[wave][pair[k].key >> p.shift & (bins - 1)] + rank[k]] = pair[k];
        __syncthreads();
    };
    place(first, std::true_type());
    for (uint32_t step = first + kPlaceStep; step < last; step += kPlaceStep)
        place(step, std::false_type());
}

// ---- gradient: sorting in one launch
//
// A workgroup a bucket of rows: it reads all indices, keeps those of its bucket in
// their order and counts those of the buckets before, which is where its own go.
// Those that it keeps fit LDS, as the row in the bucket and the position in one
// word, and are sorted there by the row's bits.  Where they do not, a row that
// most of them name goes first, already in order, and the rest is sorted; several
// such rows in one bucket go through global memory in steps.  A further workgroup
// writes the marks of indices outside the table.  (Of 16,000 indices into 30,000
// rows the sort alone took 39 us in one workgroup.)
//
// Equal indices have to lie together, their rows need no order: a row's bucket
// mixes all digits of its index, so that neither rows close together (a vocabulary
// in the order of its words' frequency) nor rows at some stride (a column of
// texels) are in one bucket.

constexpr uint32_t kPositionBits = 17;
constexpr uint32_t kMaxLow = 32 - kPositionBits, kMaxBuckets = 512;
// Indices for each pass that the other sort takes.  (The call with one against
// the other, us: 33,000 into 700 rows 21 and 25, 66,000 29 and 28; 66,000 into
// 30,000 rows 34 and 50, 131,000 46 and 51; 100,000 into 2^23 57 and 75, into
// 2^25, which would take 1024 buckets, 227 and 138.  With half of the indices on
// one row, 20,000 into 30,000 rows 40 and 50, 80,000 89 and 69, 120,000 into 2^20
// 129 and 108; with all of them 41 and 55, 105 and 86, 152 and 129.)
constexpr uint32_t kBucketPass = 40960;
// ... and for each bucket, half of what LDS holds: few rows have few buckets, a
// workgroup each.  (20,000 into 5 rows 57 and 26, into 33 21 and 24; 40,000 into 5
// rows 90 and 28, into 64 27 and 25; 4,000 into 5 rows 18 and 21.)
constexpr uint32_t kBucketShare = 4096;
static_assert(3 * kBucketPass <= 1u << kPositionBits, "up to 2^24 rows take three passes");
// Half of a CU's LDS, for a second workgroup that clears: indices that a wave can
// keep, and bits of a pass.
constexpr uint32_t kSegment = 512;
constexpr int kBucketBits = 9, kBucketBins = 1 << kBucketBits;
static_assert(2 * kBucketBits >= kMaxLow, "two passes");
constexpr int kScanAhead = 8;

struct BucketParams {
    const void* ids;
    Pair *out, *spare;
    uint32_t n, rows;
    uint32_t high, low, buckets;       // digits of an index, low that of the row in its bucket; buckets = 2^high
    int passes;                        // over the bits of the row in the bucket
    Clear clear;
};

// The bucket of an index inside the table; and back, with the row in the bucket,
// which is the index without its lowest digit.
__device__ __forceinline__ uint32_t bucket_of(const BucketParams& p, uint32_t key)
{
    return ((key ^ key >> p.high) + (key >> 2 * p.high)) & (p.buckets - 1);
}

__device__ __forceinline__ uint32_t key_of(const BucketParams& p, uint32_t bucket, uint32_t row)
{
    return row << p.high | (((bucket - (row >> p.high)) ^ row) & (p.buckets - 1));
}

// Set lanes of a mask below this one, and `base`.
__device__ __forceinline__ uint32_t lanes_below(uint64_t mask, uint32_t base)
{
    return __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(mask >> 32),
                                     __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(mask), base));
}

// emit(inside, key, i) for the wave's indices in their order, by all lanes;
// `inside` is false of those outside the table and past the wave's last.  A
// thread's instructions per index are what the scan takes (80,000 indices: six
// more, 3 us), so whole batches look at no end.
template <typename I, typename E>
__device__ __forceinline__ void scan_ids(const BucketParams& p, E emit)
{
    const uint32_t span = (p.n + 64 * kWaves - 1) / (64 * kWaves) * 64;
    const uint32_t lane = threadIdx.x & 63, first = (threadIdx.x >> 6) * span, last = min(p.n, first + span);
    const I* ids = static_cast<const I*>(p.ids);
    auto batch = [&](uint32_t i, auto whole) {
        constexpr bool all = decltype(whole)::value;
        I id[kScanAhead];
#pragma unroll
        for (int a = 0; a < kScanAhead; ++a)
            id[a] = all ? (ids + i + lane)[64 * a] : ids[min(i + 64 * a + lane, p.n - 1)];
#pragma unroll
        for (int a = 0; a < kScanAhead; ++a) {
            // rows < 2^31: a negative index is outside as an unsigned one of its own size
            const bool inside = static_cast<std::make_unsigned_t<I>>(id[a]) < p.rows;
            emit(inside && (all || i + 64 * a + lane < last), static_cast<uint32_t>(id[a]), i + 64 * a + lane);
        }
    };
    uint32_t i = first;
    for (; i + 64 * kScanAhead <= last; i += 64 * kScanAhead)
        batch(i, std::true_type());
    for (; i < last; i += 64 * kScanAhead)
        batch(i, std::false_type());
}

__device__ __forceinline__ int shift_of(const BucketParams& p, int pass) { return p.low * pass / p.passes; }

// The m kept words of `list`, in order, to out[start..].
template <int KEYS>
__device__ __forceinline__ void sort_list(const BucketParams& p, uint32_t bucket, uint32_t m, uint32_t start,
                                          uint32_t (*seen)[kBucketBins], uint32_t* list, uint32_t* wave_sums)
{
    const uint32_t tid = threadIdx.x, wave = tid >> 6;
    uint32_t v[KEYS], to[KEYS];
#pragma unroll
    for (int k = 0; k < KEYS; ++k)
        v[k] = number_of<KEYS>(k) < m ? list[number_of<KEYS>(k)] : 0;
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = shift_of(p, pass), bits = shift_of(p, pass + 1) - shift;
        const uint32_t bins = 1u << bits;
        auto digit = [&](int k) { return v[k] >> (kPositionBits + shift) & (bins - 1); };
        if (tid < bins) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                seen[w][tid] = 0;
        }
        __syncthreads();
        rank_keys<KEYS>(digit, m, seen[wave], to, [](int) {}, [](int) {});
        __syncthreads();
        uint32_t total = 0;
        if (tid < bins) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                total += seen[w][tid];
        }
        const uint32_t base = exclusive_sum(total, wave_sums);
        if (tid < bins)
            counts_to_starts(seen, tid, base);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < KEYS; ++k)
            to[k] += seen[wave][digit(k)];
        if (pass + 1 < p.passes) {
#pragma unroll
            for (int k = 0; k < KEYS; ++k)
                if (number_of<KEYS>(k) < m)
                    list[to[k]] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < KEYS; ++k)
                v[k] = number_of<KEYS>(k) < m ? list[number_of<KEYS>(k)] : 0;
        }
    }
#pragma unroll
    for (int k = 0; k < KEYS; ++k)
        if (number_of<KEYS>(k) < m)
            p.out[start + to[k]] = Pair{key_of(p, bucket, v[k] >> kPositionBits), v[k] & ((1u << kPositionBits) - 1)};
}

// The row in the bucket that most of 64 kept words name, from all waves' parts of
// `list`; the same in every wave.
__device__ __forceinline__ uint32_t frequent_row(const uint32_t* list, const uint32_t* kept_by)
{
    static_assert(kWaves == 16, "four words of every wave's");
    const uint32_t lane = threadIdx.x & 63, wave = lane & (kWaves - 1), kept = min(kept_by[wave], kSegment);
    const uint32_t row = kept ? list[wave * kSegment + (lane / kWaves) * kept / 4] >> kPositionBits : ~0u;
    uint32_t found = ~0u, most = 0;
    for (int s = 0; s < 64; ++s) {
        const uint32_t at = __shfl(row, s), count = static_cast<uint32_t>(__popcll(__ballot(row == at)));
        if (at != ~0u && count > most) {
            most = count;
            found = at;
        }
    }
    return found;
}

template <typename I>
__global__ __launch_bounds__(kSortThreads) void bucket_kernel(BucketParams p)
{
    if (blockIdx.x > p.buckets) {
        clear_share(p.clear, blockIdx.x - p.buckets - 1);
        return;
    }
    __shared__ uint32_t list[kWaves * kSegment];
    __shared__ uint32_t seen[kWaves][kBucketBins];
    __shared__ uint32_t wave_sums[kWaves], kept_by[kWaves], before_by[kWaves];
    static_assert(sizeof(list) <= sizeof(seen), "the list moves there and back");
    const uint32_t tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const uint32_t bucket = blockIdx.x;
    const bool marks = bucket == p.buckets;

    uint32_t kept = 0, before = 0;
    scan_ids<I>(p, [&](bool inside, uint32_t key, uint32_t i) {
        const uint32_t of = bucket_of(p, key);
        const bool mine = inside && of == bucket;       // none of the marks'
        const uint64_t all = __ballot(mine);
        before += __popcll(__ballot(inside && of < bucket));
        const uint32_t at = lanes_below(all, kept);
        if (mine && at < kSegment)
            list[wave * kSegment + at] = key >> p.high << kPositionBits | i;
        kept += __popcll(all);
    });
    if (lane == 0) {
        kept_by[wave] = kept;
        before_by[wave] = before;
    }
    __syncthreads();
    uint32_t m = 0, start = 0, offset = 0;
    bool fits = true;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        offset += w < wave ? kept_by[w] : 0;
        m += kept_by[w];
        start += before_by[w];
        fits = fits && kept_by[w] <= kSegment;
    }
    if (marks) {
        for (uint32_t i = start + tid; i < p.n; i += kSortThreads)
            p.out[i] = Pair{p.rows, 0};
        return;
    }
    if (m == 0)
        return;
    if (!fits) {
        // without the row that most of them name
        const uint32_t hot = frequent_row(list, kept_by);
        uint32_t equal = 0, rest = 0;
        __syncthreads();
        scan_ids<I>(p, [&](bool inside, uint32_t key, uint32_t i) {
            const bool mine = inside && bucket_of(p, key) == bucket;
            equal += __popcll(__ballot(mine && key >> p.high == hot));
            const bool other = mine && key >> p.high != hot;
            const uint64_t all = __ballot(other);
            const uint32_t at = lanes_below(all, rest);
            if (other && at < kSegment)
                list[wave * kSegment + at] = key >> p.high << kPositionBits | i;
            rest += __popcll(all);
        });
        if (lane == 0) {
            kept_by[wave] = rest;
            before_by[wave] = equal;
        }
        __syncthreads();
        uint32_t equals = 0, rests = 0, equal_at = start, rest_at = 0;
        fits = true;
#pragma unroll
        for (uint32_t w = 0; w < kWaves; ++w) {
            equal_at += w < wave ? before_by[w] : 0;
            rest_at += w < wave ? kept_by[w] : 0;
            equals += before_by[w];
            rests += kept_by[w];
            fits = fits && kept_by[w] <= kSegment;
        }
        if (fits) {
            scan_ids<I>(p, [&](bool inside, uint32_t key, uint32_t i) {
                const bool mine = inside && bucket_of(p, key) == bucket && key >> p.high == hot;
                const uint64_t all = __ballot(mine);
                if (mine)
                    p.out[lanes_below(all, equal_at)] = Pair{key, i};
                equal_at += __popcll(all);
            });
            kept = rest;
            offset = rest_at;
            m = rests;
            start += equals;
            if (m == 0)
                return;
        }
    }
    if (fits) {
        uint32_t* whole = &seen[0][0];
        for (uint32_t i = lane; i < kept; i += 64)
            whole[offset + i] = list[wave * kSegment + i];
        __syncthreads();
        for (uint32_t i = tid; i < m; i += kSortThreads)
            list[i] = whole[i];
        __syncthreads();
        if (m <= kSortThreads)
            sort_list<1>(p, bucket, m, start, seen, list, wave_sums);
        else if (m <= 4 * kSortThreads)
            sort_list<4>(p, bucket, m, start, seen, list, wave_sums);
        else
            sort_list<8>(p, bucket, m, start, seen, list, wave_sums);
        return;
    }

    // more than LDS holds: to global memory in order, then pass by pass
    Pair *from = (p.passes & 1 ? p.spare : p.out) + start, *to = (p.passes & 1 ? p.out : p.spare) + start;
    scan_ids<I>(p, [&](bool inside, uint32_t key, uint32_t i) {
        const bool mine = inside && bucket_of(p, key) == bucket;
        const uint64_t all = __ballot(mine);
        if (mine)
            from[lanes_below(all, offset)] = Pair{key, i};
        offset += __popcll(all);
    });
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = shift_of(p, pass), bits = shift_of(p, pass + 1) - shift;
        const uint32_t bins = 1u << bits;
        if (tid < bins)
            list[tid] = 0;
        __syncthreads();
        for (uint32_t i = tid; i < m; i += kSortThreads)
            atomicAdd(&list[from[i].key >> p.high >> shift & (bins - 1)], 1u);
        __syncthreads();
        uint32_t base = exclusive_sum(tid < bins ? list[tid] : 0, wave_sums);
        for (uint32_t step = 0; step < m; step += kPlaceStep) {
            Pair pair[kPlaceKeys];
            uint32_t rank[kPlaceKeys];
            auto digit = [&](int k) { return pair[k].key >> p.high >> shift & (bins - 1); };
#pragma unroll
            for (int k = 0; k < kPlaceKeys; ++k)
                pair[k] = number_of<kPlaceKeys>(k) < m - step ? from[step + number_of<kPlaceKeys>(k)] : Pair{0, 0};
            if (tid < bins) {
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    seen[w][tid] = 0;
            }
            __syncthreads();
            rank_keys<kPlaceKeys>(digit, m - step, seen[wave], rank, [](int) {}, [](int) {});
            __syncthreads();
            if (tid < bins)
                base = counts_to_starts(seen, tid, base);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kPlaceKeys; ++k)
                if (number_of<kPlaceKeys>(k) < m - step)
                    to[seen[wave][digit(k)] + rank[k]] = pair[k];
            __syncthreads();
        }
        Pair* t = from;
        from = to;
        to = t;
    }
}

// ---- gradient: sums

struct SumParams {
    const Pair* pairs;         // sorted
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

// Entries whose rows are under way together; also of those past the tile and
// of indices outside the table, whose positions are rows of `grad` too.
constexpr int kSumAhead = 8;

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
    uint32_t key = p.pairs[first].key;
    bool before = first > 0 && p.pairs[first - 1].key == key;
    float acc[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        acc[k] = 0.0f;
    auto part = [&](float* to) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            to[static_cast<uint64_t>(group) * p.width + c * V + k] = acc[k];
    };
    for (uint32_t i = first; i < last; i += kSumAhead) {
        Pair pair[kSumAhead];
        float v[kSumAhead][V];
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
            pair[a] = p.pairs[min(i + a, last - 1)];
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
            load_run<T, V>(grad + pair[a].at * p.grad_stride, v[a]);
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a) {
            if (i + a >= last)
                break;
            if (pair[a].key != key) {
                if (before)
                    part(p.head);
                else
                    finish<O, V>(p, key, e, skip, acc);
                before = false;
                key = pair[a].key;
#pragma unroll
                for (int k = 0; k < V; ++k)
                    acc[k] = 0.0f;
            }
            if (key >= p.rows)
                return;                     // indices outside the table come last
#pragma unroll
            for (int k = 0; k < V; ++k)
                acc[k] += v[a][k];
        }
    }
    if (before)
        part(p.head);
    else if (last < p.n && p.pairs[last].key == key)
        part(p.tail);
    else
        finish<O, V>(p, key, e, skip, acc);
}

// Runs over more than kLong tiles are joined by a workgroup each.
constexpr uint32_t kLong = 16;

// Whether tile t's last run begins in it and goes on into the next.
__device__ __forceinline__ bool opens(const SumParams& p, uint32_t t, uint32_t& key)
{
    if (t + 1 >= p.tiles)
        return false;
    const uint32_t first = t * p.tile, last = first + p.tile;
    key = p.pairs[last - 1].key;
    return p.pairs[last].key == key && key < p.rows && !(first > 0 && p.pairs[first - 1].key == key);
}

// Whether a run of `key` that reaches tile t - 1 reaches tile t.
__device__ __forceinline__ bool reaches(const SumParams& p, uint32_t t, uint32_t key)
{
    return t < p.tiles && p.pairs[static_cast<uint64_t>(t) * p.tile].key == key;
}

// The parts of the runs that cross tiles, in order: short ones by the lanes
// of a tile, in the first workgroups; long ones by the others, each looking
// after kLong tiles, in which at most one long run can begin.
template <typename O, int V>
__global__ __launch_bounds__(kThreads) void join_kernel(SumParams p, uint32_t short_blocks)
{
    const uint32_t c = blockIdx.y * p.lanes + threadIdx.x % p.lanes;
    const uint64_t at = c * V;
    const uint32_t e = min(c * V, p.cols - V), skip = c * V - e;
    float acc[V];
    uint32_t key;
    if (blockIdx.x < short_blocks) {
        const uint32_t t = (blockIdx.x * kThreads + threadIdx.x) / p.lanes;
        if (c >= p.runs || !opens(p, t, key) || reaches(p, t + kLong + 1, key))
            return;
#pragma unroll
        for (int k = 0; k < V; ++k)
            acc[k] = p.tail[t * static_cast<uint64_t>(p.width) + at + k];
        for (uint32_t u = t + 1; reaches(p, u, key); ++u) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                acc[k] += p.head[u * static_cast<uint64_t>(p.width) + at + k];
        }
        finish<O, V>(p, key, e, skip, acc);
        return;
    }
    __shared__ uint32_t begin, end;
    __shared__ float parts[kThreads][V];
    const uint32_t t0 = (blockIdx.x - short_blocks) * kLong;
    if (threadIdx.x == 0)
        begin = p.tiles;
    __syncthreads();
    if (threadIdx.x < kLong && opens(p, t0 + threadIdx.x, key) && reaches(p, t0 + threadIdx.x + kLong + 1, key))
        begin = t0 + threadIdx.x;
    __syncthreads();
    const uint32_t t = begin;
    if (t >= p.tiles)
        return;
    key = p.pairs[(t + 1) * static_cast<uint64_t>(p.tile) - 1].key;
    // the first tile that the run does not reach: 64 probes a round
    if (threadIdx.x < 64) {
        uint32_t low = t + kLong + 1, high = p.tiles;      // it reaches low, and not high
        while (high - low > 1) {
            const uint32_t stride = (high - low + 63) / 64;
            const uint32_t probe = low + (threadIdx.x + 1) * stride;
            const uint64_t yes = __ballot(probe < high && reaches(p, probe, key));
            const uint32_t more = static_cast<uint32_t>(__popcll(yes));
            high = min(high, low + (more + 1) * stride);
            low += more * stride;
        }
        if (threadIdx.x == 0)
            end = low + 1;
    }
    __syncthreads();
    // groups of lanes take the run's tiles in turn, then add up
    const uint32_t groups = kThreads / p.lanes, group = threadIdx.x / p.lanes;
#pragma unroll
    for (int k = 0; k < V; ++k)
        acc[k] = group == 0 && c < p.runs ? p.tail[t * static_cast<uint64_t>(p.width) + at + k] : 0.0f;
    if (c < p.runs) {
#pragma unroll 4
        for (uint32_t u = t + 1 + group; u < end; u += groups) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                acc[k] += p.head[u * static_cast<uint64_t>(p.width) + at + k];
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        parts[threadIdx.x][k] = acc[k];
    __syncthreads();
    if (group > 0 || c >= p.runs)
        return;
    for (uint32_t g = 1; g < groups; ++g)
#pragma unroll
        for (int k = 0; k < V; ++k)
            acc[k] += parts[g * p.lanes + threadIdx.x][k];
    finish<O, V>(p, key, e, skip, acc);
}

// ---- gradient of a few indices, in one launch
//
// Up to kDirect indices need no sort: every workgroup reads them all, links
// each to the next of its kind, and a group of lanes sums the chain that
// begins with its index, in order.  Further workgroups clear the rows that no
// index names.  (133 indices of 116 columns: 15.5 us a call with the sort's
// three launches.)

constexpr uint32_t kDirect = 256;
static_assert(kDirect <= kThreads, "an index a thread");

struct DirectParams {
    SumParams sum;
    const void* ids;
    uint32_t sum_blocks;       // in each of `slices` slices of the columns
    uint32_t slices;
    uint32_t clear_rows;       // rows that a workgroup clears, at most kClearRows
};

constexpr uint32_t kClearRows = 4096;

template <typename T, typename O, typename I, int V>
__global__ __launch_bounds__(kThreads) void direct_kernel(DirectParams p)
{
    __shared__ uint32_t keys[kDirect];
    __shared__ uint32_t next[kDirect];
    __shared__ uint32_t named[kClearRows / 32];
    const SumParams& q = p.sum;
    const uint32_t tid = threadIdx.x;
    uint32_t key = q.rows;
    if (tid < q.n) {
        const int64_t id = static_cast<const I*>(p.ids)[tid];
        key = static_cast<uint64_t>(id) < q.rows ? static_cast<uint32_t>(id) : q.rows;
    }
    if (blockIdx.x >= p.sum_blocks * p.slices) {
        const uint32_t first = (blockIdx.x - p.sum_blocks * p.slices) * p.clear_rows;
        const uint32_t count = min(p.clear_rows, q.rows - first);
        for (uint32_t w = tid; w < kClearRows / 32; w += kThreads)
            named[w] = 0;
        __syncthreads();
        if (key - first < count)
            atomicOr(&named[(key - first) >> 5], 1u << ((key - first) & 31));
        __syncthreads();
        float zero[V];
#pragma unroll
        for (int k = 0; k < V; ++k)
            zero[k] = 0.0f;
        for (uint64_t i = tid; i < static_cast<uint64_t>(count) * q.runs; i += kThreads) {
            const uint32_t r = static_cast<uint32_t>(i / q.runs), c = static_cast<uint32_t>(i - static_cast<uint64_t>(r) * q.runs);
            if (!(named[r >> 5] >> (r & 31) & 1))
                store_run<O, V>(static_cast<O*>(q.out) + (first + r) * q.out_stride + min(c * V, q.cols - V), zero);
        }
        return;
    }
    keys[tid] = key;
    __syncthreads();
    bool begins = key < q.rows;
    uint32_t after = kDirect;
    for (uint32_t u = 0; u < q.n; ++u) {
        const bool same = keys[u] == key;
        begins = begins && !(same && u < tid);
        after = same && u > tid ? min(after, u) : after;
    }
    // indices that begin no chain are struck out
    const uint32_t slice = blockIdx.x / p.sum_blocks, block = blockIdx.x - slice * p.sum_blocks;
    next[tid] = after;
    __syncthreads();
    if (!begins)
        keys[tid] = q.rows;
    __syncthreads();
    const uint32_t at = block * (kThreads / q.lanes) + tid / q.lanes, c = slice * q.lanes + tid % q.lanes;
    if (at >= q.n || c >= q.runs)
        return;
    key = keys[at];
    if (key >= q.rows)
        return;
    const uint32_t e = min(c * V, q.cols - V);
    const T* grad = static_cast<const T*>(q.grad) + e;
    float acc[V];
#pragma unroll
    for (int k = 0; k < V; ++k)
        acc[k] = 0.0f;
    for (uint32_t u = at; u < kDirect;) {
        uint32_t link[kSumAhead];
        float v[kSumAhead][V];
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a) {
            link[a] = u;
            u = u < kDirect ? next[u] : u;
        }
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
            load_run<T, V>(grad + (link[a] < kDirect ? link[a] : at) * q.grad_stride, v[a]);
#pragma unroll
        for (int a = 0; a < kSumAhead; ++a)
#pragma unroll
            for (int k = 0; k < V; ++k)
                acc[k] += link[a] < kDirect ? v[a][k] : 0.0f;
    }
    finish<O, V>(q, key, e, c * V - e, acc);
}

// ---- gradient: layout and launches

// Sorted entries that a group of lanes sums: where there are few lanes one
// round of loads, else more, with fewer sums to join.  (The call in tiles of 8
// and of 32, us: 4,000 indices of 64 columns 17.4 and 21.2, 33,000 27 and 33,
// 131,000 61 and 57; 640,000 of 24 105 and 85.)
constexpr uint32_t kTile = 32, kShortTile = kSumAhead;
constexpr int64_t kShortLanes = 1 << 17;

struct Plan {
    uint32_t passes, bits, stretch, stretches, tile, tiles;
    uint32_t high, low, buckets;        // buckets is 0 where the sort goes by digits
    size_t pairs[2], counts, head, tail, bytes;
};

size_t padded(size_t bytes) { return (bytes + 255) / 256 * 256; }

Plan plan_of(int64_t n, int64_t rows, int64_t cols)
{
    Plan q;
    uint32_t bits = 1;
    while ((rows >> bits) != 0)
        ++bits;                          // the largest key is `rows`
    q.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    q.bits = bits < 2 ? 2 : bits;        // counts are read by fours
    // of indices inside the table; 128 buckets, so that a CU has one, and others clear
    uint32_t inside = 1;
    while (((rows - 1) >> inside) > 0)
        ++inside;
    q.low = inside <= 10 ? 3 : inside - 7 < kMaxLow ? inside - 7 : kMaxLow;
    q.high = inside > q.low ? inside - q.low : 0;
    q.buckets = 1u << q.high;
    if (n > int64_t{kBucketPass} * q.passes || n > int64_t{kBucketShare} * q.buckets || q.buckets > kMaxBuckets)
        q.buckets = 0;
    const int64_t steps = (n + kPlaceStep - 1) / kPlaceStep;
    q.stretch = static_cast<uint32_t>((steps + kMaxStretches - 1) / kMaxStretches * kPlaceStep);
    q.stretches = q.stretch ? static_cast<uint32_t>((n + q.stretch - 1) / q.stretch) : 0;
    q.tile = n / kShortTile * ((cols + 3) / 4) <= kShortLanes ? kShortTile : kTile;
    q.tiles = static_cast<uint32_t>((n + q.tile - 1) / q.tile);
    const size_t width = static_cast<size_t>(cols + 7) / 8 * 8;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += padded(bytes);
        return here;
    };
    for (int k = 0; k < 2; ++k)
        q.pairs[k] = take(sizeof(Pair) * static_cast<size_t>(n));
    q.counts = take(4 * static_cast<size_t>(kMaxBins) * q.stretches);
    q.head = take(4 * q.tiles * width);
    q.tail = take(4 * q.tiles * width);
    q.bytes = at;
    return q;
}

// A pass; grid() sets s.clear to a launch's share and is its grid.
template <typename I, typename G>
void launch_pass(const SortParams& s, G& grid, hipStream_t stream)
{
    const dim3 counting = grid();
    count_kernel<I><<<counting, kSortThreads, 0, stream>>>(s);
    const dim3 placing = grid();
    place_kernel<I><<<placing, kSortThreads, 0, stream>>>(s);
}

// Where the sums find their indices: in `ids`, few of them, or sorted.
struct Indices {
    const void* ids;
    bool ids64, direct;
};

template <typename T, typename O, int V>
void launch_sums(SumParams p, const Indices& from, hipStream_t stream)
{
    p.runs = (p.cols + V - 1) / V;
    p.width = p.runs * V;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < p.runs)
        p.lanes *= 2;
    const uint32_t per_block = kThreads / p.lanes;
    if (from.direct) {
        DirectParams d;
        d.sum = p;
        d.ids = from.ids;
        d.sum_blocks = (p.n + per_block - 1) / per_block;
        d.slices = (p.runs + p.lanes - 1) / p.lanes;
        // 64 KB a workgroup
        const uint32_t rows = 65536 / (p.cols * static_cast<uint32_t>(sizeof(O)));
        d.clear_rows = rows < 1 ? 1 : rows > kClearRows ? kClearRows : rows;
        const uint32_t clear_blocks = p.accumulate ? 0 : (p.rows + d.clear_rows - 1) / d.clear_rows;
        const uint32_t grid = d.sum_blocks * d.slices + clear_blocks;
        if (grid == 0)
            return;
        if (from.ids64)
            direct_kernel<T, O, int64_t, V><<<grid, kThreads, 0, stream>>>(d);
        else
            direct_kernel<T, O, int32_t, V><<<grid, kThreads, 0, stream>>>(d);
        return;
    }
    const dim3 grid((p.tiles + per_block - 1) / per_block, (p.runs + p.lanes - 1) / p.lanes);
    sum_kernel<T, O, V><<<grid, kThreads, 0, stream>>>(p);
    if (p.tiles > 1)
        join_kernel<O, V><<<dim3(grid.x + (p.tiles + kLong - 1) / kLong, grid.y), kThreads, 0, stream>>>(p, grid.x);
}

template <typename T, typename O>
void launch_sums_of(const SumParams& p, const Indices& from, hipStream_t stream)
{
    constexpr int V = sizeof(T) == 4 ? 4 : 8;
    if (p.cols >= V)
        launch_sums<T, O, V>(p, from, stream);
    else
        launch_sums<T, O, 1>(p, from, stream);
}

template <typename T>
void launch_sums_to(const SumParams& p, int32_t out_dtype, const Indices& from, hipStream_t stream)
{
    if (out_dtype == SQN_F32)
        launch_sums_of<T, float>(p, from, stream);
    else if (out_dtype == SQN_F16)
        launch_sums_of<T, _Float16>(p, from, stream);
    else
        launch_sums_of<T, __bf16>(p, from, stream);
}

void launch_sums_from(const SumParams& p, int32_t dtype, int32_t out_dtype, const Indices& from, hipStream_t stream)
{
    if (dtype == SQN_F32)
        launch_sums_to<float>(p, out_dtype, from, stream);
    else if (dtype == SQN_F16)
        launch_sums_to<_Float16>(p, out_dtype, from, stream);
    else
        launch_sums_to<__bf16>(p, out_dtype, from, stream);
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
    if (table.rows == 0) {
        // every index is outside: a row of the output stands in for the one
        // that is read and not used
        p.table = out.data;
        p.table_stride = 0;
    }
    if (table.dtype == SQN_F32)
        return lookup<float>(p, ids64, stream);
    if (table.dtype == SQN_F16)
        return lookup<_Float16>(p, ids64, stream);
    return lookup<__bf16>(p, ids64, stream);
}

size_t lookup_gradient_bytes(int64_t n, int64_t rows, int64_t cols)
{
    return n <= kDirect ? 0 : plan_of(n, rows, cols).bytes;
}

hipError_t launch_lookup_gradient(const sqn_matrix& grad, const void* ids, bool ids64, float scale, bool accumulate,
                                  const sqn_matrix& table_grad, void* workspace, hipStream_t stream)
{
    SumParams p;
    p.pairs = nullptr;
    p.grad = grad.data;
    p.out = table_grad.data;
    p.head = p.tail = nullptr;
    p.grad_stride = grad.row_stride;
    p.out_stride = table_grad.row_stride;
    p.n = static_cast<uint32_t>(grad.rows);
    p.rows = static_cast<uint32_t>(table_grad.rows);
    p.cols = static_cast<uint32_t>(grad.cols);
    p.tile = p.tiles = 0;
    p.scale = scale;
    p.accumulate = accumulate ? 1 : 0;
    if (p.n <= kDirect) {
        launch_sums_from(p, grad.dtype, table_grad.dtype, Indices{ids, ids64, true}, stream);
        return hipGetLastError();
    }

    const Plan q = plan_of(grad.rows, table_grad.rows, table_grad.cols);
    char* ws = static_cast<char*>(workspace);
    Pair* pairs[2] = {reinterpret_cast<Pair*>(ws + q.pairs[0]), reinterpret_cast<Pair*>(ws + q.pairs[1])};

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
    s.bits = s.shift = 0;
    s.in = nullptr;
    s.out = pairs[0];
    const uint32_t launches = q.buckets ? 1 : 2 * q.passes;
    uint32_t launch = 0;
    // the next launch's grid, with its share of the clearing
    auto grid = [&]() {
        c.first = pieces / launches * launch;
        c.last = ++launch == launches ? pieces : pieces / launches * launch;
        const uint64_t want = (c.last - c.first + 4096 - 1) / 4096;
        // many more than there are CUs: they do not begin together
        c.blocks = static_cast<uint32_t>(want < 2048 ? want : 2048);
        s.clear = c;
        return dim3((q.buckets ? q.buckets + 1 : q.stretches) + c.blocks);
    };
    if (q.buckets) {
        const dim3 all = grid();
        const BucketParams b{ids, pairs[0], pairs[1], s.n, s.rows, q.high, q.low, q.buckets,
                             (static_cast<int>(q.low) + kBucketBits - 1) / kBucketBits, c};
        if (ids64)
            bucket_kernel<int64_t><<<all, kSortThreads, 0, stream>>>(b);
        else
            bucket_kernel<int32_t><<<all, kSortThreads, 0, stream>>>(b);
    } else {
        for (uint32_t pass = 0; pass < q.passes; ++pass) {
            s.shift = static_cast<int>(q.bits * pass / q.passes);
            s.bits = static_cast<int>(q.bits * (pass + 1) / q.passes) - s.shift;
            s.in = pairs[(pass + 1) & 1];
            s.out = pairs[pass & 1];
            if (pass > 0)
                launch_pass<Sorted>(s, grid, stream);
            else if (ids64)
                launch_pass<int64_t>(s, grid, stream);
            else
                launch_pass<int32_t>(s, grid, stream);
        }
    }
    p.pairs = s.out;
    p.head = reinterpret_cast<float*>(ws + q.head);
    p.tail = reinterpret_cast<float*>(ws + q.tail);
    p.tile = q.tile;
    p.tiles = q.tiles;
    launch_sums_from(p, grad.dtype, table_grad.dtype, Indices{ids, ids64, false}, stream);
    return hipGetLastError();
}

}  // namespace sqn
