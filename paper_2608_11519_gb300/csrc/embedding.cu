// Token embeddings (flarepp_embedding_*): the scaled lookup and the gradient of the table.
//
// The gradient sums the rows of dY by id. Adding them with atomics would make the result depend on
// their order and serialises where ids repeat (byte sequences meet each row hundreds of times), so
// the positions are sorted by id first: a stable least-digit-first radix sort of (id, position) in
// one pass for tables of up to 2,047 rows, two up to 4 M, three beyond (up to 1,024 positions: by
// counting for each what comes before it). Then equal stretches of
// the sorted positions are summed in parallel whatever the lengths of the runs of one id; a run that
// crosses from one stretch into the next leaves float32 partial sums, which a last kernel adds in
// order. The gradient is written once: a bit per row says which rows no id names.
//
// Many rows are bound by bytes, few by launches. Measured: the lookup of 131,072 rows of 256 bf16 values
// 17 us, 4.0 TB/s of writes, as fast as HBM fills; the gradient of those rows (257 of a table) 31 us, of which
// the sums 16.6 (alone, on cold caches) and the rest the latencies of four short launches, which overlap; the
// gradient of 262,144 rows of 512 float32 values (131,072 of a table, most of them met never) 181 us: the sums
// 113 at the copy rate, the zeros 28, the sort 34.
//
// What a kernel reads may come from the kernel before it, which it overlaps up to pdl_wait. Inputs are
// therefore not __restrict__: loads of memory promised to stay constant may move above that wait.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "checks.h"
#include "layer_status.cuh"
#include "tc_ptx.cuh"

namespace flarepp {
namespace {

// ------------------------------------------------------------------ vectors of 2 to 16 bytes
template <int BYTES>
struct Raw;
template <>
struct Raw<16> { using t = uint4; };
template <>
struct Raw<8> { using t = uint2; };
template <>
struct Raw<4> { using t = uint32_t; };
template <>
struct Raw<2> { using t = uint16_t; };

template <typename E, int N>
struct alignas(sizeof(E) * N) Vec {
    E v[N];
};
__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float& d, float x) { d = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16& d, float x) { d = __float2bfloat16_rn(x); }

template <typename E, int N>
__device__ __forceinline__ Vec<E, N> load_vec(const E* p) {
    using R = typename Raw<sizeof(E) * N>::t;
    const R r = *reinterpret_cast<const R*>(p);
    Vec<E, N> v;
    *reinterpret_cast<R*>(&v) = r;
    return v;
}
template <typename E, int N>
__device__ __forceinline__ void store_vec(E* p, const Vec<E, N>& v) {
    using R = typename Raw<sizeof(E) * N>::t;
    *reinterpret_cast<R*>(p) = *reinterpret_cast<const R*>(&v);
}

// The row that an id names, or -1 for an empty position (an id of V or more is one too, and sets
// `beyond`, which a thread records once: an atomic among the loads would keep them from being in flight
// together, 262,144 ids counted in 6.4 us instead of 4.5).
template <typename I>
__device__ __forceinline__ int64_t row_of(I id, int64_t V, bool* beyond) {
    if ((int64_t)id >= V) *beyond = true;
    return (int64_t)id >= V || id < 0 ? -1 : (int64_t)id;
}
__device__ __forceinline__ void record(bool beyond, int* status) {
    if (beyond) record_status(status, FLAREPP_ERR_INVALID_ARGUMENT);
}

// ------------------------------------------------------------------ lookup
// threadIdx.x walks a row's vectors, threadIdx.y the block's rows; four rows a thread, so that
// four table loads are in flight (eight: 22 us instead of 17 for 131,072 rows of 512 bytes).
constexpr int kLookupRows = 4;

template <typename E, int N, typename I>
__global__ void __launch_bounds__(256)
    lookup_kernel(const I* ids, const E* table, int64_t T, int64_t V,
                  int64_t C, float scale, E* __restrict__ Y, int* status) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int64_t t0 = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * kLookupRows;
    int64_t row[kLookupRows];
    bool beyond = false;
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k)
        row[k] = t0 + k < T ? row_of(ids[t0 + k], V, &beyond) : -1;
    record(beyond, status);
    for (int64_t c = (int64_t)threadIdx.x * N; c < C; c += (int64_t)blockDim.x * N) {
        Vec<E, N> x[kLookupRows];
#pragma unroll
        for (int k = 0; k < kLookupRows; ++k)
            if (row[k] >= 0) x[k] = load_vec<E, N>(table + row[k] * C + c);
#pragma unroll
        for (int k = 0; k < kLookupRows; ++k) {
            if (t0 + k >= T) break;
#pragma unroll
            for (int i = 0; i < N; ++i)
                from_f32(x[k].v[i], row[k] >= 0 ? to_f32(x[k].v[i]) * scale : 0.f);
            store_vec<E, N>(Y + (t0 + k) * C + c, x[k]);
        }
    }
}

// Rows that only words of four bytes or less divide: threadIdx.x walks the 16-byte blocks of the output
// that lie within the row. Each comes from the two blocks of the table that hold it, shifted by what the
// row is off there; the values before the first block and behind the last are copied one by one.
// 131,072 rows of 255 bf16 values take 31 us (57 value by value), of 254 31 (32 in pairs), 500,000 of 33 42
// (53). Few rows are too few blocks (1,000 of 1,023: 6.6 us, 3.5 value by value) and rows without a
// block in them all edges (2 M of 3: 27 and 16).
constexpr int64_t kShiftedRows = 64 * kNumSMs;
template <typename E, typename I>
__global__ void __launch_bounds__(256)
    lookup_shifted_kernel(const I* ids, const E* table, int64_t T, int64_t V, int64_t C, float scale,
                          E* __restrict__ Y, int* status) {
    constexpr int L = 16 / sizeof(E);
    tc::pdl_trigger();
    tc::pdl_wait();
    const int64_t t0 = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * kLookupRows;
    const E* end = table + V * C;
    const E* from[kLookupRows];   // the row, or null for zeros
    int head[kLookupRows], blocks[kLookupRows];
    int most = 0;
    bool beyond = false;
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
        const int64_t row = t0 + k < T ? row_of(ids[t0 + k], V, &beyond) : -1;
        from[k] = row >= 0 ? table + row * C : nullptr;
        const unsigned off = (unsigned)((uintptr_t)(Y + (t0 + k) * C) % 16);
        head[k] = (int)min(C, (int64_t)((16 - off) % 16 / sizeof(E)));
        blocks[k] = t0 + k < T ? (int)((C - head[k]) / L) : 0;
        most = max(most, blocks[k]);
    }
    record(beyond, status);
    for (int j = threadIdx.x; j < most; j += blockDim.x) {
        uint4 lo[kLookupRows], hi[kLookupRows];
#pragma unroll
        for (int k = 0; k < kLookupRows; ++k) {
            lo[k] = hi[k] = make_uint4(0, 0, 0, 0);
            if (j >= blocks[k] || !from[k]) continue;
            const E* src = from[k] + head[k] + j * L;
            const uint4* base = reinterpret_cast<const uint4*>((uintptr_t)src / 16 * 16);
            if (reinterpret_cast<const E*>(base + 2) <= end) {
                lo[k] = base[0];
                hi[k] = base[1];
            } else {  // the table's last values, as they would come from there
                __align__(16) E v[2 * L];
                const E* b = reinterpret_cast<const E*>(base);
#pragma unroll
                for (int i = 0; i < 2 * L; ++i)
                    if (b + i < end) v[i] = b[i];
                    else from_f32(v[i], 0.f);
                lo[k] = reinterpret_cast<const uint4*>(v)[0];
                hi[k] = reinterpret_cast<const uint4*>(v)[1];
            }
        }
#pragma unroll
        for (int k = 0; k < kLookupRows; ++k) {
            if (j >= blocks[k]) continue;
            uint32_t w[8] = {lo[k].x, lo[k].y, lo[k].z, lo[k].w, hi[k].x, hi[k].y, hi[k].z, hi[k].w};
            const unsigned off = (unsigned)((uintptr_t)(from[k] + head[k]) % 16);
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = off & 8 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = off & 4 ? w[i + 1] : w[i];
            if (sizeof(E) == 2)
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (off & 2) * 8);
            Vec<E, L> o;
            *reinterpret_cast<uint4*>(&o) = make_uint4(w[0], w[1], w[2], w[3]);
#pragma unroll
            for (int i = 0; i < L; ++i) from_f32(o.v[i], from[k] ? to_f32(o.v[i]) * scale : 0.f);
            store_vec<E, L>(Y + (t0 + k) * C + head[k] + j * L, o);
        }
    }
#pragma unroll
    for (int k = 0; k < kLookupRows; ++k) {
        if (t0 + k >= T) break;
        const int behind = head[k] + blocks[k] * L, n = (int)C - blocks[k] * L;
        for (int i = threadIdx.x; i < n; i += blockDim.x) {
            const int c = i < head[k] ? i : behind + i - head[k];
            from_f32(Y[(t0 + k) * C + c], from[k] ? to_f32(from[k][c]) * scale : 0.f);
        }
    }
}

// ------------------------------------------------------------------ sort
// A block sorts a contiguous tile of the positions, a warp a contiguous stretch of the tile, 32
// positions a step: the order of equal digits is the order of the tiles, stretches, steps and
// lanes, so the sort is stable.
constexpr int kSortThreads = 256;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kMaxBits = 11;
constexpr int kHeld = 4;  // positions per lane held in registers: a stretch of a tile of 1,024

struct SortPlan {
    int passes, bits;     // digits, and bits of each
    int64_t tile, tiles;  // positions per block, blocks
};

// An id as a sort key: empty positions come last, as V.
template <typename I>
__device__ __forceinline__ uint32_t key_of(I id, int64_t V, bool* beyond) {
    const int64_t r = row_of(id, V, beyond);
    return r < 0 ? (uint32_t)V : (uint32_t)r;
}
// That of position i, from the pass before if there was one.
template <typename I>
__device__ __forceinline__ uint32_t key_at(const I* ids, const uint32_t* keys, int64_t i,
                                           int64_t V, bool* beyond) {
    return keys ? keys[i] : key_of(ids[i], V, beyond);
}

// hist[digit][tile] = how often the tile has the digit. The first pass also clears the words that the sums
// count and mark in (a memset's place in the stream, which no launch overlaps, costs 3 us).
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
    count_kernel(const I* ids, const uint32_t* keys, int64_t T,
                 int64_t V, int64_t tile, int shift, int bins, uint32_t* __restrict__ hist,
                 uint32_t* __restrict__ words, int64_t n_words, int* status) {
    extern __shared__ uint32_t cnt[];
    tc::pdl_trigger();
    for (int d = threadIdx.x; d < bins; d += kSortThreads) cnt[d] = 0;
    __syncthreads();
    tc::pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < n_words;
         i += (int64_t)gridDim.x * kSortThreads)
        words[i] = 0;
    const int64_t i0 = (int64_t)blockIdx.x * tile, i1 = min(T, i0 + tile);
    bool beyond = false;
#pragma unroll 4
    for (int64_t i = i0 + threadIdx.x; i < i1; i += kSortThreads)
        atomicAdd(&cnt[(key_at(ids, keys, i, V, &beyond) >> shift) & (bins - 1)], 1u);
    record(beyond, status);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kSortThreads)
        hist[(int64_t)d * gridDim.x + blockIdx.x] = cnt[d];
}

// Turn each digit's counts into what precedes a tile within the digit; total[digit] = all of it.
// One warp per digit.
__global__ void __launch_bounds__(256)
    scan_kernel(uint32_t* __restrict__ hist, int64_t tiles, int bins,
                uint32_t* __restrict__ total) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int d = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (d >= bins) return;
    uint32_t* h = hist + (int64_t)d * tiles;
    uint32_t sum = 0;
    for (int64_t b = 0; b < tiles; b += 32) {
        const uint32_t v = b + lane < tiles ? h[b + lane] : 0;
        uint32_t s = v;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += u;
        }
        if (b + lane < tiles) h[b + lane] = sum + s - v;
        sum += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) total[d] = sum;
}

// Move every position to its place in the order of the digit.
template <typename I>
__global__ void __launch_bounds__(kSortThreads)
    place_kernel(const I* ids, const uint32_t* keys,
                 const uint32_t* pos, int64_t T, int64_t V, int64_t tile, int shift,
                 int bins, const uint32_t* hist, const uint32_t* total,
                 uint32_t* __restrict__ keys_out, uint32_t* __restrict__ pos_out) {
    extern __shared__ uint32_t sm[];  // [kSortWarps][bins] places, [bins] starts of the digits
    uint32_t* start = sm + kSortWarps * bins;
    __shared__ uint32_t warp_sum[kSortWarps];
    tc::pdl_trigger();
    for (int d = threadIdx.x; d < kSortWarps * bins; d += kSortThreads) sm[d] = 0;
    tc::pdl_wait();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t t0 = (int64_t)blockIdx.x * tile, t1 = min(T, t0 + tile);
    const int64_t stretch = (tile + kSortWarps * 32 - 1) / (kSortWarps * 32) * 32;
    const int64_t i0 = t0 + warp * stretch, i1 = min(t1, i0 + stretch);
    uint32_t key[kHeld];  // of the positions b + 32 k + lane
    bool beyond;          // recorded by the count
    auto load_keys = [&](int64_t b) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int64_t i = b + 32 * k + lane;
            key[k] = i < i1 ? key_at(ids, keys, i, V, &beyond) : (uint32_t)V;
        }
    };
    load_keys(i0);
    // starts: an exclusive scan of the totals, a stretch of bins per thread
    const int per = (bins + kSortThreads - 1) / kSortThreads;
    uint32_t mine = 0;
    for (int k = 0; k < per; ++k) {
        const int d = threadIdx.x * per + k;
        if (d < bins) {
            start[d] = mine;
            mine += total[d];
        }
    }
    uint32_t s = mine;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
    }
    if (lane == 31) warp_sum[warp] = s;
    __syncthreads();
    uint32_t before = s - mine;
    for (int w = 0; w < warp; ++w) before += warp_sum[w];
    for (int k = 0; k < per; ++k) {
        const int d = threadIdx.x * per + k;
        if (d < bins) start[d] += before;
    }
    // counts of each warp's stretch
    uint32_t* mine_at = sm + warp * bins;
    for (int64_t b = i0; b < i1; b += 32 * kHeld) {
        if (b != i0) load_keys(b);
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (b + 32 * k + lane < i1) atomicAdd(&mine_at[(key[k] >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    // places: start of the digit + tiles before + stretches before
    for (int d = threadIdx.x; d < bins; d += kSortThreads) {
        uint32_t at = start[d] + hist[(int64_t)d * gridDim.x + blockIdx.x];
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t n = sm[w * bins + d];
            sm[w * bins + d] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int64_t b = i0; b < i1; b += 32 * kHeld) {
        if (i1 - i0 > 32 * kHeld) load_keys(b);
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int64_t i = b + 32 * k + lane;
            if (b + 32 * k >= i1) break;
            const bool in = i < i1;
            const uint32_t d = in ? (key[k] >> shift) & (bins - 1) : 0xffffffffu;
            const uint32_t same = __match_any_sync(0xffffffffu, d);
            const uint32_t rank = __popc(same & ((1u << lane) - 1u));
            uint32_t at = 0;
            if (in) at = mine_at[d] + rank;
            __syncwarp();
            if (in && rank == 0) mine_at[d] += __popc(same);
            __syncwarp();
            if (in) {
                keys_out[at] = key[k];
                pos_out[at] = pos ? pos[i] : (uint32_t)i;
            }
        }
    }
}

// Few positions, in one launch instead of three or six: a position's place is the number of keys that come
// before it, T comparisons each, which kFewSplit threads share. A block holds all keys and places
// kFewPlaced positions; the blocks also clear the words that the sums count on.
constexpr int kFewThreads = 256, kFewSplit = 4, kFewPlaced = kFewThreads / kFewSplit;
constexpr int64_t kFewPositions = 1024;  // 2,000 take 22 us in all, with the radix passes 15 to 25
constexpr int64_t kClearWords = 1 << 16;  // words that a block clears; more take a memset

template <typename I>
__global__ void __launch_bounds__(kFewThreads)
    few_kernel(const I* ids, int T, int64_t V, uint32_t* __restrict__ keys_out,
               uint32_t* __restrict__ pos_out, uint32_t* __restrict__ words, int64_t n_words,
               int* status) {
    extern __shared__ uint4 few_keys[];  // [groups]: four keys each, beyond T the largest number
    uint32_t* key = reinterpret_cast<uint32_t*>(few_keys);
    const int groups = (T + 3) / 4;
    tc::pdl_trigger();
    tc::pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kFewThreads + threadIdx.x; i < n_words;
         i += (int64_t)gridDim.x * kFewThreads)
        words[i] = 0;
    bool beyond = false;
    I id[kFewPositions / kFewThreads];
#pragma unroll
    for (int k = 0; k < kFewPositions / kFewThreads; ++k) {
        const int i = k * kFewThreads + threadIdx.x;
        if (i < T) id[k] = ids[i];
    }
#pragma unroll
    for (int k = 0; k < kFewPositions / kFewThreads; ++k) {
        const int i = k * kFewThreads + threadIdx.x;
        if (i < 4 * groups)
            key[i] = i < T ? key_of(id[k], V, &beyond) : 0xffffffffu;
    }
    record(beyond && blockIdx.x == 0, status);
    __syncthreads();
    const int i = blockIdx.x * kFewPlaced + threadIdx.x / kFewSplit;
    const uint32_t mine = i < T ? key[i] : 0;
    int before = 0;
    // equal keys come in the order of their positions: those of earlier positions count too
#pragma unroll 4
    for (int g = threadIdx.x % kFewSplit; g < groups; g += kFewSplit) {
        const uint4 k = few_keys[g];
        const int j = 4 * g;
        before += (k.x < mine + (j < i)) + (k.y < mine + (j + 1 < i)) + (k.z < mine + (j + 2 < i)) +
                  (k.w < mine + (j + 3 < i));
    }
#pragma unroll
    for (int o = 1; o < kFewSplit; o *= 2) before += __shfl_xor_sync(0xffffffffu, before, o);
    if (i < T && threadIdx.x % kFewSplit == 0) {
        keys_out[before] = mine;
        pos_out[before] = (uint32_t)i;
    }
}

// ------------------------------------------------------------------ sums
// Thread (x, y) of a block sums units_of<E, N>() vectors of N columns of one stretch of the sorted
// positions. A run that lies within the stretch goes to the table; one that began before it leaves its sum
// in head[stretch], one that begins here and goes on in tail[stretch], and the stretch on a list of crossing
// runs: those of few parts from the front of `crossing`, those of many from its back (the order does not
// matter: each run is a sum of its own). A run's first stretch sets the row's bit in `met`.
constexpr int kSumThreads = 256;
constexpr int kMaxStretch = 256;
// a crossing run of more parts is joined by a whole block, one of up to so many by a row of threads
// (what it can hold at once)
constexpr int short_run(int n) { return n == 8 ? 4 : 8; }
constexpr int kMaxHeld = 4096;   // positions whose keys and places a block holds
constexpr int kBatch = 4;        // rows of a group of copies
constexpr int kRing = 16;        // rows in flight per thread
// Vectors per thread. What a position costs whatever its vectors (its key, its place, the turn of the
// loop: some 30 instructions) bounds the sums of narrow vectors, so a thread takes several of those
// (64,185 rows of 346 bf16 values: 75 us with one, 54 with four).
template <typename E, int N>
constexpr int units_of() {
    return sizeof(E) * N >= 16 ? 1 : sizeof(E) * N == 8 ? 2 : 4;
}
constexpr int kJoinThreads = 512, kJoinBlocks = 2 * kNumSMs;
constexpr int kZeroRows = 8;     // rows per warp that writes zeros

// An asynchronous copy of one vector into shared memory (two bytes, which the instruction does not
// know, at once).
template <typename E, int N>
__device__ __forceinline__ void copy_async(Vec<E, N>* dst, const E* src) {
    constexpr int kBytes = sizeof(E) * N;
    if constexpr (kBytes >= 4)
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(tc::smem_u32(dst)), "l"(src),
                     "n"(kBytes)
                     : "memory");
    else
        *dst = load_vec<E, N>(src);
}

// Zeros for those of kZeroRows rows that no id names: a stretch of such rows at a time, in 16-byte stores
// whatever the alignment of a row.
template <typename E>
__device__ void zero_rows(const uint32_t* met, int64_t v0, int64_t V, int64_t C,
                          int lane, E* __restrict__ dtable) {
    E zero;
    from_f32(zero, 0.f);
    uint32_t gone = ~met[v0 / 32] >> (v0 % 32) & ((1u << kZeroRows) - 1u);
    if (V - v0 < kZeroRows) gone &= (1u << (V - v0)) - 1u;
    while (gone) {
        const int v = __ffs(gone) - 1, rows = __ffs(~(gone >> v)) - 1;
        gone &= ~(((1u << rows) - 1u) << v);
        E* at = dtable + (v0 + v) * C;
        const int64_t n = rows * C;
        const int64_t before = min(n, (int64_t)((16 - (uintptr_t)at % 16) % 16 / sizeof(E)));
        const int64_t wide = (n - before) * sizeof(E) / 16, after = before + wide * (16 / sizeof(E));
        if (lane < before) at[lane] = zero;
#pragma unroll 4
        for (int64_t k = lane; k < wide; k += 32)
            reinterpret_cast<uint4*>(at + before)[k] = make_uint4(0, 0, 0, 0);
        if (lane < n - after) at[after + lane] = zero;
    }
}

template <typename E, int N>
__global__ void __launch_bounds__(kSumThreads)
    sum_kernel(const uint32_t* keys, const uint32_t* pos,
               const E* dY, int64_t T, int64_t V, int64_t C, int stretch, float scale,
               E* __restrict__ dtable, float* __restrict__ head, float* __restrict__ tail,
               uint32_t* __restrict__ met, uint32_t* __restrict__ crossing, int64_t stretches,
               uint32_t* __restrict__ n_crossing) {
    extern __shared__ uint8_t sum_smem[];
    constexpr int U = units_of<E, N>();
    // the rows in flight, U slots per thread: [kRing][U][kSumThreads]; the block's keys; its positions
    Vec<E, N>* ring = reinterpret_cast<Vec<E, N>*>(sum_smem);
    uint32_t* held = reinterpret_cast<uint32_t*>(sum_smem + sizeof(Vec<E, N>) * kRing * U * kSumThreads);
    const int tid = threadIdx.y * blockDim.x + threadIdx.x;
    tc::pdl_trigger();
    tc::pdl_wait();
    const int span = blockDim.y * stretch;
    const int64_t b0 = (int64_t)blockIdx.x * span;
    uint32_t* held_pos = held + span;
    for (int i = tid; i < span; i += kSumThreads) {
        const bool in = b0 + i < T;
        held[i] = in ? keys[b0 + i] : (uint32_t)V;
        held_pos[i] = in ? pos[b0 + i] : 0;
    }
    __syncthreads();
    // unit u: the N columns at c + u * next (row of a block: neighbouring vectors), if they exist
    const int64_t c = ((int64_t)blockIdx.y * U * blockDim.x + threadIdx.x) * N;
    const int next = blockDim.x * N;
    const int64_t st = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    const int64_t i0 = st * stretch;
    if (c >= C || i0 >= T) return;
    const int units = (int)min((int64_t)U, (C - 1 - c) / next + 1);
    const uint32_t* key = held + threadIdx.y * stretch;
    const uint32_t* at = held_pos + threadIdx.y * stretch;
    uint32_t cur = key[0];
    if (cur == (uint32_t)V) return;  // empty positions come last, and those beyond T count as such
    bool began = i0 == 0 || keys[i0 - 1] != cur;
    const bool goes_on = i0 + stretch < T && keys[i0 + stretch] == key[stretch - 1];
    float acc[U][N];
    auto clear = [&] {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) acc[u][k] = 0.f;
    };
    clear();
    const bool first = blockIdx.y == 0 && threadIdx.x == 0;
    auto flush = [&](bool more) {
        if (began && first) {
            atomicOr(met + (cur >> 5), 1u << (cur & 31));
            if (more) {
                const int64_t far = (st + 1 + short_run(N)) * stretch;
                if (far < T && keys[far] == cur)
                    crossing[stretches - 1 - atomicAdd(n_crossing + 1, 1u)] = (uint32_t)st;
                else
                    crossing[atomicAdd(n_crossing, 1u)] = (uint32_t)st;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= units) break;
            if (began && !more) {
                Vec<E, N> o;
#pragma unroll
                for (int k = 0; k < N; ++k) from_f32(o.v[k], acc[u][k] * scale);
                store_vec<E, N>(dtable + (int64_t)cur * C + c + u * next, o);
            } else {
                Vec<float, N> o;
#pragma unroll
                for (int k = 0; k < N; ++k) o.v[k] = acc[u][k];
                *reinterpret_cast<Vec<float, N>*>((began ? tail : head) + st * C + c + u * next) = o;
            }
        }
    };
    // Batches of rows come in by asynchronous copies, each thread's vectors into slots of its own:
    // kRing rows in flight per thread without registers to hold them.
    auto fetch = [&](int batch) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = batch * kBatch + k;
            if (i < stretch && key[i] != (uint32_t)V) {
                const E* row = dY + (uint64_t)at[i] * (uint32_t)C + c;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (u < units) copy_async(ring + (i % kRing * U + u) * kSumThreads + tid, row + u * next);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int b = 0; b < kRing / kBatch - 1; ++b) fetch(b);
    for (int b = 0; b < stretch / kBatch; ++b) {
        fetch(b + kRing / kBatch - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing / kBatch - 1) : "memory");
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = b * kBatch + k;
            if (key[i] != cur) {
                flush(false);
                began = true;
                cur = key[i];
                clear();
                if (cur == (uint32_t)V) return;  // only empty positions follow, none was fetched
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= units) break;
                const Vec<E, N> x = ring[(i % kRing * U + u) * kSumThreads + tid];
#pragma unroll
                for (int j = 0; j < N; ++j) acc[u][j] += to_f32(x.v[j]);
            }
        }
    }
    flush(goes_on);
}

// The runs that cross stretches, then the zeros of the rows that no id names. A run of many parts takes
// a block: the threads look at one stretch each to find where the run ends, the rows of threads add
// equal shares of the parts in order, and the shares are added in order. A run of few parts takes a row of
// threads, and the blocks that the long runs leave free take them first. A block does all three: as many as
// run at once are launched.
template <typename E, int N>
__global__ void __launch_bounds__(kJoinThreads, 2)
    join_kernel(const uint32_t* keys, int64_t T, int64_t V, int64_t C, int stretch,
                float scale, const float* head, const float* tail,
                const uint32_t* met, const uint32_t* crossing,
                int64_t stretches, const uint32_t* n_crossing, E* __restrict__ dtable) {
    extern __shared__ float share[];  // [blockDim.y][blockDim.x * N]
    const int tid = threadIdx.y * blockDim.x + threadIdx.x;
    tc::pdl_trigger();
    tc::pdl_wait();
    const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * N;
    const unsigned n_short = n_crossing[0], n_long = n_crossing[1];
    const int row = blockDim.x * N;
    auto write = [&](uint32_t key, const float* acc) {
        Vec<E, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) from_f32(o.v[k], acc[k] * scale);
        store_vec<E, N>(dtable + (int64_t)key * C + c, o);
    };
    for (unsigned item = blockIdx.x; item < n_long; item += gridDim.x) {
        const int64_t st = crossing[stretches - 1 - item];
        const uint32_t key = keys[(st + 1) * stretch];
        int64_t parts = 0;  // stretches st + 1 .. st + parts begin with the run's key
        for (;;) {
            const int64_t at = (st + 1 + parts + tid) * stretch;
            const int more = __syncthreads_count(at < T && keys[at] == key);
            parts += more;
            if (more < kJoinThreads) break;
        }
        const int64_t per = (parts + blockDim.y - 1) / blockDim.y;
        const int64_t p0 = threadIdx.y * per, p1 = min(parts, p0 + per);
        float acc[N];
#pragma unroll
        for (int k = 0; k < N; ++k) acc[k] = 0.f;
        if (c < C) {
            if (threadIdx.y == 0) {
                const Vec<float, N> v = *reinterpret_cast<const Vec<float, N>*>(tail + st * C + c);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] = v.v[k];
            }
#pragma unroll 4
            for (int64_t p = p0; p < p1; ++p) {
                const Vec<float, N> v =
                    *reinterpret_cast<const Vec<float, N>*>(head + (st + 1 + p) * C + c);
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += v.v[k];
            }
        }
#pragma unroll
        for (int k = 0; k < N; ++k) share[threadIdx.y * row + threadIdx.x * N + k] = acc[k];
        __syncthreads();
        if (threadIdx.y == 0 && c < C) {
            const int ys = (int)min((int64_t)blockDim.y, parts);  // the rest have no share
#pragma unroll 4
            for (int y = 1; y < ys; ++y)
#pragma unroll
                for (int k = 0; k < N; ++k) acc[k] += share[y * row + threadIdx.x * N + k];
            write(key, acc);
        }
        __syncthreads();
    }
    if (c < C)
        for (unsigned item = threadIdx.y * gridDim.x + (gridDim.x - 1 - blockIdx.x); item < n_short;
             item += gridDim.x * blockDim.y) {
            constexpr int kHold = short_run(N);
            const int64_t st = crossing[item];
            const uint32_t key = keys[(st + 1) * stretch];
            Vec<float, N> part[kHold];
            bool has[kHold];
#pragma unroll
            for (int p = 0; p < kHold; ++p) {
                const int64_t at = (st + 1 + p) * stretch;
                has[p] = at < T && keys[at] == key;
                if (has[p]) part[p] = *reinterpret_cast<const Vec<float, N>*>(head + (st + 1 + p) * C + c);
            }
            Vec<float, N> acc = *reinterpret_cast<const Vec<float, N>*>(tail + st * C + c);
#pragma unroll
            for (int p = 0; p < kHold; ++p)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (has[p]) acc.v[k] += part[p].v[k];
            write(key, acc.v);
        }
    // whole warps from here: threads 32 w .. 32 w + 31 of the block
    const int64_t warps = (int64_t)gridDim.x * gridDim.y * (kJoinThreads / 32);
    for (int64_t g = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kJoinThreads / 32) + tid / 32;
         g * kZeroRows < V; g += warps)
        zero_rows<E>(met, g * kZeroRows, V, C, tid % 32, dtable);
}

// ------------------------------------------------------------------ host side

flarepp_status check_shape(const flarepp_embedding_shape* s) {
    if (!s || s->T < 0 || s->V < 1 || s->C < 1) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->dtype != FLAREPP_F32 && s->dtype != FLAREPP_BF16) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->id_bytes != 4 && s->id_bytes != 8) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->T > 0x7fffffff || s->V > 0x7ffffffe || s->C > (1 << 20)) return FLAREPP_ERR_UNSUPPORTED;
    return FLAREPP_OK;
}

size_t elem(const flarepp_embedding_shape& s) { return s.dtype == FLAREPP_BF16 ? 2 : 4; }

// Values per vector: the widest that divides a row (rows then keep the base's alignment).
int vec_of(const flarepp_embedding_shape& s) {
    int n = (int)(16 / elem(s));
    while (s.C % n) n /= 2;
    return n;
}
int units_of(const flarepp_embedding_shape& s) {
    const size_t bytes = elem(s) * vec_of(s);
    return bytes >= 16 ? 1 : bytes == 8 ? 2 : 4;
}
// Threads along a row: enough for its vectors, a power of two up to `most`.
int lanes_for(int64_t vecs, int most) {
    int x = 1;
    while (x < most && x < vecs) x *= 2;
    return x;
}

SortPlan sort_plan(const flarepp_embedding_shape& s) {
    SortPlan p{};
    int bits = 1;
    while (((int64_t)1 << bits) <= s.V) ++bits;  // keys 0..V
    p.passes = (int)cdiv(bits, kMaxBits);
    p.bits = (int)cdiv(bits, p.passes);
    p.tile = cdiv(cdiv(s.T, 2 * kNumSMs), 512) * 512;  // about two blocks per SM
    p.tiles = cdiv(s.T, p.tile);
    return p;
}

struct Layout {
    SortPlan sort;
    int stretch;
    int64_t stretches;
    size_t off_met, met_bytes;  // the numbers of short and long crossing runs, then a bit per row
    size_t off_crossing, off_keys[2], off_pos[2], off_hist, off_total, off_head, off_tail, total;
};
Layout layout_of(const flarepp_embedding_shape& s) {
    Layout L{};
    L.sort = sort_plan(s);
    // Stretches so long that about 24 warps per SM have one each (with 64 KB of rows in flight three blocks
    // fit), in whole batches: in multiples of 16, and at least one, 131,072 rows of 256 values took 34 us
    // instead of 31 and 257 rows 13 instead of 9.5.
    const int64_t units = cdiv(cdiv(s.C, vec_of(s)), units_of(s)), x = lanes_for(units, 32);
    const int64_t want = cdiv(s.T * cdiv(units, x) * x, (int64_t)24 * 32 * kNumSMs);
    int64_t most = kMaxHeld / (kSumThreads / x);
    if (most > kMaxStretch) most = kMaxStretch;
    L.stretch = (int)(cdiv(want, kBatch) * kBatch);
    if (want > most) L.stretch = (int)most;
    L.stretches = cdiv(s.T, L.stretch);
    auto take = [&](int64_t bytes) {
        const size_t at = L.total;
        L.total = align_up(at + (size_t)bytes, kWsAlign);
        return at;
    };
    const int64_t bins = (int64_t)1 << L.sort.bits;
    L.met_bytes = 8 + (size_t)cdiv(s.V, 32) * 4;
    L.off_met = take((int64_t)L.met_bytes);
    L.off_crossing = take(L.stretches * 4);
    for (int i = 0; i < 2; ++i) {
        L.off_keys[i] = take(s.T * 4);
        L.off_pos[i] = take(s.T * 4);
    }
    L.off_hist = take(bins * L.sort.tiles * 4);
    L.off_total = take(bins * 4);
    L.off_head = take(L.stretches * s.C * 4);
    L.off_tail = take(L.stretches * s.C * 4);
    return L;
}

template <typename E, int N, typename I>
cudaError_t lookup(const flarepp_embedding_shape& s, const void* ids, const void* table,
                   float scale, void* Y, int* status, cudaStream_t st) {
    if (sizeof(E) * N <= 4 && s.T >= kShiftedRows && s.C * sizeof(E) >= 32) {
        const int x = lanes_for(cdiv(s.C * sizeof(E), 16), 32), y = 256 / x;
        return launch_pdl(lookup_shifted_kernel<E, I>, dim3((unsigned)cdiv(s.T, y * kLookupRows)),
                          dim3(x, y), 0, st, (const I*)ids, (const E*)table, s.T, s.V, s.C, scale,
                          (E*)Y, status);
    }
    const int x = lanes_for(cdiv(s.C, N), 256), y = 256 / x;
    return launch_pdl(lookup_kernel<E, N, I>, dim3((unsigned)cdiv(s.T, y * kLookupRows)),
                      dim3(x, y), 0, st, (const I*)ids, (const E*)table, s.T, s.V, s.C, scale,
                      (E*)Y, status);
}
template <typename E, int N>
cudaError_t lookup(const flarepp_embedding_shape& s, const void* ids, const void* table,
                   float scale, void* Y, int* status, cudaStream_t st) {
    return s.id_bytes == 4 ? lookup<E, N, int32_t>(s, ids, table, scale, Y, status, st)
                           : lookup<E, N, int64_t>(s, ids, table, scale, Y, status, st);
}

// keys and positions in order of the id; returns which of the two buffers holds them
template <typename I>
cudaError_t sort(const flarepp_embedding_shape& s, const Layout& L, const void* ids, char* ws,
                 int* status, int* at, cudaStream_t st) {
    const int bins = 1 << L.sort.bits;
    uint32_t* hist = (uint32_t*)(ws + L.off_hist);
    uint32_t* total = (uint32_t*)(ws + L.off_total);
    const uint32_t *keys = nullptr, *pos = nullptr;
    const unsigned tiles = (unsigned)L.sort.tiles;
    int64_t words = (int64_t)(L.met_bytes / 4);
    if (words > kClearWords * tiles) {
        const cudaError_t e = cudaMemsetAsync(ws + L.off_met, 0, L.met_bytes, st);
        if (e != cudaSuccess) return e;
        words = 0;
    }
    for (int p = 0; p < L.sort.passes; ++p) {
        const int shift = p * L.sort.bits;
        *at = p & 1;
        uint32_t* ko = (uint32_t*)(ws + L.off_keys[*at]);
        uint32_t* po = (uint32_t*)(ws + L.off_pos[*at]);
        cudaError_t e = launch_pdl(count_kernel<I>, dim3(tiles), dim3(kSortThreads), bins * 4, st,
                                   (const I*)ids, keys, s.T, s.V, L.sort.tile, shift, bins, hist,
                                   (uint32_t*)(ws + L.off_met), p == 0 ? words : 0,
                                   status);
        if (e == cudaSuccess)
            e = launch_pdl(scan_kernel, dim3((unsigned)cdiv(bins, 8)), dim3(256), 0, st, hist,
                           L.sort.tiles, bins, total);
        const size_t smem = (size_t)(kSortWarps + 1) * bins * 4;
        if (e == cudaSuccess && smem > 48 * 1024)
            e = cudaFuncSetAttribute(place_kernel<I>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (kSortWarps + 1) << (kMaxBits + 2));
        if (e == cudaSuccess)
            e = launch_pdl(place_kernel<I>, dim3(tiles), dim3(kSortThreads), smem, st,
                           (const I*)ids, keys, pos, s.T, s.V, L.sort.tile, shift, bins,
                           (const uint32_t*)hist, (const uint32_t*)total, ko, po);
        if (e != cudaSuccess) return e;
        keys = ko;
        pos = po;
    }
    return cudaSuccess;
}

template <typename I>
cudaError_t sort_few(const flarepp_embedding_shape& s, const Layout& L, const void* ids, char* ws,
                     int* status, cudaStream_t st) {
    const unsigned blocks = (unsigned)cdiv(s.T, kFewPlaced);
    int64_t words = (int64_t)(L.met_bytes / 4);
    if (words > kClearWords * blocks) {
        const cudaError_t e = cudaMemsetAsync(ws + L.off_met, 0, L.met_bytes, st);
        if (e != cudaSuccess) return e;
        words = 0;
    }
    return launch_pdl(few_kernel<I>, dim3(blocks), dim3(kFewThreads), (size_t)cdiv(s.T, 4) * 16, st,
                      (const I*)ids, (int)s.T, s.V, (uint32_t*)(ws + L.off_keys[0]),
                      (uint32_t*)(ws + L.off_pos[0]), (uint32_t*)(ws + L.off_met), words, status);
}

template <typename E, int N>
cudaError_t sums(const flarepp_embedding_shape& s, const Layout& L, int at, const void* dY,
                 float scale, void* dtable, char* ws, cudaStream_t st) {
    constexpr int U = units_of<E, N>();
    const int64_t vecs = cdiv(s.C, N);
    const int x = lanes_for(vecs, 32);
    const unsigned col_blocks = (unsigned)cdiv(vecs, x);
    const int sum_x = lanes_for(cdiv(vecs, U), 32), sum_y = kSumThreads / sum_x;
    const dim3 sum_grid((unsigned)cdiv(L.stretches, sum_y), (unsigned)cdiv(cdiv(vecs, U), sum_x));
    // the join: as many blocks as run at once, fewer where there is less to do
    const int64_t zero_blocks = cdiv(s.V, kZeroRows * (kJoinThreads / 32));
    const int64_t useful = L.stretches > zero_blocks ? L.stretches : zero_blocks;
    const int64_t join_most = cdiv(kJoinBlocks, col_blocks);
    const unsigned join_blocks = (unsigned)(useful < join_most ? useful : join_most);
    const uint32_t* keys = (const uint32_t*)(ws + L.off_keys[at]);
    const uint32_t* pos = (const uint32_t*)(ws + L.off_pos[at]);
    uint32_t* n_crossing = (uint32_t*)(ws + L.off_met);
    uint32_t* met = n_crossing + 2;
    uint32_t* crossing = (uint32_t*)(ws + L.off_crossing);
    float* head = (float*)(ws + L.off_head);
    float* tail = (float*)(ws + L.off_tail);
    constexpr size_t kRingBytes = sizeof(E) * N * U * kRing * kSumThreads;
    const size_t held = kRingBytes + (size_t)sum_y * L.stretch * 8;
    cudaError_t e = cudaSuccess;
    if (held > 48 * 1024)
        e = cudaFuncSetAttribute(sum_kernel<E, N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)kRingBytes + kMaxHeld * 8);
    if (e == cudaSuccess)
        e = launch_pdl(sum_kernel<E, N>, sum_grid, dim3(sum_x, sum_y), held, st, keys,
                       pos, (const E*)dY, s.T, s.V, s.C, L.stretch, scale, (E*)dtable, head, tail,
                       met, crossing, L.stretches, n_crossing);
    if (e == cudaSuccess)
        e = launch_pdl(join_kernel<E, N>, dim3(join_blocks, col_blocks),
                       dim3(x, kJoinThreads / x), (size_t)kJoinThreads * N * 4, st, keys, s.T, s.V,
                       s.C, L.stretch, scale, (const float*)head, (const float*)tail,
                       (const uint32_t*)met, (const uint32_t*)crossing, L.stretches,
                       (const uint32_t*)n_crossing, (E*)dtable);
    return e;
}

flarepp_status embedding_fwd(const flarepp_embedding_shape* shape, const void* ids,
                             const void* table, float scale, void* Y, int32_t* status,
                             cudaStream_t st) {
    const flarepp_status bad = check_shape(shape);
    if (bad != FLAREPP_OK) return bad;
    const flarepp_embedding_shape s = *shape;
    if (!isfinite(scale) || !aligned4(status)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s.T == 0) return FLAREPP_OK;
    if (!ids || !table || !Y || !aligned16(ids) || !aligned16(table) || !aligned16(Y))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const Span outs[2] = {{Y, (size_t)s.T * s.C * elem(s)}, {status, 4}};
    const Span ins[2] = {{ids, (size_t)s.T * s.id_bytes}, {table, (size_t)s.V * s.C * elem(s)}};
    if (!disjoint(outs, 2, ins, 2)) return FLAREPP_ERR_INVALID_ARGUMENT;
    using B = __nv_bfloat16;
    cudaError_t e;
    if (s.dtype == FLAREPP_BF16) switch (vec_of(s)) {
        case 8: e = lookup<B, 8>(s, ids, table, scale, Y, status, st); break;
        case 4: e = lookup<B, 4>(s, ids, table, scale, Y, status, st); break;
        case 2: e = lookup<B, 2>(s, ids, table, scale, Y, status, st); break;
        default: e = lookup<B, 1>(s, ids, table, scale, Y, status, st);
    } else switch (vec_of(s)) {
        case 4: e = lookup<float, 4>(s, ids, table, scale, Y, status, st); break;
        case 2: e = lookup<float, 2>(s, ids, table, scale, Y, status, st); break;
        default: e = lookup<float, 1>(s, ids, table, scale, Y, status, st);
    }
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

flarepp_status embedding_bwd(const flarepp_embedding_shape* shape, const void* ids, const void* dY,
                             float scale, void* dtable, void* workspace, size_t workspace_bytes,
                             int32_t* status, cudaStream_t st) {
    const flarepp_status bad = check_shape(shape);
    if (bad != FLAREPP_OK) return bad;
    const flarepp_embedding_shape s = *shape;
    if (!isfinite(scale) || !aligned4(status)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!dtable || !aligned16(dtable)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const size_t out_bytes = (size_t)s.V * s.C * elem(s);
    const Layout L = s.T ? layout_of(s) : Layout{};
    if (s.T) {
        if (!ids || !dY || !aligned16(ids) || !aligned16(dY)) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (!workspace || (uintptr_t)workspace % kWsAlign || workspace_bytes < L.total)
            return FLAREPP_ERR_WORKSPACE;
        const Span outs[3] = {{dtable, out_bytes}, {workspace, L.total}, {status, 4}};
        const Span ins[2] = {{ids, (size_t)s.T * s.id_bytes}, {dY, (size_t)s.T * s.C * elem(s)}};
        if (!disjoint(outs, 3, ins, 2)) return FLAREPP_ERR_INVALID_ARGUMENT;
    }
    if (s.T == 0)
        return cudaMemsetAsync(dtable, 0, out_bytes, st) == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
    char* ws = (char*)workspace;
    int at = 0;
    cudaError_t e;
    if (s.T <= kFewPositions) {
        e = s.id_bytes == 4 ? sort_few<int32_t>(s, L, ids, ws, status, st)
                            : sort_few<int64_t>(s, L, ids, ws, status, st);
    } else {
        e = s.id_bytes == 4 ? sort<int32_t>(s, L, ids, ws, status, &at, st)
                            : sort<int64_t>(s, L, ids, ws, status, &at, st);
    }
    if (e != cudaSuccess) return FLAREPP_ERR_CUDA;
    using B = __nv_bfloat16;
    if (s.dtype == FLAREPP_BF16) switch (vec_of(s)) {
        case 8: e = sums<B, 8>(s, L, at, dY, scale, dtable, ws, st); break;
        case 4: e = sums<B, 4>(s, L, at, dY, scale, dtable, ws, st); break;
        case 2: e = sums<B, 2>(s, L, at, dY, scale, dtable, ws, st); break;
        default: e = sums<B, 1>(s, L, at, dY, scale, dtable, ws, st);
    } else switch (vec_of(s)) {
        case 4: e = sums<float, 4>(s, L, at, dY, scale, dtable, ws, st); break;
        case 2: e = sums<float, 2>(s, L, at, dY, scale, dtable, ws, st); break;
        default: e = sums<float, 1>(s, L, at, dY, scale, dtable, ws, st);
    }
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

}  // namespace

cudaError_t take_embedding_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

}  // namespace flarepp

extern "C" {

flarepp_status flarepp_embedding_fwd(const flarepp_embedding_shape* shape, const void* ids,
                                     const void* table, float scale, void* Y, int32_t* status,
                                     void* stream) {
    return flarepp::embedding_fwd(shape, ids, table, scale, Y, status, (cudaStream_t)stream);
}

size_t flarepp_embedding_bwd_workspace_bytes(const flarepp_embedding_shape* shape) {
    if (flarepp::check_shape(shape) != FLAREPP_OK || shape->T == 0) return 0;
    return flarepp::layout_of(*shape).total;
}

flarepp_status flarepp_embedding_bwd(const flarepp_embedding_shape* shape, const void* ids,
                                     const void* dY, float scale, void* dtable, void* workspace,
                                     size_t workspace_bytes, int32_t* status, void* stream) {
    return flarepp::embedding_bwd(shape, ids, dY, scale, dtable, workspace, workspace_bytes,
                                  status, (cudaStream_t)stream);
}

}  // extern "C"
