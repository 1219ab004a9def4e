// The tensor-core product of the linear layer (tcgen05 / TMEM / TMA, bf16 operands, float32 sums):
//   D[m][n] = sum_k A(m, k) B(n, k)
// with either operand stored contraction-innermost (K-major) or row-innermost (MN-major), which
// covers the layer's three products without a transposed copy: Z = X W^T (both K-major),
// dX = dZ W (W MN-major), dW = dZ^T X (both MN-major).
//
// Cut: a pair of CTAs (cta_group::2) shares a tile of 256 rows x NT <= 256 columns, the contraction
// runs in slices of 64 (a 128-byte swizzled row). Each CTA loads its own 128 rows of A and half of
// the columns of B, so a slice costs 32 KB of shared-memory fill per CTA instead of 48 KB and B crosses
// the L2 half as often. The walk over tiles is persistent; chunks cut a long contraction when there are few
// tiles. Few tokens have a kernel of their own below.
//
// Roles (20 warps): warp 0 the TMA producer, warp 1 the MMA issuer (in the pair's leader),
// warps 4..19 the epilogue: two groups of eight warps take the tiles in turn, so that one group's
// loads and stores fall into the other one's arithmetic; a warp takes four 32-row x 32-column blocks of
// a tile (TMEM lane = tile row), staged in shared memory by turns for their TMA stores. Group g reads TMEM accumulator g
// of 256 columns, so the epilogue of a tile overlaps the products of the next. Sixteen epilogue warps, because a memory-bound layer leaves
// about 16 issue slots per output value for everything, and the activation's chain of dependent
// instructions needs four warps per scheduler to hide (with eight warps of 64 columns a half and
// unpaired arithmetic the 65,536 x 256 -> 512 GELU layer took 46 us). Every wait is bounded (2 s of %globaltimer): on expiry the kernel records
// FLAREPP_ERR_TIMEOUT in the status word, every role leaves its loops, the producer waits for its
// copies in flight, the issuer for its products, and TMEM is freed.
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "linear_internal.h"
#include "tc_pair_ptx.cuh"

namespace flarepp {
namespace {

using namespace tc;

constexpr int kThreads = 640;
constexpr int kFirstEpiWarp = 4;
constexpr int kEpiWarps = 16;
constexpr int kSlice = 64;  // contraction values per ring stage: one 128-byte row
constexpr int kATile = 128 * kSlice * 2;
constexpr int kMaxNT = 256;
constexpr uint32_t kTmemCols = 512;
constexpr uint64_t kWaitLimitNs = 2000000000ull;
constexpr int kMaxStages = 8;
// the launches' numbers for the test hook of the bounded waits (flarepp_test_wait_fault)
constexpr int kProductKernel = 16, kFewKernel = 17;
constexpr int kDeepSlices = 12;  // slices of a contraction from which the deep form runs
constexpr int kBlockBytes = 32 * 32 * 2;  // what an epilogue warp stages at a time
constexpr int kNumBars = 2 * kMaxStages + 4 + 1 + 2 * kEpiWarps;

enum Out { kOutEpilogue, kOutPart };

// DEEP: the epilogue gives most of its shared memory to the ring (one staged block per warp, the
// bias read from global memory): for long contractions, where the products are the bound and their
// loads have to be further ahead.
template <int OUT, bool DEEP>
struct Cfg {
    static constexpr int kBTile = kMaxNT / 2 * kSlice * 2;
    static constexpr int kStage = kATile + kBTile;
    // per epilogue warp: 32-row x 32-column bf16 blocks
    static constexpr int kBlocks = DEEP ? 1 : 2;
    static constexpr int kStaging = OUT == kOutEpilogue ? kEpiWarps * kBlocks * kBlockBytes : 0;
    // per epilogue warp: the bias of its 128 columns of the tile, float32
    static constexpr int kBias = OUT == kOutEpilogue && !DEEP ? kEpiWarps * 128 * 4 : 0;
    static constexpr int kFit = (232448 - 1024 - kStaging - kBias - kNumBars * 8 - 16) / kStage;
    static constexpr int kStages = kFit > kMaxStages ? kMaxStages : kFit;
    static constexpr int kSmem = 1024 + kStages * kStage + kStaging + kBias + kNumBars * 8 + 16;
};

// The bound of every wait of a launch, where a wait that gave up is recorded, and (for tests) the ring
// item that CTA 0's producer never loads, or -1.
struct Waits {
    uint64_t limit_ns;
    int* status;
    int64_t withheld;
};

struct Gemm {
    int M, N, NT;
    int row_tiles, col_tiles, tiles, n_work;
    int slices, chunks;  // of the contraction; chunk c takes the slices c, c + chunks, ...
    int backward;        // walk the tiles from the last to the first
    uint32_t idesc;
    int act;
    int tma_out;  // the output's pitch suits TMA
    const __nv_bfloat16* bias;
    const __nv_bfloat16* R;
    __nv_bfloat16* Y;
    __nv_bfloat16* Z;
    float* part;
    int64_t ldp;
    Waits waits;
};

struct Work {
    int rt, ct, chunk;
};

// Work item v: the tiles of a chunk in groups of 8 row tiles, columns outermost within a group, so
// that the CTAs at work at one time share few rows of A and few columns of B in the L2.
__device__ __forceinline__ Work work_of(const Gemm& p, int v) {
    Work w;
    if (p.backward) v = p.n_work - 1 - v;
    w.chunk = v / p.tiles;
    const int t = v - w.chunk * p.tiles;
    const int per = 8 * p.col_tiles;
    const int g = t / per, in = t - g * per;
    const int rows = min(8, p.row_tiles - 8 * g);
    w.ct = in / rows;
    w.rt = 8 * g + in - w.ct * rows;
    return w;
}

template <int CG>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    return CG == 2 ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity);
}

// All lanes of a warp wait for a phase; false once this wait or another one of the CTA gave up.
template <int CG>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                          const Waits& w) {
    bool got = try_wait<CG>(bar, parity);
    if (!got) {
        const uint64_t t0 = globaltimer_ns();
        for (uint32_t i = 1;; ++i) {
            got = try_wait<CG>(bar, parity);
            if (got) break;
            if ((i & 63u) == 0) {
                if (*abort_flag) break;
                if (globaltimer_ns() - t0 > w.limit_ns) {
                    *abort_flag = 1;
                    if (w.status) atomicExch(w.status, (int)FLAREPP_ERR_TIMEOUT);
                    break;
                }
            }
        }
    }
    return __all_sync(0xffffffffu, got);
}

// One operand's tile of `rows` rows for the slice at contraction index k: K-major as one box of
// 64 x rows, MN-major as boxes of 64 rows x 64 contraction values ("atoms").
template <int CG, bool MN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* m, int row, int rows,
                                          int k, uint32_t bar) {
    if (!MN) {
        if (CG == 2) tma_load_2d_pair(dst, m, k, row, bar);
        else tma_load_2d(dst, m, k, row, bar);
    } else {
        for (int r = 0; r < rows; r += 64, dst += 64 * kSlice * 2) {
            if (CG == 2) tma_load_2d_pair(dst, m, row + r, k, bar);
            else tma_load_2d(dst, m, row + r, k, bar);
        }
    }
}

// The descriptor of the 16 contraction values at step s of a slice.
template <bool MN>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, int s) {
    return MN ? smem_desc(addr + s * 16 * 128, 64 * kSlice * 2, 1024, kSw128)
              : smem_desc(addr + s * 32, 16, 1024, kSw128);
}

template <bool A_MN, bool B_MN, int OUT, bool DEEP>
__global__ void __launch_bounds__(kThreads, 1)
    lin_gemm_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmY, const __grid_constant__ CUtensorMap tmZ,
                    const __grid_constant__ CUtensorMap tmR, const Gemm prm) {
    using C = Cfg<OUT, DEEP>;
    constexpr int kS = C::kStages;
    extern __shared__ uint8_t smem_raw[];
    // the same offset in both CTAs of a pair: the dynamic shared memory starts at one address
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* staging = smem + kS * C::kStage;
    uint64_t* bars = reinterpret_cast<uint64_t*>(staging + C::kStaging + C::kBias);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t full0 = smem_u32(bars);
    const uint32_t empty0 = full0 + 8u * kMaxStages;
    const uint32_t accfull0 = empty0 + 8u * kMaxStages;
    const uint32_t accempty0 = accfull0 + 16u;
    const uint32_t fin = accempty0 + 16u;
    const uint32_t rfull0 = fin + 8u;  // one per staged block
    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int first = (int)blockIdx.x / 2, pairs = (int)gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kS; ++s) {
            mbar_init(full0 + 8u * s, 1);
            mbar_init(empty0 + 8u * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(accfull0 + 8u * b, 1);
            mbar_init(accempty0 + 8u * b, kEpiWarps / 2 * 2);
        }
        mbar_init(fin, 1);
        for (int w = 0; w < 2 * kEpiWarps; ++w) mbar_init(rfull0 + 8u * w, 1);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    if (warp == 1) {
        tmem_alloc_pair(smem_u32(tmem_slot), kTmemCols);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // the other CTA's barriers exist
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer
        uint32_t it = 0;
        bool ok = true;
        const int b_rows = prm.NT / 2;
        // MN-major tiles come in whole 64-row atoms
        const uint32_t b_bytes = (uint32_t)(B_MN ? (b_rows + 63) / 64 * 64 : b_rows) * kSlice * 2;
        const uint32_t bytes = 2 * (kATile + b_bytes);
        for (int v = first; v < prm.n_work && ok; v += pairs) {
            const Work w = work_of(prm, v);
            const int m0 = (w.rt * 2 + (int)rank) * 128;
            const int n0 = w.ct * prm.NT + (int)rank * b_rows;
            for (int s = w.chunk; s < prm.slices; s += prm.chunks, ++it) {
                const int st = it % kS;
                if (it >= (uint32_t)kS &&
                    !warp_wait<2>(empty0 + 8u * st, (it / kS - 1) & 1, abort_flag, prm.waits)) {
                    ok = false;
                    break;
                }
                if (elect_one() && !(blockIdx.x == 0 && it == prm.waits.withheld)) {
                    const uint32_t dst = smem_u32(smem + st * C::kStage);
                    const uint32_t full = full0 + 8u * st;
                    if (rank == 0) mbar_expect_tx(full, bytes);
                    // both CTAs' bytes count on the leader's barrier
                    const uint32_t bar = map_to_rank(full, 0);
                    load_tile<2, A_MN>(dst, &tmA, m0, 128, s * kSlice, bar);
                    load_tile<2, B_MN>(dst + kATile, &tmB, n0, b_rows, s * kSlice, bar);
                }
                __syncwarp();
            }
        }
        if (!ok && rank == 0) {  // wait (bounded) until every copy issued has landed
            const uint64_t t0 = globaltimer_ns();
            for (int st = 0; st < kS && (uint32_t)st < it; ++st) {
                const uint32_t x = it - 1 - ((it - 1 - st) % kS);
                while (!mbar_try_wait(full0 + 8u * st, (x / kS) & 1) &&
                       globaltimer_ns() - t0 < kWaitLimitNs) {
                }
            }
        } else if (!ok) {  // its bytes count on the leader's barriers: give them a millisecond
            const uint64_t t0 = globaltimer_ns();
            while (globaltimer_ns() - t0 < 1000000ull) {
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------ MMA issuer
        uint32_t it = 0, j = 0;
        bool ok = true;
        for (int v = first; v < prm.n_work && ok; v += pairs, ++j) {
            const Work w = work_of(prm, v);
            const int ab = j & 1;
            if (j >= 2 &&
                !warp_wait<2>(accempty0 + 8u * ab, ((j >> 1) - 1) & 1, abort_flag, prm.waits)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t acc = tmem + ab * kMaxNT;
            for (int s = w.chunk; s < prm.slices; s += prm.chunks, ++it) {
                const int st = it % kS;
                if (!warp_wait<2>(full0 + 8u * st, (it / kS) & 1, abort_flag, prm.waits)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t a = smem_u32(smem + st * C::kStage);
                const uint32_t b = a + kATile;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kSlice / 16; ++k) {
                        const uint64_t ad = tile_desc<A_MN>(a, k), bd = tile_desc<B_MN>(b, k);
                        const uint32_t more = (s > w.chunk || k > 0) ? 1u : 0u;
                        mma_ss_pair(acc, ad, bd, prm.idesc, more);
                    }
                    mma_commit_pair(empty0 + 8u * st);
                }
                __syncwarp();
            }
            if (!ok) break;
            if (elect_one()) {
                mma_commit_pair(accfull0 + 8u * ab);
            }
            __syncwarp();
        }
        if (elect_one()) {
            mma_commit_pair(fin);
        }
        __syncwarp();
        const uint64_t tw = globaltimer_ns();
        while (!__all_sync(0xffffffffu, mbar_try_wait(fin, 0)) &&
               globaltimer_ns() - tw < kWaitLimitNs) {
        }
    } else if (warp >= kFirstEpiWarp) {
        // ------------------------------------------------------------ epilogue
        const int e = warp - kFirstEpiWarp;
        const int ab = e / (kEpiWarps / 2);  // this warp's group and accumulator
        const int q = warp % 4;              // the TMEM lanes this warp may read
        const int cfirst = 64 * (e % (kEpiWarps / 2) / 4);
        uint8_t* staged = staging + e * C::kBlocks * kBlockBytes;
        // the bias of columns cfirst .. cfirst + 63 and cfirst + 128 .. cfirst + 191 of the tile
        float* my_bias = reinterpret_cast<float*>(staging + C::kStaging) + e * 128;
        int bias_ct = -1;
        // 16-byte piece g of this lane's row in a staged block, swizzled as the maps expect it
        auto piece = [&](int h, int g) {
            return reinterpret_cast<uint4*>(staged + h * kBlockBytes + lane * 64 +
                                            ((g ^ (lane >> 1 & 3)) << 4));
        };
        const uint32_t rfull = rfull0 + 16u * e;
        uint32_t phase = 0, r_phase = 0;
        bool ok = true;
        for (int v = first + ab * pairs; v < prm.n_work && ok; v += 2 * pairs, phase ^= 1) {
            const Work w = work_of(prm, v);
            const int row0 = (w.rt * 2 + (int)rank) * 128 + 32 * q;
            const int n0 = w.ct * prm.NT;  // first column of the tile
            // columns of the tile that exist
            const int width = row0 < prm.M ? min(prm.NT, prm.N - n0) : 0;
            const int rows = min(32, prm.M - row0);
            const uint32_t acc = tmem + ((uint32_t)(32 * q) << 16) + ab * kMaxNT;
            const bool tma_r = OUT == kOutEpilogue && prm.R && prm.tma_out;
            // block h of R at column c, into the staged block that Y leaves from
            auto fetch_r = [&](int h, int c) {
                if (lane == 0) {
                    mbar_expect_tx(rfull + 8u * h, kBlockBytes);
                    tma_load_2d(smem_u32(staged + h * kBlockBytes), &tmR, n0 + c, row0, rfull + 8u * h);
                }
            };
            if (tma_r && !prm.Z) {  // ahead of the products
                if (lane == 0) bulk_wait_read();
                for (int h = 0; h < C::kBlocks; ++h)
                    if (cfirst + 32 * h < width) fetch_r(h, cfirst + 32 * h);
            }
            if (C::kBias && prm.bias && bias_ct != w.ct) {
                bias_ct = w.ct;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = n0 + cfirst + 128 * (i / 2) + 32 * (i % 2) + lane;
                    my_bias[32 * i + lane] = n < prm.N ? __bfloat162float(prm.bias[n]) : 0.f;
                }
                __syncwarp();
            }
            ok = warp_wait<2>(accfull0 + 8u * ab, phase, abort_flag, prm.waits);
            tc_fence_after();
            for (int c = cfirst; c < width && ok; c += c % 64 ? 96 : 32) {
                const int h = DEEP ? 0 : c / 32 & 1;  // staged block
                if (OUT != kOutEpilogue) {
                    float x[32];
                    tmem_ld32(acc + c, reinterpret_cast<uint32_t*>(x));
                    tmem_wait_ld32(reinterpret_cast<uint32_t*>(x));
                    const int row = row0 + lane, at = n0 + c;
                    if (row >= prm.M) continue;
                    float* d = prm.part + ((int64_t)w.chunk * prm.M + row) * prm.ldp + at;
                    const int n = min(prm.NT - c, (int)prm.ldp - at);
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (i < n)
                            *reinterpret_cast<float4*>(d + i) =
                                make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                    continue;
                }
                // sums with the bias, as 16 pairs
                uint64_t x[16];
                auto load = [&] {
                    uint32_t r[32];
                    tmem_ld32(acc + c, r);
                    tmem_wait_ld32(r);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        x[i] = pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
                    if (!prm.bias) return;
                    if (DEEP) {
                        const int at = n0 + c;
                        if (at + 32 <= prm.N) {
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                const uint4 u = __ldg(reinterpret_cast<const uint4*>(prm.bias + at) + g);
                                x[4 * g] = add2(x[4 * g], unpack_bf16x2(u.x));
                                x[4 * g + 1] = add2(x[4 * g + 1], unpack_bf16x2(u.y));
                                x[4 * g + 2] = add2(x[4 * g + 2], unpack_bf16x2(u.z));
                                x[4 * g + 3] = add2(x[4 * g + 3], unpack_bf16x2(u.w));
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int n = at + 2 * i;
                                x[i] = add2(x[i], pair(n < prm.N ? __bfloat162float(prm.bias[n]) : 0.f,
                                                       n + 1 < prm.N ? __bfloat162float(prm.bias[n + 1]) : 0.f));
                            }
                        }
                        return;
                    }
                    const float4* b4 = reinterpret_cast<const float4*>(my_bias + (c / 128) * 64 + (c & 32));
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const float4 f = b4[g];
                        x[2 * g] = add2(x[2 * g], pair(f.x, f.y));
                        x[2 * g + 1] = add2(x[2 * g + 1], pair(f.z, f.w));
                    }
                };
                auto store = [&](int hb) {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *piece(hb, g) = make_uint4(pack_bf16x2(x[4 * g]), pack_bf16x2(x[4 * g + 1]),
                                                   pack_bf16x2(x[4 * g + 2]), pack_bf16x2(x[4 * g + 3]));
                };
                // value (r, cc) of a staged block, for outputs whose lines TMA cannot address
                auto value = [&](int hb, int r, int cc) {
                    return reinterpret_cast<__nv_bfloat16*>(staged + hb * kBlockBytes + r * 64 +
                                                            (((cc >> 3) ^ (r >> 1 & 3)) << 4) + (cc & 7) * 2);
                };
                const int cols = min(32, width - c);
                auto flush = [&](int hb, const CUtensorMap* map, __nv_bfloat16* out) {
                    if (prm.tma_out) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(map, smem_u32(staged + hb * kBlockBytes), n0 + c, row0);
                            bulk_commit();
                        }
                    } else {
                        __syncwarp();
#pragma unroll 8
                        for (int r = 0; r < 32; ++r)
                            if (r < rows && lane < cols)
                                out[(int64_t)(row0 + r) * prm.N + n0 + c + lane] = *value(hb, r, lane);
                        __syncwarp();
                    }
                };
                // Without Z and R, block h was last stored two blocks ago; with Z the two staged blocks are
                // Z's and Y's, and each waits for the store before.
                const int hy = prm.Z ? 0 : h;
                load();
                if (prm.Z) {
                    if (lane == 0) bulk_wait_read();
                    __syncwarp();
                    store(C::kBlocks - 1);
                    flush(C::kBlocks - 1, &tmZ, prm.Z);
                    if (DEEP) {  // Y leaves from the same block
                        if (lane == 0) bulk_wait_read();
                        __syncwarp();
                    }
                    if (tma_r) fetch_r(0, c);
                }
                if (c + (c % 64 ? 96 : 32) >= width) {  // the last block: the accumulator is read
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(map_to_rank(accempty0 + 8u * ab, 0));
                }
                switch (prm.act) {
                    case FLAREPP_ACT_RELU:
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = act_value2(FLAREPP_ACT_RELU, x[i]);
                        break;
                    case FLAREPP_ACT_GELU:
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = act_value2(FLAREPP_ACT_GELU, x[i]);
                        break;
                    case FLAREPP_ACT_SILU:
#pragma unroll
                        for (int i = 0; i < 16; ++i) x[i] = act_value2(FLAREPP_ACT_SILU, x[i]);
                        break;
                }
                if (prm.R) {
                    if (tma_r) {
                        ok = warp_wait<1>(rfull + 8u * hy, r_phase >> hy & 1, abort_flag, prm.waits);
                        if (!ok) break;
                        r_phase ^= 1u << hy;
                    } else {
#pragma unroll 8
                        for (int r = 0; r < 32; ++r)
                            if (r < rows && lane < cols)
                                *value(hy, r, lane) = prm.R[(int64_t)(row0 + r) * prm.N + n0 + c + lane];
                        __syncwarp();
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const uint4 u = *piece(hy, g);
                        x[4 * g] = add2(x[4 * g], unpack_bf16x2(u.x));
                        x[4 * g + 1] = add2(x[4 * g + 1], unpack_bf16x2(u.y));
                        x[4 * g + 2] = add2(x[4 * g + 2], unpack_bf16x2(u.z));
                        x[4 * g + 3] = add2(x[4 * g + 3], unpack_bf16x2(u.w));
                    }
                } else if (!prm.Z) {
                    if (lane == 0) {
                        if (DEEP) bulk_wait_read();
                        else bulk_wait_read_1();
                    }
                    __syncwarp();
                }
                store(hy);
                flush(hy, &tmY, prm.Y);
                // this staged block's next turn
                const int then = DEEP ? c + (c % 64 ? 96 : 32) : c + 128;
                if (tma_r && !prm.Z && then < width) {
                    if (lane == 0) bulk_wait_read();
                    fetch_r(h, then);
                }
            }
            if (ok && (width <= cfirst || OUT != kOutEpilogue)) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(accempty0 + 8u * ab, 0));
            }
        }
        if (OUT == kOutEpilogue) {
            if (!ok && prm.R) {  // a wait gave up: let the copies in flight land (a millisecond)
                const uint64_t t0 = globaltimer_ns();
                while (globaltimer_ns() - t0 < 1000000ull) {
                }
            }
            if (lane == 0) bulk_wait_all();
        }
    }
    tc_fence_before();
    __syncthreads();
    // no CTA leaves while the other one may still signal it or read its shared memory
    cluster_sync();
    tc_fence_after();
    if (warp == 1) tmem_dealloc_pair(tmem, kTmemCols);
}

// ------------------------------------------------------------------ few rows
// The layer for up to 256 rows of tokens: the weights are the tile's rows (128 of them, whatever the
// number of tokens) and the tokens its columns, so the tensor cores' 128 rows are never idle and the
// weights, whose bytes are the bound, are read once. A cluster of up to eight CTAs shares a tile, each
// with every S-th slice of the contraction, so that a few tiles still draw on many SMs; the CTAs
// leave their float32 sums in shared memory, and each adds a share of the columns over the cluster in
// rank order and runs the epilogue on it. One launch, no workspace (48 rows of 4096 -> 1001 took 8.8 us
// as chunk sums in memory and a second kernel).
constexpr int kFewThreads = 256;
constexpr int kFewStages = 4;
constexpr int kFewRing = kFewStages * (kATile + kMaxNT * kSlice * 2);
constexpr int kFewBars = 2 * kFewStages + 1;
constexpr int kFewSmem = 1024 + kFewRing + kFewBars * 8 + 16;
static_assert(kMaxNT * 128 * 4 <= kFewRing, "the sums reuse the ring");

struct Few {
    int M, N, NT;  // weights' rows, tokens, columns of the tile
    int slices, share;  // slices of the contraction, CTAs per tile
    uint32_t idesc, tmem_cols;
    int act;
    const __nv_bfloat16* bias;  // [M]
    const __nv_bfloat16* R;     // [N][M], as Y and Z
    __nv_bfloat16* Y;
    __nv_bfloat16* Z;
    Waits waits;
};

__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr));
    return v;
}

template <bool A_MN>
__global__ void __launch_bounds__(kFewThreads, 1)
    lin_few_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                   const Few prm) {
    extern __shared__ uint8_t smem_raw[];
    // the same offset in every CTA of the cluster
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kFewRing);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kFewBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8u * kFewStages;
    const uint32_t done = empty0 + 8u * kFewStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = prm.share > 1 ? (int)cluster_rank() : 0;
    const int m0 = (int)blockIdx.x / prm.share * 128;
    const uint32_t stage_bytes = kATile + prm.NT * kSlice * 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kFewStages; ++s) {
            mbar_init(full0 + 8u * s, 1);
            mbar_init(empty0 + 8u * s, 1);
        }
        mbar_init(done, 1);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tmA);
        prefetch_tmap(&tmB);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), prm.tmem_cols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    if (warp == 0) {
        uint32_t it = 0;
        bool ok = true;
        for (int s = rank; s < prm.slices; s += prm.share, ++it) {
            const int st = it % kFewStages;
            if (it >= (uint32_t)kFewStages &&
                !warp_wait<1>(empty0 + 8u * st, (it / kFewStages - 1) & 1, abort_flag, prm.waits)) {
                ok = false;
                break;
            }
            if (elect_one() && !(blockIdx.x == 0 && it == prm.waits.withheld)) {
                const uint32_t dst = smem_u32(smem + st * (kFewRing / kFewStages));
                mbar_expect_tx(full0 + 8u * st, stage_bytes);
                load_tile<1, A_MN>(dst, &tmA, m0, 128, s * kSlice, full0 + 8u * st);
                load_tile<1, false>(dst + kATile, &tmB, 0, prm.NT, s * kSlice, full0 + 8u * st);
            }
            __syncwarp();
        }
        if (!ok) {  // wait (bounded) until every copy issued has landed
            const uint64_t t0 = globaltimer_ns();
            for (int st = 0; st < kFewStages && (uint32_t)st < it; ++st) {
                const uint32_t x = it - 1 - ((it - 1 - st) % kFewStages);
                while (!mbar_try_wait(full0 + 8u * st, (x / kFewStages) & 1) &&
                       globaltimer_ns() - t0 < kWaitLimitNs) {
                }
            }
        }
    } else if (warp == 1) {
        uint32_t it = 0;
        for (int s = rank; s < prm.slices; s += prm.share, ++it) {
            const int st = it % kFewStages;
            if (!warp_wait<1>(full0 + 8u * st, (it / kFewStages) & 1, abort_flag, prm.waits)) break;
            tc_fence_after();
            const uint32_t a = smem_u32(smem + st * (kFewRing / kFewStages)), b = a + kATile;
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < kSlice / 16; ++k)
                    mma_ss(tmem, tile_desc<A_MN>(a, k), tile_desc<false>(b, k), prm.idesc,
                           (it > 0 || k > 0) ? 1u : 0u);
                mma_commit(empty0 + 8u * st);
            }
            __syncwarp();
        }
        if (elect_one()) mma_commit(done);
        __syncwarp();
    }
    __syncwarp();
    // every warp: the sums from TMEM into sums[token][128], over the ring (its copies and products
    // are done)
    const bool ok = warp_wait<1>(done, 0, abort_flag, prm.waits);
    float* sums = reinterpret_cast<float*>(smem);
    __syncthreads();  // an issuer that gave up has left its loop too
    tc_fence_after();
    if (ok) {
        const int q = warp % 4;
        float* mine = sums + 32 * q + lane;
        for (int c = 16 * (warp / 4); c < prm.NT; c += 32) {
            uint32_t r[16];
            tmem_ld16(tmem + ((uint32_t)(32 * q) << 16) + c, r);
            tmem_wait_ld16(r);
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(c + i) * 128] = __uint_as_float(r[i]);
        }
    }
    tc_fence_before();
    if (prm.share > 1) cluster_sync();
    else __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, prm.tmem_cols);
    // a warp takes a token at a time, a lane four of its outputs
    const int m = m0 + 4 * lane;
    const bool vec = prm.M % 4 == 0;
    for (int t = rank + prm.share * warp; t < prm.N; t += prm.share * (kFewThreads / 32)) {
        if (m >= prm.M) break;
        const uint32_t at = smem_u32(sums + t * 128 + 4 * lane);
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < prm.share) v[k] = load_cluster(prm.share > 1 ? map_to_rank(at, k) : at);
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < prm.share) {
                x[0] += v[k].x;
                x[1] += v[k].y;
                x[2] += v[k].z;
                x[3] += v[k].w;
            }
        const int64_t o = (int64_t)t * prm.M + m;
        if (prm.bias)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (m + k < prm.M) x[k] += __bfloat162float(prm.bias[m + k]);
        if (prm.Z) {
            if (vec)
                *reinterpret_cast<uint2*>(prm.Z + o) =
                    make_uint2(pack_bf16x2(pair(x[0], x[1])), pack_bf16x2(pair(x[2], x[3])));
            else
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (m + k < prm.M) prm.Z[o + k] = __float2bfloat16_rn(x[k]);
        }
        const float2 y0 = halves(act_value2(prm.act, pair(x[0], x[1])));
        const float2 y1 = halves(act_value2(prm.act, pair(x[2], x[3])));
        float y[4] = {y0.x, y0.y, y1.x, y1.y};
        if (prm.R)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (m + k < prm.M) y[k] += __bfloat162float(prm.R[o + k]);
        if (vec)
            *reinterpret_cast<uint2*>(prm.Y + o) =
                make_uint2(pack_bf16x2(pair(y[0], y[1])), pack_bf16x2(pair(y[2], y[3])));
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (m + k < prm.M) prm.Y[o + k] = __float2bfloat16_rn(y[k]);
    }
    __syncwarp();
    if (prm.share > 1) cluster_sync();  // the other CTAs may still read this one's sums
}

// ------------------------------------------------------------------ host side

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> fn{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 f = fn.load(std::memory_order_acquire);
    if (f) return f;
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
        fn.store(f = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p),
                 std::memory_order_release);
    return f;
}

// bf16 [lines][inner] with `pitch` elements from line to line, boxes of box_inner x box_lines,
// swizzled to their 128- or 64-byte lines
bool make_map(CUtensorMap* m, const void* base, int64_t inner, int64_t lines, int64_t pitch,
              int box_inner, int box_lines) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)lines};
    cuuint64_t strides[1] = {(cuuint64_t)pitch * 2};
    cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_lines};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_inner == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool A_MN, bool B_MN, int OUT, bool DEEP>
cudaError_t launch(const CUtensorMap* m, const Gemm& p, cudaStream_t st) {
    using C = Cfg<OUT, DEEP>;
    static_assert(C::kSmem <= 232448 && C::kStages >= 3, "shared memory budget");
    auto kernel = lin_gemm_kernel<A_MN, B_MN, OUT, DEEP>;
    static std::atomic<int> fits[64];  // tiles that run at once on each device (0: not asked yet)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = C::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    int n = fits[dev].load();
    if (n == 0) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        if (e != cudaSuccess) return e;
        n = kNumSMs / 2;
        // a die's odd SM cannot hold a pair
        cfg.gridDim = dim3(kNumSMs / 2 * 2);
        int most = 0;
        cudaLaunchConfig_t ask = cfg;
        ask.attrs = &attr[1];
        ask.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&most, kernel, &ask);
        if (e != cudaSuccess) return e;
        if (most > 0 && most < n) n = most;
        fits[dev].store(n);
    }
    cfg.gridDim = dim3((unsigned)((p.n_work < n ? p.n_work : n) * 2));
    return cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], m[2], m[3], m[4], p);
}

template <bool A_MN>
cudaError_t launch_few(const CUtensorMap* m, const Few& p, unsigned tiles, cudaStream_t st) {
    auto kernel = lin_few_kernel<A_MN>;
    static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
        if (e != cudaSuccess) return e;
        ready.fetch_or(uint64_t(1) << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(tiles * (unsigned)p.share);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = kFewSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)p.share;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = p.share > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], p);
}

}  // namespace

cudaError_t lin_few(int64_t rows, int64_t cols, int64_t K, const LinOperand& x,
                    const LinOperand& w, const LinEpilogue& e, int* status, cudaStream_t st) {
    Few p{};
    p.M = (int)cols;
    p.N = (int)rows;
    p.NT = (int)cdiv(rows, 16) * 16;
    p.slices = (int)cdiv(K, kSlice);
    const int64_t tiles = cdiv(cols, 128);
    p.share = 1;  // as many CTAs as the SMs take, with two slices each at least
    while (p.share < 8 && tiles * p.share * 2 <= kNumSMs && p.slices >= 4 * p.share) p.share *= 2;
    p.idesc = idesc_bf16_f32(128, p.NT, w.mn, false);
    p.tmem_cols = 32;
    while ((int)p.tmem_cols < p.NT) p.tmem_cols *= 2;
    p.act = e.act;
    p.bias = (const __nv_bfloat16*)e.bias;
    p.R = (const __nv_bfloat16*)e.R;
    p.Y = (__nv_bfloat16*)e.Y;
    p.Z = (__nv_bfloat16*)e.Z;
    p.waits.status = status;
    test_fault_for(kFewKernel, &p.waits.limit_ns, &p.waits.withheld);
    CUtensorMap m[2];
    const bool ok = (w.mn ? make_map(&m[0], w.t, cols, K, w.pitch, 64, kSlice)
                          : make_map(&m[0], w.t, K, cols, w.pitch, kSlice, 128)) &&
                    make_map(&m[1], x.t, K, rows, x.pitch, kSlice, p.NT);
    if (!ok) return cudaErrorInvalidValue;
    return w.mn ? launch_few<true>(m, p, (unsigned)tiles, st)
                : launch_few<false>(m, p, (unsigned)tiles, st);
}

LinPlan lin_plan(int64_t M, int64_t N, int64_t K) {
    LinPlan p{};
    // equal column tiles, in whole 32-column blocks where there are several
    const int64_t ct = cdiv(N, kMaxNT);
    p.NT = (int)(ct == 1 ? cdiv(N, 16) * 16 : cdiv(cdiv(N, ct), 32) * 32);
    const int64_t tiles = cdiv(M, 256) * cdiv(N, p.NT);
    // How many chunks: the time of the waves of work items (0.3 us a slice and about 4 us of a wave's
    // own) and, with more than one, of writing and reading the partial sums (8 bytes a value at about 5 TB/s)
    // and of one launch more. Chunks have at least four slices.
    const int64_t slices = cdiv(K, kSlice), units = kNumSMs / 2;
    double best = 0;
    for (int64_t c = 1; c <= 64 && (c == 1 || slices / c >= 4); ++c) {
        const double waves = (double)cdiv(tiles * c, units);
        const double us = waves * (0.3 * (double)cdiv(slices, c) * p.NT / kMaxNT + 4) +
                          (c > 1 ? 3 + (double)c * M * N * 8 / 5e6 : 0);
        if (c == 1 || us < best) {
            best = us;
            p.chunks = (int)c;
        }
    }
    return p;
}

cudaError_t lin_gemm(const LinPlan& plan, int64_t M, int64_t N, int64_t K, const LinOperand& a,
                     const LinOperand& b, const LinEpilogue& e, int* status, cudaStream_t st) {
    Gemm p{};
    p.M = (int)M;
    p.N = (int)N;
    p.NT = plan.NT;
    const int64_t row_tiles = cdiv(M, 256), col_tiles = cdiv(N, plan.NT);
    if (row_tiles * col_tiles * plan.chunks > 0x7fffffff) return cudaErrorInvalidValue;
    p.row_tiles = (int)row_tiles;
    p.col_tiles = (int)col_tiles;
    p.tiles = (int)(row_tiles * col_tiles);
    p.n_work = p.tiles * plan.chunks;
    p.slices = (int)cdiv(K, kSlice);
    p.chunks = plan.chunks;
    p.backward = e.backward;
    p.idesc = idesc_bf16_f32(256, plan.NT, a.mn, b.mn);
    p.act = e.act;
    p.tma_out = N % 8 == 0;
    p.bias = (const __nv_bfloat16*)e.bias;
    p.R = (const __nv_bfloat16*)e.R;
    p.Y = (__nv_bfloat16*)e.Y;
    p.Z = (__nv_bfloat16*)e.Z;
    p.part = e.part;
    p.ldp = e.ldp;
    p.waits.status = status;
    test_fault_for(kProductKernel, &p.waits.limit_ns, &p.waits.withheld);
    CUtensorMap m[5];
    const int b_rows = plan.NT / 2;
    bool ok = a.mn ? make_map(&m[0], a.t, M, K, a.pitch, 64, kSlice)
                   : make_map(&m[0], a.t, K, M, a.pitch, kSlice, 128);
    ok = ok && (b.mn ? make_map(&m[1], b.t, N, K, b.pitch, 64, kSlice)
                     : make_map(&m[1], b.t, K, N, b.pitch, kSlice, b_rows));
    m[2] = m[3] = m[4] = m[0];  // unused unless set below
    if (!e.part && p.tma_out) {
        ok = ok && make_map(&m[2], e.Y, N, M, N, 32, 32);
        if (e.Z) ok = ok && make_map(&m[3], e.Z, N, M, N, 32, 32);
        if (e.R) ok = ok && make_map(&m[4], e.R, N, M, N, 32, 32);
    }
    if (!ok) return cudaErrorInvalidValue;
    const bool part = e.part != nullptr;
    const bool deep = p.slices >= kDeepSlices;
    if (a.mn)
        return part ? launch<true, true, kOutPart, true>(m, p, st)
               : deep          ? launch<true, true, kOutEpilogue, true>(m, p, st)
                               : launch<true, true, kOutEpilogue, false>(m, p, st);
    if (b.mn)
        return part ? launch<false, true, kOutPart, true>(m, p, st)
               : deep          ? launch<false, true, kOutEpilogue, true>(m, p, st)
                               : launch<false, true, kOutEpilogue, false>(m, p, st);
    return part ? launch<false, false, kOutPart, true>(m, p, st)
           : deep          ? launch<false, false, kOutEpilogue, true>(m, p, st)
                           : launch<false, false, kOutEpilogue, false>(m, p, st);
}

}  // namespace flarepp
