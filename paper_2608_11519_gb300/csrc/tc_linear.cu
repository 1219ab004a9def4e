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
// tiles. Few tokens (tc_linear_few.cu) and the backward of narrow layers (tc_linear_fused.cu) have kernels of
// their own.
//
// Roles (20 warps): warp 0 the TMA producer, warp 1 the MMA issuer (in the pair's leader),
// warps 4..19 the epilogue: two groups of eight warps take the tiles in turn, so that one group's
// loads and stores fall into the other one's arithmetic; a warp takes four 32-row x 32-column blocks of
// a tile (TMEM lane = tile row), staged in shared memory by turns for their TMA stores. Group g reads
// TMEM accumulator g of 256 columns, so the epilogue of a tile overlaps the products of the next.
// Every wait is bounded (2 s of %globaltimer): on expiry the kernel records FLAREPP_ERR_TIMEOUT in the
// status word, every role leaves its loops, the producer waits for its copies in flight, the issuer for
// its products, and TMEM is freed.
//
// What bounds it: long contractions the tensor cores (16384 x 4096 x 4096: 317 us, 1732 TFLOP/s, after a pause
// of 50 ms; 323 one after another, the clock then held at 1.5 GHz by the power limit); wide outputs of short
// contractions the writes, which HBM takes at 4.0 TB/s where nothing is read (measured with fills) and at up to
// 2.4 beside twice as many reads. GELU takes 24 cycles of the special-function unit and 20 of the multiply-add
// pipe (22 with the bias) per pair of outputs and scheduler, about what the writes leave, and a group waits for
// its accumulator's next products after that: 65,536 x 256 -> 512 takes 23.0 us without an activation, 28.1 with
// SiLU and 31.3 with GELU. Measured and left: sixteen warps on every tile (36 us: a tile's fixed latencies are
// then in every warp's way), 16-column halves with the next loads ahead (38 us: too few independent chains),
// eight warps of 64 columns and unpaired arithmetic (46 us), more registers for the epilogue by setmaxnreg
// (spills).
#include <type_traits>

#include "tc_linear_common.cuh"

namespace flarepp {
namespace {

constexpr int kThreads = 640;
constexpr int kFirstEpiWarp = 4;
constexpr int kEpiWarps = 16;
constexpr int kMaxStages = 8;
constexpr int kDeepSlices = 12;  // slices of a contraction from which the deep form runs
constexpr int kNumBars = 2 * kMaxStages + 4 + 1 + 2 * kEpiWarps;

// outputs by TMA (N a multiple of 8), by plain stores, or the partial sums of a cut contraction
enum Out { kOutTma, kOutPlain, kOutPart };

// DEEP: the epilogue gives most of its shared memory to the ring (one staged block per warp, the
// bias read from global memory): for long contractions, where the products are the bound and their
// loads have to be further ahead.
template <int OUT, bool DEEP>
struct Cfg {
    static constexpr int kBTile = kMaxNT / 2 * kSlice * 2;
    static constexpr int kStage = kATile + kBTile;
    // per epilogue warp: 32-row x 32-column bf16 blocks
    static constexpr int kBlocks = DEEP ? 1 : 2;
    static constexpr int kStaging = OUT != kOutPart ? kEpiWarps * kBlocks * kBlockBytes : 0;
    // per epilogue warp: the bias of its 128 columns of the tile, float32
    static constexpr int kBias = OUT != kOutPart && !DEEP ? kEpiWarps * 128 * 4 : 0;
    static constexpr int kFit = (kMaxSmem - 1024 - kStaging - kBias - kNumBars * 8 - 16) / kStage;
    static constexpr int kStages = kFit > kMaxStages ? kMaxStages : kFit;
    static constexpr int kSmem = 1024 + kStages * kStage + kStaging + kBias + kNumBars * 8 + 16;
};

struct Gemm {
    int M, N, NT;
    int row_tiles, col_tiles, tiles, n_work;
    int slices, chunks;  // of the contraction; chunk c takes the slices c, c + chunks, ...
    int backward;        // walk the tiles from the last to the first
    uint32_t idesc;
    int act;
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
            linger();
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
        int turn = 0;  // the staged block whose store is the longest ago
        bool ok = true;
        for (int v = first + ab * pairs; v < prm.n_work && ok; v += 2 * pairs, phase ^= 1) {
            const Work w = work_of(prm, v);
            const int row0 = (w.rt * 2 + (int)rank) * 128 + 32 * q;
            const int n0 = w.ct * prm.NT;  // first column of the tile
            // columns of the tile that exist
            const int width = row0 < prm.M ? min(prm.NT, prm.N - n0) : 0;
            const int rows = min(32, prm.M - row0);
            const uint32_t acc = tmem + ((uint32_t)(32 * q) << 16) + ab * kMaxNT;
            const bool tma_r = OUT == kOutTma && prm.R;
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
                // Staged block: with R on its way into it, by the column; else the two by turns, across
                // tiles too (widths such as 160 have an odd number of blocks), so that the wait for all
                // stores but the last one is a wait for this block's.
                const int h = DEEP ? 0 : tma_r ? c / 32 & 1 : turn;
                if (OUT == kOutPart) {
                    float x[32];
                    tmem_ld32(acc + c, reinterpret_cast<uint32_t*>(x));
                    tmem_wait_ld32(reinterpret_cast<uint32_t*>(x));
                    const int row = row0 + lane, at = n0 + c;
                    const int n = row < prm.M ? min(prm.NT - c, (int)prm.ldp - at) : 0;
                    float* d = prm.part + ((int64_t)w.chunk * prm.M + row) * prm.ldp + at;
#pragma unroll
                    for (int i = 0; i < 32; i += 4)
                        if (i < n)
                            *reinterpret_cast<float4*>(d + i) =
                                make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
                    __syncwarp();  // the next load from TMEM wants the whole warp
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
                                const uint4 u = reinterpret_cast<const uint4*>(prm.bias + at)[g];
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
                // Value (r, cc) of a staged block, for outputs whose lines TMA cannot address. Those leave
                // (and R comes) a row at a time in words of VW values, VW = 4, 2 or 1 by what divides N.
                auto value = [&](int hb, int r, int cc) {
                    return staged + hb * kBlockBytes + r * 64 + (((cc >> 3) ^ (r >> 1 & 3)) << 4) +
                           (cc & 7) * 2;
                };
                const int cols = min(32, width - c);
                auto each_word = [&](auto word, int hb, auto act_on) {
                    using V = decltype(word);
                    constexpr int VW = sizeof(V) / 2;
                    const int cc = lane % (32 / VW) * VW;
#pragma unroll 16
                    for (int r = lane / (32 / VW); r < 32; r += VW)
                        if (r < rows && cc < cols)
                            act_on(reinterpret_cast<V*>(value(hb, r, cc)),
                                   (int64_t)(row0 + r) * prm.N + n0 + c + cc);
                };
                auto copy_rows = [&](int hb, auto act_on) {
                    if (prm.N % 4 == 0) each_word(uint2{}, hb, act_on);
                    else if (prm.N % 2 == 0) each_word(uint32_t{}, hb, act_on);
                    else each_word(uint16_t{}, hb, act_on);
                };
                auto flush = [&](int hb, const CUtensorMap* map, __nv_bfloat16* out) {
                    if (OUT == kOutTma) {
                        fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(map, smem_u32(staged + hb * kBlockBytes), n0 + c, row0);
                            bulk_commit();
                        }
                    } else {
                        __syncwarp();
                        copy_rows(hb, [&](auto* word, int64_t i) {
                            *reinterpret_cast<decltype(word)>(out + i) = *word;
                        });
                        __syncwarp();
                    }
                };
                // Without Z and R, block h was last stored two stores ago; with Z the two staged blocks are
                // Z's and Y's, and each waits for the store before.
                const int hy = prm.Z ? 0 : h;
                if (OUT == kOutPlain && prm.R) {  // while no sums take registers
                    copy_rows(hy, [&](auto* word, int64_t i) {
                        *word = *reinterpret_cast<const std::remove_pointer_t<decltype(word)>*>(prm.R + i);
                    });
                    __syncwarp();
                }
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
                turn ^= 1;
                // this staged block's next turn
                const int then = DEEP ? c + (c % 64 ? 96 : 32) : c + 128;
                if (tma_r && !prm.Z && then < width) {
                    if (lane == 0) bulk_wait_read();
                    fetch_r(h, then);
                }
                __syncwarp();  // lane 0 comes back before the next load from TMEM
            }
            if (ok && (width <= cfirst || OUT == kOutPart)) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(map_to_rank(accempty0 + 8u * ab, 0));
            }
        }
        if (OUT == kOutTma) {
            if (!ok && prm.R) linger();  // the blocks of R in flight
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

// ------------------------------------------------------------------ host side

template <bool A_MN, bool B_MN, int OUT, bool DEEP>
cudaError_t launch(const CUtensorMap* m, const Gemm& p, cudaStream_t st) {
    using C = Cfg<OUT, DEEP>;
    static_assert(C::kSmem <= kMaxSmem && C::kStages >= 3, "shared memory budget");
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

}  // namespace

cudaError_t take_product_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

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
    if (!e.part && N % 8 == 0) {
        ok = ok && make_map(&m[2], e.Y, N, M, N, 32, 32);
        if (e.Z) ok = ok && make_map(&m[3], e.Z, N, M, N, 32, 32);
        if (e.R) ok = ok && make_map(&m[4], e.R, N, M, N, 32, 32);
    }
    if (!ok) return cudaErrorInvalidValue;
    // plain stores need the second staged block (for R beside Z), so they run the form that has it
    const Out out = e.part ? kOutPart : N % 8 ? kOutPlain : kOutTma;
    const bool deep = p.slices >= kDeepSlices;
    if (a.mn)
        return out == kOutPart    ? launch<true, true, kOutPart, true>(m, p, st)
               : out == kOutPlain ? launch<true, true, kOutPlain, false>(m, p, st)
               : deep             ? launch<true, true, kOutTma, true>(m, p, st)
                                  : launch<true, true, kOutTma, false>(m, p, st);
    if (b.mn)
        return out == kOutPart    ? launch<false, true, kOutPart, true>(m, p, st)
               : out == kOutPlain ? launch<false, true, kOutPlain, false>(m, p, st)
               : deep             ? launch<false, true, kOutTma, true>(m, p, st)
                                  : launch<false, true, kOutTma, false>(m, p, st);
    return out == kOutPart    ? launch<false, false, kOutPart, true>(m, p, st)
           : out == kOutPlain ? launch<false, false, kOutPlain, false>(m, p, st)
           : deep             ? launch<false, false, kOutTma, true>(m, p, st)
                              : launch<false, false, kOutTma, false>(m, p, st);
}

}  // namespace flarepp
