// The backward of a narrow linear layer with an activation (tcgen05 / TMEM / TMA, CTA pairs): in one
// pass over dY and Z,
//   dZ = dY o act'(Z) (kept for dW),  dX = dZ W,  and the column sums of dZ for db.
//
// A layer whose inputs fit one column tile (in <= 256) meets each value of dZ once on the way to dX, so dZ is
// made where the product needs it: the slices of dY and Z come into the ring as they are, eight warps
// turn dY's tile into dZ's in place (the swizzled tile that the tensor cores read), store it for dW and
// add up its columns, and the pair's leader multiplies. A separate pass would read dZ once more, and its
// launch: for 131,072 rows of 256 -> 512 with GELU, dZ with its column sums and dX take 107 us apart and 92
// here, of which the bytes (268 MB read, 201 MB written) are about 70. What is left is the ring: four stages of
// 32 KB, of which two are being made or multiplied, keep some 64 KB a SM in flight.
//
// Roles (28 warps): warp 0 the TMA producer of dY and Z, warp 2 that of W, warp 1 the MMA issuer (in the
// pair's leader), warp 3 dZ's stores, warps 4..19 dZ, warps 20..27 the epilogue, which writes dX from two
// TMEM accumulators of 256 columns by turns. The dZ warps are two groups of eight (16 rows of the CTA's 128 a
// warp) that take
// the slices in turn: making a slice is a chain of latencies (shared memory, the slope, the proxy fence),
// and one group alone, of eight or of sixteen warps, took 115 us for the layer above, as did stores
// issued by the dZ warps themselves, which freed a stage only at their next slice. A ring stage is
// free again when its products are done and its stores have read it. Waits are bounded as in tc_linear.cu.
#include "tc_linear_common.cuh"

namespace flarepp {
namespace {

constexpr int kThreads = 896;
constexpr int kFirstDzWarp = 4, kGroups = 2, kGroupWarps = 8, kDzWarps = kGroups * kGroupWarps;
constexpr int kFirstEpiWarp = 20, kEpiWarps = 8;
constexpr int kDzTile = 128 * kSlice * 2;           // of dY (then dZ), of Z
constexpr uint32_t kS = 4, kStage = 2 * kDzTile;    // ring of dY and Z
// a group sees every phase of its stages, without which a wait by parity would name two phases
static_assert(kS % kGroups == 0, "a stage is always the same group's");
constexpr uint32_t kSW = 3, kStageW = kMaxNT / 2 * kSlice * 2;  // ring of the CTA's half of W's columns
constexpr int kStaging = kEpiWarps * kBlockBytes;
constexpr int kNumBars = 4 * kS + 2 * kSW + 4 + 1;
constexpr int kFixed = 1024 + kS * kStage + kSW * kStageW + kStaging + kNumBars * 8 + 16;

struct Fused {
    int T, K, NT;  // rows, columns of dX, the tile's columns
    int row_tiles, slices;
    uint32_t idesc;
    int store_dz;
    int N;
    float* db_part;  // [gridDim.x][ldz] or null
    int64_t ldz;
    Waits waits;
};

template <int ACT>
__global__ void __launch_bounds__(kThreads, 1)
    lin_fused_kernel(const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmZ,
                     const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmD,
                     const __grid_constant__ CUtensorMap tmX, const Fused prm) {
    extern __shared__ uint8_t smem_raw[];
    // the same offset in both CTAs of a pair: the dynamic shared memory starts at one address
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    const int db_width = prm.slices * kSlice;
    uint8_t* ring_w = smem + kS * kStage;
    uint8_t* staging = ring_w + kSW * kStageW;
    float* db_sums = reinterpret_cast<float*>(staging + kStaging);  // [kDzWarps][db_width]
    uint64_t* bars = reinterpret_cast<uint64_t*>(db_sums + kDzWarps * db_width);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t raw0 = smem_u32(bars);  // dY and Z of this CTA have landed
    const uint32_t full0 = raw0 + 8u * kS;    // leader: both CTAs' dZ is made
    const uint32_t empty0 = full0 + 8u * kS;  // products done, dZ stored
    const uint32_t wfull0 = empty0 + 8u * kS;   // leader: both halves of W's slice have landed
    const uint32_t wempty0 = wfull0 + 8u * kSW;
    const uint32_t accfull0 = wempty0 + 8u * kSW;
    const uint32_t accempty0 = accfull0 + 16u;
    const uint32_t fin = accempty0 + 16u;
    const uint32_t made0 = fin + 8u;  // this CTA's dZ is made (for its store)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int first = (int)blockIdx.x / 2, pairs = (int)gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < kS; ++s) {
            mbar_init(raw0 + 8u * s, 1);
            mbar_init(full0 + 8u * s, 2 * kGroupWarps);
            mbar_init(empty0 + 8u * s, 1 + (prm.store_dz ? 1 : kGroupWarps));
            mbar_init(made0 + 8u * s, kGroupWarps);
        }
        for (uint32_t s = 0; s < kSW; ++s) {
            mbar_init(wfull0 + 8u * s, 1);
            mbar_init(wempty0 + 8u * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(accfull0 + 8u * b, 1);
            mbar_init(accempty0 + 8u * b, kEpiWarps * 2);
        }
        mbar_init(fin, 1);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tmG);
        prefetch_tmap(&tmZ);
        prefetch_tmap(&tmW);
    }
    for (int i = threadIdx.x; i < kDzWarps * db_width; i += kThreads) db_sums[i] = 0.f;
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

    // The tiles go from the last rows to the first (dW, next, finds the rows that it starts with in the L2).
    if (warp == 0) {
        // ------------------------------------------------------------ TMA producer of dY and Z
        uint32_t it = 0;
        bool ok = true;
        for (int v = first; v < prm.row_tiles && ok; v += pairs) {
            const int m0 = ((prm.row_tiles - 1 - v) * 2 + (int)rank) * 128;
            for (int s = 0; s < prm.slices; ++s, ++it) {
                const uint32_t st = it % kS;
                if (it >= kS &&
                    !warp_wait<2>(empty0 + 8u * st, (it / kS - 1) & 1, abort_flag, prm.waits)) {
                    ok = false;
                    break;
                }
                if (elect_one() && !(blockIdx.x == 0 && it == prm.waits.withheld)) {
                    const uint32_t dst = smem_u32(smem + st * kStage);
                    const uint32_t raw = raw0 + 8u * st;
                    mbar_expect_tx(raw, 2 * kDzTile);
                    tma_load_2d(dst, &tmG, s * kSlice, m0, raw);
                    tma_load_2d(dst + kDzTile, &tmZ, s * kSlice, m0, raw);
                }
                __syncwarp();
            }
        }
        if (!ok) linger();  // its copies in flight
    } else if (warp == 2) {
        // ------------------------------------------------------------ TMA producer of W
        const int b_rows = prm.NT / 2;
        const uint32_t b_bytes = (uint32_t)((b_rows + 63) / 64 * 64) * kSlice * 2;
        uint32_t it = 0;
        bool ok = true;
        for (int v = first; v < prm.row_tiles && ok; v += pairs)
            for (int s = 0; s < prm.slices; ++s, ++it) {
                const uint32_t st = it % kSW;
                if (it >= kSW &&
                    !warp_wait<2>(wempty0 + 8u * st, (it / kSW - 1) & 1, abort_flag, prm.waits)) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    const uint32_t full = wfull0 + 8u * st;
                    if (rank == 0) mbar_expect_tx(full, 2 * b_bytes);
                    load_tile<2, true>(smem_u32(ring_w + st * kStageW), &tmW, (int)rank * b_rows,
                                       b_rows, s * kSlice, map_to_rank(full, 0));
                }
                __syncwarp();
            }
        if (!ok) linger();
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------ MMA issuer
        uint32_t it = 0, j = 0;
        bool ok = true;
        for (int v = first; v < prm.row_tiles && ok; v += pairs, ++j) {
            const uint32_t ab = j & 1;
            if (j >= 2 &&
                !warp_wait<2>(accempty0 + 8u * ab, ((j >> 1) - 1) & 1, abort_flag, prm.waits)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t acc = tmem + ab * kMaxNT;
            for (int s = 0; s < prm.slices; ++s, ++it) {
                const uint32_t st = it % kS, sw = it % kSW;
                if (!warp_wait<2>(wfull0 + 8u * sw, (it / kSW) & 1, abort_flag, prm.waits) ||
                    !warp_wait<2>(full0 + 8u * st, (it / kS) & 1, abort_flag, prm.waits)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t a = smem_u32(smem + st * kStage), b = smem_u32(ring_w + sw * kStageW);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < kSlice / 16; ++k)
                        mma_ss_pair(acc, tile_desc<false>(a, k), tile_desc<true>(b, k), prm.idesc,
                                    (s > 0 || k > 0) ? 1u : 0u);
                    mma_commit_pair(empty0 + 8u * st);
                    mma_commit_pair(wempty0 + 8u * sw);
                }
                __syncwarp();
            }
            if (!ok) break;
            if (elect_one()) mma_commit_pair(accfull0 + 8u * ab);
            __syncwarp();
        }
        if (elect_one()) mma_commit_pair(fin);
        __syncwarp();
        const uint64_t tw = globaltimer_ns();
        while (!__all_sync(0xffffffffu, mbar_try_wait(fin, 0)) &&
               globaltimer_ns() - tw < kWaitLimitNs) {
        }
    } else if (warp == 3 && prm.store_dz) {
        // ------------------------------------------------------------ dZ to memory
        uint32_t it = 0;
        bool ok = true;
        for (int v = first; v < prm.row_tiles && ok; v += pairs) {
            const int m0 = ((prm.row_tiles - 1 - v) * 2 + (int)rank) * 128;
            for (int s = 0; s < prm.slices; ++s, ++it) {
                const uint32_t st = it % kS;
                ok = warp_wait<1>(made0 + 8u * st, (it / kS) & 1, abort_flag, prm.waits);
                if (!ok) break;
                if (lane == 0) {
                    if (m0 < prm.T) {
                        tma_store_2d(&tmD, smem_u32(smem + st * kStage), s * kSlice, m0);
                        bulk_commit();
                        bulk_wait_read();
                    }
                    mbar_arrive(empty0 + 8u * st);
                }
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait_all();
    } else if (warp >= kFirstDzWarp && warp < kFirstEpiWarp) {
        // ------------------------------------------------------------ dZ
        // A lane takes 16-byte piece g (eight columns) of every fourth of its warp's rows.
        const int w = (warp - kFirstDzWarp) % kGroupWarps, g = lane & 7, r0 = 16 * w + (lane >> 3);
        const uint32_t group = (warp - kFirstDzWarp) / kGroupWarps;
        float* mine = db_sums + (warp - kFirstDzWarp) * db_width + g * 8;
        uint32_t it = 0;
        bool ok = true;
        for (int v = first; v < prm.row_tiles && ok; v += pairs) {
            for (int s = 0; s < prm.slices; ++s, ++it) {
                if (it % kGroups != group) continue;
                const uint32_t st = it % kS;
                ok = warp_wait<1>(raw0 + 8u * st, (it / kS) & 1, abort_flag, prm.waits);
                if (!ok) break;
                uint8_t* tile = smem + st * kStage;
                uint64_t sum[4] = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    uint4 d[2], z[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = r0 + 4 * (i + h), off = row * 128 + ((g ^ (row & 7)) << 4);
                        d[h] = *reinterpret_cast<const uint4*>(tile + off);
                        z[h] = *reinterpret_cast<const uint4*>(tile + kDzTile + off);
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t* dp = reinterpret_cast<uint32_t*>(&d[h]);
                        const uint32_t* zp = reinterpret_cast<const uint32_t*>(&z[h]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint64_t x =
                                mul2(unpack_bf16x2(dp[k]), act_slope2(ACT, unpack_bf16x2(zp[k])));
                            sum[k] = add2(sum[k], x);
                            dp[k] = pack_bf16x2(x);
                        }
                        const int row = r0 + 4 * (i + h), off = row * 128 + ((g ^ (row & 7)) << 4);
                        *reinterpret_cast<uint4*>(tile + off) = d[h];
                    }
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_cluster(map_to_rank(full0 + 8u * st, 0));
                    mbar_arrive((prm.store_dz ? made0 : empty0) + 8u * st);
                }
                if (prm.db_part) {  // over the lanes that share g, in a fixed order
                    float f[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 h = halves(sum[k]);
                        f[2 * k] = h.x;
                        f[2 * k + 1] = h.y;
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        f[k] += __shfl_xor_sync(0xffffffffu, f[k], 8);
                        f[k] += __shfl_xor_sync(0xffffffffu, f[k], 16);
                    }
                    if (lane < 8) {
                        float4* t = reinterpret_cast<float4*>(mine + s * kSlice);
                        float4 a = t[0], b = t[1];
                        t[0] = make_float4(a.x + f[0], a.y + f[1], a.z + f[2], a.w + f[3]);
                        t[1] = make_float4(b.x + f[4], b.y + f[5], b.z + f[6], b.w + f[7]);
                    }
                }
            }
        }
    } else if (warp >= kFirstEpiWarp) {
        // ------------------------------------------------------------ epilogue: dX
        const int e = warp - kFirstEpiWarp;
        const int q = warp % 4;  // the TMEM lanes this warp may read
        const int cfirst = 128 * (e / 4);
        uint8_t* staged = staging + e * kBlockBytes;
        uint32_t j = 0;
        for (int v = first; v < prm.row_tiles; v += pairs, ++j) {
            const uint32_t ab = j & 1;
            const int row0 = ((prm.row_tiles - 1 - v) * 2 + (int)rank) * 128 + 32 * q;
            const int cend = row0 < prm.T ? min(prm.K, cfirst + 128) : 0;
            const uint32_t acc = tmem + ((uint32_t)(32 * q) << 16) + ab * kMaxNT;
            if (!warp_wait<2>(accfull0 + 8u * ab, j >> 1 & 1, abort_flag, prm.waits)) break;
            tc_fence_after();
            for (int c = cfirst; c < cend; c += 32) {
                uint32_t r[32];
                tmem_ld32(acc + c, r);
                tmem_wait_ld32(r);
                if (lane == 0) bulk_wait_read();
                __syncwarp();
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t o[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        o[k] = pack_bf16x2(pair(__uint_as_float(r[8 * g + 2 * k]),
                                                __uint_as_float(r[8 * g + 2 * k + 1])));
                    // 16-byte pieces swizzled as the map of 64-byte lines expects them
                    *reinterpret_cast<uint4*>(staged + lane * 64 + ((g ^ (lane >> 1 & 3)) << 4)) =
                        make_uint4(o[0], o[1], o[2], o[3]);
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) {
                    tma_store_2d(&tmX, smem_u32(staged), c, row0);
                    bulk_commit();
                }
                __syncwarp();  // the next load from TMEM wants the whole warp
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_rank(accempty0 + 8u * ab, 0));
        }
        if (lane == 0) bulk_wait_all();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (prm.db_part)
        for (int c = threadIdx.x; c < prm.N; c += kThreads) {
            float f = db_sums[c];
#pragma unroll
            for (int w = 1; w < kDzWarps; ++w) f += db_sums[w * db_width + c];
            prm.db_part[(int64_t)blockIdx.x * prm.ldz + c] = f;
        }
    __syncwarp();  // the sums end at different columns of a warp
    cluster_sync();  // no CTA leaves while the other one may still signal it or read its shared memory
    tc_fence_after();
    if (warp == 1) tmem_dealloc_pair(tmem, kTmemCols);
}

size_t smem_for(int64_t out) {
    return (size_t)kFixed + kDzWarps * cdiv(out, kSlice) * kSlice * 4;
}

template <int ACT>
cudaError_t launch(const CUtensorMap* m, const Fused& p, int* ctas, cudaStream_t st) {
    auto kernel = lin_fused_kernel<ACT>;
    static std::atomic<int> fits[64];  // pairs that run at once on each device (0: not asked yet)
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem_for(p.N);
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
        static_assert(kFixed + kDzWarps * kFusedOut * 4 <= kMaxSmem, "shared memory budget");
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)smem_for(kFusedOut));
        if (e != cudaSuccess) return e;
        n = kNumSMs / 2;
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
    *ctas = (p.row_tiles < n ? p.row_tiles : n) * 2;
    cfg.gridDim = dim3((unsigned)*ctas);
    return cudaLaunchKernelEx(&cfg, kernel, m[0], m[1], m[2], m[3], m[4], p);
}

}  // namespace

cudaError_t take_fused_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

cudaError_t lin_fused(int64_t T, int64_t K, int64_t N, int act, const void* dY, const void* Z,
                      const LinOperand& w, void* dX, void* dZ, float* db_part, int64_t ldz,
                      int* ctas, int* status, cudaStream_t st) {
    Fused p{};
    p.T = (int)T;
    p.K = (int)K;
    p.N = (int)N;
    p.NT = (int)cdiv(K, 16) * 16;
    p.row_tiles = (int)cdiv(T, 256);
    p.slices = (int)cdiv(N, kSlice);
    p.idesc = idesc_bf16_f32(256, p.NT, false, true);
    p.store_dz = dZ != nullptr;
    p.db_part = db_part;
    p.ldz = ldz;
    p.waits.status = status;
    test_fault_for(kFusedKernel, &p.waits.limit_ns, &p.waits.withheld);
    CUtensorMap m[5];
    bool ok = make_map(&m[0], dY, N, T, N, kSlice, 128) && make_map(&m[1], Z, N, T, N, kSlice, 128) &&
              make_map(&m[2], w.t, K, N, w.pitch, 64, kSlice) && make_map(&m[4], dX, K, T, K, 32, 32);
    m[3] = m[0];  // unused without dZ
    if (dZ) ok = ok && make_map(&m[3], dZ, N, T, ldz, kSlice, 128);
    if (!ok) return cudaErrorInvalidValue;
    switch (act) {
        case FLAREPP_ACT_RELU: return launch<FLAREPP_ACT_RELU>(m, p, ctas, st);
        case FLAREPP_ACT_GELU: return launch<FLAREPP_ACT_GELU>(m, p, ctas, st);
        case FLAREPP_ACT_SILU: return launch<FLAREPP_ACT_SILU>(m, p, ctas, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace flarepp
