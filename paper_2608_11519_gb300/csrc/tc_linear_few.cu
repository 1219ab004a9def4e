// The linear layer's product for few rows of tokens (tcgen05 / TMEM / TMA, clusters).
// The layer for up to 256 rows of tokens: the weights are the tile's rows (128 of them, whatever the
// number of tokens) and the tokens its columns, so the tensor cores' 128 rows are never idle and the
// weights, whose bytes are the bound, are read once. A cluster of up to eight CTAs shares a tile, each
// with every S-th slice of the contraction, so that a few tiles still draw on many SMs; the CTAs
// leave their float32 sums in shared memory, and each adds a share of the columns over the cluster in
// rank order and runs the epilogue on it. One launch, no workspace: 48 rows of 4096 -> 1001 take 5.9 us
// (8.8 as chunk sums in memory and a second kernel), of which the 8.7 MB are 1.3; the rest is the launch,
// the first loads' latency and the exchange.
#include "tc_linear_common.cuh"

namespace flarepp {
namespace {

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

cudaError_t take_few_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

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

}  // namespace flarepp
