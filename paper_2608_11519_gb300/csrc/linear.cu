// The linear layer (flarepp_linear_*): argument checks, workspace layout, the launch sequence of
// its products (tc_linear.cu), and the memory-bound kernels around them.
//
// A kernel overlaps the one before it up to pdl_wait, and its inputs may come from there. They are
// therefore not __restrict__: loads of memory promised to stay constant may move above that wait.
#include <cuda_runtime.h>
#include <math.h>

#include "checks.h"
#include "linear_internal.h"
#include "tc_ptx.cuh"

namespace flarepp {
namespace {

constexpr int kDzThreads = 256;  // also of the blocks that copy lines

// Up to four rows the layer can run on the CUDA cores (gemv_kernel): a weight then meets so few
// multiplications that its bytes are the bound, and one launch without tensor maps is the shortest
// path. That ends where rows x weights pass about 12 M (with weights from memory, in a graph): 2 rows of
// 4096 -> 1001 take 4.6 us here and 6.0 in lin_few, 4 rows 7.8 and 6.1; 2 rows of 4096 -> 4096, beyond it, 9.5
// and 10.1. One row is always faster here (4096 -> 4096: 8.2 and 10.1).
constexpr int64_t kGemvRows = 4;
bool use_gemv(int64_t T, int64_t K, int64_t N) {
    return K % 8 == 0 && (T == 1 || (T <= kGemvRows && T * K * N <= 12000000));
}
// Rows up to which lin_few is faster than tiles of 256 rows: 200 rows of 4096 -> 4096 take 14.4 us in
// lin_few and 19.5 in tiles, 200 rows of 256 -> 512 8.7 and 6.5 (a short contraction leaves lin_few's CTAs
// mostly with their epilogues).
bool use_few(int64_t T, int64_t depth) { return T <= (depth >= 1024 ? kFewRows : kFewRows / 2); }
constexpr int kGemvWarps = 8;

constexpr int64_t kPadWRows = 4096;

// The pitch of lines that the layer lays out itself: whole 128-byte lines, so that a 128-byte row of
// a TMA box is one line and not parts of two.
int64_t pitch_of(int64_t n) { return cdiv(n, 64) * 64; }
// What TMA cannot address is laid out anew; so is W where its lines are not whole 128-byte lines and
// 16 or more row tiles read it (20,011 rows of 1000 -> 1544: 65 us as it lies, 60 with the copy; the
// lines of X, read as often as written, are not worth one).
bool pad_x(int64_t K) { return K % 8 != 0; }
bool pad_w(int64_t K, int64_t T) { return K % 8 != 0 || (K % 64 != 0 && T >= kPadWRows); }

// The layer for T <= RT rows, `in` a multiple of 8. A warp takes RW rows of W at a time, a lane every
// 32nd vector of eight weights of each, U of them in flight (RW * U = 8 loads of 16 bytes a lane
// keep the memory busy from a thousand warps); `split` warps share a row where there are few rows of
// W, and their sums are added in order.
template <int RT, int RW>
__global__ void __launch_bounds__(kGemvWarps * 32)
    gemv_kernel(const __nv_bfloat16* X, const __nv_bfloat16* W, int T,
                int K, int N, int split, int act, const __nv_bfloat16* bias,
                const __nv_bfloat16* R, __nv_bfloat16* __restrict__ Y,
                __nv_bfloat16* __restrict__ Z) {
    constexpr int U = 8 / RW;
    __shared__ float sums[kGemvWarps][RW][RT];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int share = warp % split;
    const int n0 = (blockIdx.x * (kGemvWarps / split) + warp / split) * RW;
    const int vecs = K / 8, per = (vecs + split - 1) / split;
    const int v1 = min(vecs, (share + 1) * per);
    uint64_t acc[RW][RT];
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[r][t] = 0;
    for (int v = share * per + lane; v < v1; v += 32 * U) {
        uint4 w[U][RW];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int r = 0; r < RW; ++r)
                w[u][r] = v + 32 * u < v1 && n0 + r < N
                              ? reinterpret_cast<const uint4*>(W + (int64_t)(n0 + r) * K)[v + 32 * u]
                              : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (v + 32 * u >= v1) break;
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (t >= T) break;
                const uint4 x = reinterpret_cast<const uint4*>(X + (int64_t)t * K)[v + 32 * u];
                const uint64_t x0 = unpack_bf16x2(x.x), x1 = unpack_bf16x2(x.y);
                const uint64_t x2 = unpack_bf16x2(x.z), x3 = unpack_bf16x2(x.w);
#pragma unroll
                for (int r = 0; r < RW; ++r) {
                    acc[r][t] = fma2(x0, unpack_bf16x2(w[u][r].x), acc[r][t]);
                    acc[r][t] = fma2(x1, unpack_bf16x2(w[u][r].y), acc[r][t]);
                    acc[r][t] = fma2(x2, unpack_bf16x2(w[u][r].z), acc[r][t]);
                    acc[r][t] = fma2(x3, unpack_bf16x2(w[u][r].w), acc[r][t]);
                }
            }
        }
    }
    float mine = 0.f;  // the sum of output (r, t) in lane r * RT + t
#pragma unroll
    for (int r = 0; r < RW; ++r)
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            const float2 f = halves(acc[r][t]);
            float s = f.x + f.y;
#pragma unroll
            for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (lane == r * RT + t) mine = s;
        }
    const int r = lane / RT, t = lane % RT, n = n0 + r;
    if (split > 1) {
        if (lane < RW * RT) sums[warp][r][t] = mine;
        __syncthreads();
        if (share) return;
        if (lane < RW * RT)
            for (int k = 1; k < split; ++k) mine += sums[warp + k][r][t];
    }
    if (lane >= RW * RT || t >= T || n >= N) return;
    if (bias) mine += __bfloat162float(bias[n]);
    const int64_t at = (int64_t)t * N + n;
    if (Z) Z[at] = __float2bfloat16_rn(mine);
    float y = halves(act_value2(act, pair(mine, mine))).x;
    if (R) y += __bfloat162float(R[at]);
    Y[at] = __float2bfloat16_rn(y);
}

template <int BYTES>
struct Bytes;
template <>
struct Bytes<2> { using T = uint16_t; };
template <>
struct Bytes<4> { using T = uint32_t; };
template <>
struct Bytes<8> { using T = uint2; };
template <>
struct Bytes<16> { using T = uint4; };

// dst [rows][pitch] = src [rows][cols] with zeros behind each row: the 16-byte line pitch that
// TMA asks for. One thread per eight values, read in words of VW, which `cols` is a multiple of.
struct Pad {
    const __nv_bfloat16* src;
    int64_t rows, cols, pitch;
    __nv_bfloat16* dst;
    unsigned blocks;  // of 256 threads; 0: nothing to do
};
template <int VW>
__device__ void pad_rows(const Pad& p, unsigned block) {
    using Piece = typename Bytes<2 * VW>::T;
    const int64_t per = p.pitch / 8, n = p.rows * per;
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < n; i += (int64_t)p.blocks * 256) {
        const int64_t r = i / per, c = (i - r * per) * 8;
        __align__(16) __nv_bfloat16 v[8];
#pragma unroll
        for (int k = 0; k < 8; k += VW)
            *reinterpret_cast<Piece*>(v + k) =
                c + k < p.cols ? *reinterpret_cast<const Piece*>(p.src + r * p.cols + c + k) : Piece{};
        *reinterpret_cast<uint4*>(p.dst + r * p.pitch + c) = *reinterpret_cast<const uint4*>(v);
    }
}
// Blocks a.blocks + b.blocks: the first ones' share of a, the others' of b.
__device__ void pad_both(const Pad& a, const Pad& b, unsigned block) {
    const Pad& p = block < a.blocks ? a : b;
    if (block >= a.blocks) block -= a.blocks;
    if (p.cols % 8 == 0) pad_rows<8>(p, block);
    else if (p.cols % 4 == 0) pad_rows<4>(p, block);
    else if (p.cols % 2 == 0) pad_rows<2>(p, block);
    else pad_rows<1>(p, block);
}
__global__ void __launch_bounds__(256) pad_kernel(const Pad a, const Pad b) {
    tc::pdl_trigger();
    tc::pdl_wait();
    pad_both(a, b, blockIdx.x);
}

// The column sums of dZ: what dz_kernel's blocks left in part[n_part][ldz], for db.
struct DbSums {
    const float* part;
    int n_part;
    int64_t cols, ldz;
    __nv_bfloat16* db;
};

// db of 32 columns: YS threads a column, each over a stretch of the partial sums in order, the
// stretches added in order.
template <int YS>
__device__ void sum_db(const DbSums& d, int64_t group) {
    __shared__ float sums[YS][33];
    const int lane = threadIdx.x % 32, ty = threadIdx.x / 32;
    const int64_t c = group * 32 + lane;
    const int per = (d.n_part + YS - 1) / YS;
    float s = 0.f;
    if (c < d.cols)
#pragma unroll 16
        for (int k = ty * per; k < min(d.n_part, (ty + 1) * per); ++k) s += d.part[k * d.ldz + c];
    sums[ty][lane] = s;
    __syncthreads();
    if (ty == 0 && c < d.cols) {
#pragma unroll
        for (int k = 1; k < YS; ++k) s += sums[k][lane];
        d.db[c] = __float2bfloat16_rn(s);
    }
}
constexpr int kDbThreads = 1024;
__global__ void __launch_bounds__(kDbThreads) db_kernel(const DbSums d) {
    tc::pdl_trigger();
    tc::pdl_wait();
    sum_db<kDbThreads / 32>(d, blockIdx.x);
}

// What follows the float32 sums of a cut contraction: the chunks added in order (with SPLIT > 1 as
// SPLIT stretches of chunks, the stretches in order after that: many chunks would otherwise be one
// long chain of loads), then the epilogue (bias, activation, residual). SPLIT threads per four
// columns. The blocks from `blocks` on sum db instead, which then needs no launch of its own.
constexpr int kFinishThreads = 256;
template <int SPLIT>
__global__ void __launch_bounds__(kFinishThreads)
    finish_kernel(const float* part, int chunks, int64_t rows,
                              int64_t cols, int64_t ldp, int act,
                              const __nv_bfloat16* bias,
                              const __nv_bfloat16* R, __nv_bfloat16* __restrict__ Y,
                              __nv_bfloat16* __restrict__ Z, unsigned blocks, const DbSums db) {
    tc::pdl_trigger();
    tc::pdl_wait();
    if (blockIdx.x >= blocks) {
        sum_db<kFinishThreads / 32>(db, blockIdx.x - blocks);
        return;
    }
    constexpr int kQuads = kFinishThreads / SPLIT;
    const int64_t per = ldp / 4;
    const int quad = threadIdx.x % kQuads, part_of = threadIdx.x / kQuads;
    const int64_t i = (int64_t)blockIdx.x * kQuads + quad;
    const bool in = i < rows * per;
    const int64_t r = in ? i / per : 0, c = in ? (i - r * per) * 4 : 0;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    const int stretch = (chunks + SPLIT - 1) / SPLIT;
    const int k1 = min(chunks, (part_of + 1) * stretch);
    const float* p = part + ((int64_t)part_of * stretch * rows + r) * ldp + c;
    if (in)
#pragma unroll 8
        for (int k = part_of * stretch; k < k1; ++k, p += rows * ldp) {
            const float4 v = *reinterpret_cast<const float4*>(p);
            x[0] += v.x;
            x[1] += v.y;
            x[2] += v.z;
            x[3] += v.w;
        }
    if (SPLIT > 1) {
        __shared__ float4 sums[SPLIT][kQuads];
        sums[part_of][quad] = make_float4(x[0], x[1], x[2], x[3]);
        __syncthreads();
        if (part_of > 0) return;
#pragma unroll
        for (int k = 1; k < SPLIT; ++k) {
            const float4 v = sums[k][quad];
            x[0] += v.x;
            x[1] += v.y;
            x[2] += v.z;
            x[3] += v.w;
        }
    }
    if (!in) return;
    const int64_t at = r * cols + c;
    if (bias)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] += c + k < cols ? __bfloat162float(bias[c + k]) : 0.f;
    if (Z)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c + k < cols) Z[at + k] = __float2bfloat16_rn(x[k]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float2 y = halves(act_value2(act, pair(x[2 * h], x[2 * h + 1])));
        x[2 * h] = y.x;
        x[2 * h + 1] = y.y;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (c + k >= cols) break;
        if (R) x[k] += __bfloat162float(R[at + k]);
        Y[at + k] = __float2bfloat16_rn(x[k]);
    }
}

// dZ = dY o act'(Z) into lines of `ldz` values (not written when dZ is null), and the column sums
// of the unrounded dZ over the block's rows into db_part[blockIdx.y][ldz]. `lanes` threads (a power of
// two up to 32) take eight columns each of a row, and the block as many rows at once as it has room for.
// The blocks from gx * gy on copy a and b instead, which then need no launch of their own.
// VW: values that a load takes, which `cols` is a multiple of (30,000 x 900: 37 us with single values).
template <int VW>
__global__ void __launch_bounds__(kDzThreads, 4)
    dz_kernel(const __nv_bfloat16* dY, const __nv_bfloat16* Z,
              int64_t rows, int64_t cols, int64_t rows_per, int lanes, int act, int64_t ldz,
              __nv_bfloat16* __restrict__ dZ, float* __restrict__ db_part, unsigned gx, unsigned gy,
              const Pad a, const Pad b) {
    tc::pdl_trigger();
    tc::pdl_wait();
    if (blockIdx.x >= gx * gy) {
        pad_both(a, b, blockIdx.x - gx * gy);
        return;
    }
    const unsigned bx = blockIdx.x % gx, by = blockIdx.x / gx;
    __shared__ float sums[kDzThreads * 8];  // [rows at once][lanes * 8]
    const int lane = threadIdx.x % lanes, ty = threadIdx.x / lanes, at_once = kDzThreads / lanes;
    const int64_t c = ((int64_t)bx * lanes + lane) * 8;
    const int64_t r1 = min(rows, (int64_t)(by + 1) * rows_per);
    uint64_t sum[4] = {0, 0, 0, 0};  // pairs
    if (c < cols) {
#pragma unroll 2
        for (int64_t r = (int64_t)by * rows_per + ty; r < r1; r += at_once) {
            __align__(16) __nv_bfloat16 g[8], z[8];
            const int64_t at = r * cols + c;
            using Piece = typename Bytes<2 * VW>::T;
#pragma unroll
            for (int k = 0; k < 8; k += VW) {
                const bool in = VW == 8 || c + k < cols;
                auto load = [&](const __nv_bfloat16* p) {
                    return in ? *reinterpret_cast<const Piece*>(p + at + k) : Piece{};
                };
                *reinterpret_cast<Piece*>(g + k) = load(dY);
                if (Z) *reinterpret_cast<Piece*>(z + k) = load(Z);
            }
            uint32_t* gp = reinterpret_cast<uint32_t*>(g);
            const uint32_t* zp = reinterpret_cast<const uint32_t*>(z);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint64_t v = unpack_bf16x2(gp[k]);
                if (Z) v = mul2(v, act_slope2(act, unpack_bf16x2(zp[k])));
                sum[k] = add2(sum[k], v);
                gp[k] = pack_bf16x2(v);
            }
            if (dZ) *reinterpret_cast<uint4*>(dZ + r * ldz + c) = *reinterpret_cast<uint4*>(g);
        }
    }
    if (!db_part) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        *reinterpret_cast<float2*>(&sums[threadIdx.x * 8 + 2 * k]) = halves(sum[k]);
    __syncthreads();
    const int width = lanes * 8;
    const int64_t col = (int64_t)bx * width + threadIdx.x;
    if ((int)threadIdx.x < width && col < cols) {
        float s = 0.f;
#pragma unroll 8
        for (int k = 0; k < at_once; ++k) s += sums[k * width + threadIdx.x];
        db_part[(int64_t)by * ldz + col] = s;
    }
}

// ------------------------------------------------------------------ host side

struct Shape {
    int64_t T, K, N;
    int act;
};

flarepp_status check_shape(const flarepp_linear_shape* s, Shape* o) {
    if (!s || s->rows < 0 || s->in < 1 || s->out < 1) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->dtype != FLAREPP_F32 && s->dtype != FLAREPP_BF16) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->act < FLAREPP_ACT_NONE || s->act > FLAREPP_ACT_SILU) return FLAREPP_ERR_INVALID_ARGUMENT;
    // the rows of the last tile of 256 have 32-bit numbers
    if (s->dtype != FLAREPP_BF16 || s->rows > 0x7fffff00 || s->in > (1 << 20) || s->out > (1 << 20))
        return FLAREPP_ERR_UNSUPPORTED;
    *o = {s->rows, s->in, s->out, s->act};
    return FLAREPP_OK;
}

size_t take(size_t* off, int64_t bytes) {
    const size_t at = *off;
    *off = align_up(at + (size_t)bytes, kWsAlign);
    return at;
}

size_t part_bytes(const LinPlan& p, int64_t rows, int64_t cols) {
    return (size_t)p.chunks * (size_t)rows * (size_t)(cdiv(cols, 4) * 4) * 4;
}

struct FwdLayout {
    bool gemv, few;
    LinPlan plan;
    bool split;  // the sums go through partials and finish_kernel
    size_t off_x, off_w, off_part, total;
};
FwdLayout fwd_layout(const Shape& s) {
    FwdLayout L{};
    L.gemv = use_gemv(s.T, s.K, s.N);
    if (L.gemv) return L;
    L.few = use_few(s.T, s.K);
    if (!L.few) L.plan = lin_plan(s.T, s.N, s.K);
    L.split = L.plan.chunks > 1;
    L.off_x = take(&L.total, pad_x(s.K) ? s.T * pitch_of(s.K) * 2 : 0);
    L.off_w = take(&L.total, pad_w(s.K, s.T) ? s.N * pitch_of(s.K) * 2 : 0);
    L.off_part = take(&L.total, L.split ? (int64_t)part_bytes(L.plan, s.T, s.N) : 0);
    return L;
}

// Whether one kernel makes dZ on its way to dX (lin_fused): with rows for every pair of CTAs, and outputs
// that fill its slices of 64.
bool use_fused(const Shape& s) {
    return s.act != FLAREPP_ACT_NONE && s.K % 8 == 0 && s.K <= kFusedIn && s.N % 8 == 0 &&
           s.N >= 64 && s.N <= kFusedOut && s.T >= 64 * kNumSMs;
}

struct BwdLayout {
    bool few, fused;
    LinPlan plan_x, plan_w;
    bool split_x, split_w;
    bool own_dz;  // dZ is laid out in the workspace (else the products read dY)
    int dz_lanes;
    int64_t dz_blocks, dz_rows;
    size_t off_x, off_w, off_dz, off_db, off_px, off_pw, total;
};
BwdLayout bwd_layout(const Shape& s) {
    BwdLayout L{};
    L.few = use_few(s.T, s.N);
    L.fused = use_fused(s);
    if (!L.few) L.plan_x = lin_plan(s.T, s.K, s.N);
    L.plan_w = lin_plan(s.N, s.K, s.T);
    L.split_x = L.plan_x.chunks > 1;
    L.split_w = L.plan_w.chunks > 1;
    L.own_dz = s.act != FLAREPP_ACT_NONE || s.N % 8 != 0;
    // one wave of dz_kernel's blocks, four per SM, each of at least four rounds of rows
    L.dz_lanes = 1;
    while (L.dz_lanes < 32 && L.dz_lanes * 8 < s.N) L.dz_lanes *= 2;
    const int64_t at_once = kDzThreads / L.dz_lanes;
    int64_t want = 4 * kNumSMs / cdiv(s.N, L.dz_lanes * 8);
    if (want > cdiv(s.T, 4 * at_once)) want = cdiv(s.T, 4 * at_once);
    if (want < 1) want = 1;
    L.dz_rows = cdiv(cdiv(s.T, want), at_once) * at_once;
    L.dz_blocks = cdiv(s.T, L.dz_rows);
    L.off_x = take(&L.total, pad_x(s.K) ? s.T * pitch_of(s.K) * 2 : 0);
    L.off_w = take(&L.total, pad_w(s.K, s.T) ? s.N * pitch_of(s.K) * 2 : 0);
    L.off_dz = take(&L.total, L.own_dz ? s.T * pitch_of(s.N) * 2 : 0);
    L.off_db = take(&L.total, (L.dz_blocks > kNumSMs ? L.dz_blocks : kNumSMs) * pitch_of(s.N) * 4);
    L.off_px = take(&L.total, L.split_x ? (int64_t)part_bytes(L.plan_x, s.T, s.K) : 0);
    L.off_pw = take(&L.total, L.split_w ? (int64_t)part_bytes(L.plan_w, s.N, s.K) : 0);
    return L;
}

Pad pad(const void* src, int64_t rows, int64_t cols, void* dst) {
    const int64_t blocks = cdiv(rows * pitch_of(cols) / 8, 256);
    return {(const __nv_bfloat16*)src, rows, cols, pitch_of(cols), (__nv_bfloat16*)dst,
            (unsigned)(blocks < 32 * kNumSMs ? blocks : 32 * kNumSMs)};
}
cudaError_t pads(const Pad& a, const Pad& b, cudaStream_t st) {
    if (a.blocks + b.blocks == 0) return cudaSuccess;
    return launch_pdl(pad_kernel, dim3(a.blocks + b.blocks), dim3(256), 0, st, a, b);
}

cudaError_t finish(const float* part, const LinPlan& plan, int64_t rows, int64_t cols,
                   const LinEpilogue& e, const DbSums& db, cudaStream_t st) {
    const int64_t ldp = cdiv(cols, 4) * 4, n = rows * (ldp / 4);
    // over 16 chunks: eight threads share them (38 chunks of 512 x 256 sums: 14 us with one)
    const int split = plan.chunks > 16 ? 8 : 1;
    auto kernel = split == 8 ? finish_kernel<8> : finish_kernel<1>;
    const unsigned blocks = (unsigned)cdiv(n * split, kFinishThreads);
    const unsigned more = db.db ? (unsigned)cdiv(db.cols, 32) : 0;
    return launch_pdl(kernel, dim3(blocks + more), dim3(kFinishThreads), 0, st, part, plan.chunks,
                      rows, cols, ldp, e.act, (const __nv_bfloat16*)e.bias,
                      (const __nv_bfloat16*)e.R, (__nv_bfloat16*)e.Y, (__nv_bfloat16*)e.Z, blocks,
                      db);
}

// out [rows][cols] = epilogue(sum_k a(row, k) b(col, k)), through partials where the plan cuts
// the contraction
cudaError_t product(const LinPlan& plan, bool split, int64_t rows, int64_t cols, int64_t depth,
                    const LinOperand& a, const LinOperand& b, const LinEpilogue& e, float* part,
                    int* status, cudaStream_t st, const DbSums& db = DbSums{}) {
    if (!split) return lin_gemm(plan, rows, cols, depth, a, b, e, status, st);
    LinEpilogue sums{};
    sums.part = part;
    sums.ldp = cdiv(cols, 4) * 4;
    const cudaError_t err = lin_gemm(plan, rows, cols, depth, a, b, sums, status, st);
    return err != cudaSuccess ? err : finish(part, plan, rows, cols, e, db, st);
}

template <int RT>
cudaError_t gemv(const Shape& s, const void* X, const void* W, const LinEpilogue& e,
                 cudaStream_t st) {
    // four rows of W at once where a row alone is less than half of a warp's loads in flight
    const int rw = s.K <= 1024 ? 4 : 1;
    int split = 1;  // at least eight warps per SM, and half a kilobyte of a row for each
    while (split < kGemvWarps && cdiv(s.N, rw) * split < 8 * kNumSMs && s.K / split > 512) split *= 2;
    const unsigned blocks = (unsigned)cdiv(cdiv(s.N, rw), kGemvWarps / split);
    auto kernel = rw == 4 ? gemv_kernel<RT, 4> : gemv_kernel<RT, 1>;
    using B = __nv_bfloat16;
    return launch_pdl(kernel, dim3(blocks), dim3(kGemvWarps * 32), 0, st, (const B*)X, (const B*)W,
                      (int)s.T, (int)s.K, (int)s.N, split, e.act, (const B*)e.bias,
                      (const B*)e.R, (B*)e.Y, (B*)e.Z);
}

flarepp_status linear_fwd(const flarepp_linear_shape* shape, const void* X, const void* W,
                          const void* b, const void* R, void* Y, void* Z, void* workspace,
                          size_t workspace_bytes, int32_t* status, cudaStream_t st) {
    Shape s;
    const flarepp_status bad = check_shape(shape, &s);
    if (bad != FLAREPP_OK) return bad;
    if (s.T == 0) return FLAREPP_OK;
    const void* all[6] = {X, W, Y, b, R, Z};
    for (int i = 0; i < 6; ++i)
        if ((i < 3 && !all[i]) || !aligned16(all[i])) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!aligned4(status)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const size_t y_bytes = (size_t)s.T * s.N * 2;
    const FwdLayout L = fwd_layout(s);
    if (L.total && (!workspace || (uintptr_t)workspace % kWsAlign || workspace_bytes < L.total))
        return FLAREPP_ERR_WORKSPACE;
    const Span outs[4] = {{Y, y_bytes}, {Z, y_bytes}, {workspace, L.total}, {status, 4}};
    const Span ins[4] = {{X, (size_t)s.T * s.K * 2}, {W, (size_t)s.N * s.K * 2},
                         {b, (size_t)s.N * 2}, {R, y_bytes}};
    if (!disjoint(outs, 4, ins, 4)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const LinEpilogue e{s.act, b, R, Y, Z, nullptr, 0, 0};
    if (L.gemv) {
        const cudaError_t err = s.T == 1   ? gemv<1>(s, X, W, e, st)
                                : s.T == 2 ? gemv<2>(s, X, W, e, st)
                                           : gemv<4>(s, X, W, e, st);
        return err == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
    }
    char* ws = (char*)workspace;
    LinOperand x{X, s.K, 0}, w{W, s.K, 0};
    Pad px{}, pw{};
    if (pad_x(s.K)) {
        px = pad(X, s.T, s.K, ws + L.off_x);
        x = {px.dst, px.pitch, 0};
    }
    if (pad_w(s.K, s.T)) {
        pw = pad(W, s.N, s.K, ws + L.off_w);
        w = {pw.dst, pw.pitch, 0};
    }
    if (pads(px, pw, st) != cudaSuccess) return FLAREPP_ERR_CUDA;
    const cudaError_t err = L.few ? lin_few(s.T, s.N, s.K, x, w, e, status, st)
                                  : product(L.plan, L.split, s.T, s.N, s.K, x, w, e,
                                            (float*)(ws + L.off_part), status, st);
    return err == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

flarepp_status linear_bwd(const flarepp_linear_shape* shape, const void* X, const void* W,
                          const void* Z, const void* dY, void* dX, void* dW, void* db,
                          void* workspace, size_t workspace_bytes, int32_t* status,
                          cudaStream_t st) {
    Shape s;
    const flarepp_status bad = check_shape(shape, &s);
    if (bad != FLAREPP_OK) return bad;
    if (s.act == FLAREPP_ACT_NONE) Z = nullptr;
    if (!dW) X = nullptr;
    if (!dX) W = nullptr;
    const void* all[7] = {X, W, Z, dY, dX, dW, db};
    for (const void* p : all)
        if (!aligned16(p)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!aligned4(status)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const size_t w_bytes = (size_t)s.N * s.K * 2, b_bytes = (size_t)s.N * 2;
    const size_t x_bytes = (size_t)s.T * s.K * 2, y_bytes = (size_t)s.T * s.N * 2;
    const BwdLayout L = s.T ? bwd_layout(s) : BwdLayout{};
    if (s.T) {
        if (!dY || (dW && !X) || (dX && !W) || (s.act != FLAREPP_ACT_NONE && !Z))
            return FLAREPP_ERR_INVALID_ARGUMENT;
        if (!workspace || (uintptr_t)workspace % kWsAlign || workspace_bytes < L.total)
            return FLAREPP_ERR_WORKSPACE;
    }
    const Span outs[5] = {{dX, x_bytes}, {dW, w_bytes}, {db, b_bytes}, {workspace, L.total}, {status, 4}};
    const Span ins[4] = {{X, x_bytes}, {W, w_bytes}, {Z, y_bytes}, {dY, y_bytes}};
    if (!disjoint(outs, 5, ins, 4)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s.T == 0) {
        if ((dW && cudaMemsetAsync(dW, 0, w_bytes, st) != cudaSuccess) ||
            (db && cudaMemsetAsync(db, 0, b_bytes, st) != cudaSuccess))
            return FLAREPP_ERR_CUDA;
        return FLAREPP_OK;
    }
    char* ws = (char*)workspace;
    const int64_t ldz = pitch_of(s.N);
    const bool own_dz = L.own_dz && (dX || dW);
    cudaError_t e = cudaSuccess;
    const bool fused = L.fused && dX;
    LinOperand x{X, s.K, 0}, w{W, s.K, 0};
    Pad px{}, pw{};
    if (pad_x(s.K)) {
        if (dW) px = pad(X, s.T, s.K, ws + L.off_x);
        x = {ws + L.off_x, pitch_of(s.K), 0};
    }
    if (pad_w(s.K, s.T)) {
        if (dX) pw = pad(W, s.N, s.K, ws + L.off_w);
        w = {ws + L.off_w, pitch_of(s.K), 0};
    }
    if (!fused && (own_dz || db)) {
        const unsigned gx = (unsigned)cdiv(s.N, L.dz_lanes * 8), gy = (unsigned)L.dz_blocks;
        auto kernel = s.N % 2 ? dz_kernel<1> : s.N % 4 ? dz_kernel<2> : s.N % 8 ? dz_kernel<4> : dz_kernel<8>;
        e = launch_pdl(kernel, dim3(gx * gy + px.blocks + pw.blocks), dim3(kDzThreads), 0, st,
                       (const __nv_bfloat16*)dY, (const __nv_bfloat16*)Z, s.T, s.N, L.dz_rows, L.dz_lanes,
                       s.act, ldz, (__nv_bfloat16*)(own_dz ? ws + L.off_dz : nullptr),
                       (float*)(db ? ws + L.off_db : nullptr), gx, gy, px, pw);
    } else {
        e = pads(px, pw, st);
    }
    int db_parts = (int)L.dz_blocks;
    if (e == cudaSuccess && fused)
        e = lin_fused(s.T, s.K, s.N, s.act, dY, Z, {w.t, w.pitch, 1}, dX,
                      dW ? ws + L.off_dz : nullptr, (float*)(db ? ws + L.off_db : nullptr), ldz,
                      &db_parts, status, st);
    DbSums sums{(const float*)(ws + L.off_db), db_parts, s.N, ldz, (__nv_bfloat16*)db};
    if (e == cudaSuccess && db && !(dW && L.split_w)) {
        e = launch_pdl(db_kernel, dim3((unsigned)cdiv(s.N, 32)), dim3(kDbThreads), 0, st, sums);
        sums.db = nullptr;
    }
    const LinOperand dz{own_dz ? ws + L.off_dz : dY, own_dz ? ldz : s.N, 0};
    // dX takes the rows from the last to the first and dW from the first on: each then finds in the L2
    // what was written or read last
    if (e == cudaSuccess && dX && !fused) {
        const LinEpilogue to_dx{FLAREPP_ACT_NONE, nullptr, nullptr, dX, nullptr, nullptr, 0, 1};
        const LinOperand wt{w.t, w.pitch, 1};
        e = L.few ? lin_few(s.T, s.K, s.N, dz, wt, to_dx, status, st)
                  : product(L.plan_x, L.split_x, s.T, s.K, s.N, dz, wt, to_dx,
                            (float*)(ws + L.off_px), status, st);
    }
    if (e == cudaSuccess && dW)
        e = product(L.plan_w, L.split_w, s.N, s.K, s.T, {dz.t, dz.pitch, 1}, {x.t, x.pitch, 1},
                    {FLAREPP_ACT_NONE, nullptr, nullptr, dW, nullptr, nullptr, 0, 0},
                    (float*)(ws + L.off_pw), status, st, sums);
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

}  // namespace
}  // namespace flarepp

extern "C" {

size_t flarepp_linear_workspace_bytes(const flarepp_linear_shape* shape) {
    flarepp::Shape s;
    if (flarepp::check_shape(shape, &s) != FLAREPP_OK || s.T == 0) return 0;
    return flarepp::fwd_layout(s).total;
}

flarepp_status flarepp_linear_fwd(const flarepp_linear_shape* shape, const void* X, const void* W,
                                  const void* b, const void* R, void* Y, void* Z,
                                  void* workspace, size_t workspace_bytes, int32_t* status,
                                  void* stream) {
    return flarepp::linear_fwd(shape, X, W, b, R, Y, Z, workspace, workspace_bytes, status,
                               (cudaStream_t)stream);
}

size_t flarepp_linear_bwd_workspace_bytes(const flarepp_linear_shape* shape) {
    flarepp::Shape s;
    if (flarepp::check_shape(shape, &s) != FLAREPP_OK || s.T == 0) return 0;
    return flarepp::bwd_layout(s).total;
}

flarepp_status flarepp_linear_bwd(const flarepp_linear_shape* shape, const void* X, const void* W,
                                  const void* Z, const void* dY, void* dX, void* dW, void* db,
                                  void* workspace, size_t workspace_bytes, int32_t* status,
                                  void* stream) {
    return flarepp::linear_bwd(shape, X, W, Z, dY, dX, dW, db, workspace, workspace_bytes, status,
                               (cudaStream_t)stream);
}

}  // extern "C"
