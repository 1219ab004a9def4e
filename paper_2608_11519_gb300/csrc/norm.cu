// Group norm with an activation, channels last (flarepp_group_norm_*): X [B, N, C], statistics of every
// sample and group over its N rows and w = C / G channels,
//   xhat = (x - mean) rstd,  z = gamma xhat + beta,  y = act(z),
// and the gradients, with dz = dy act'(z), g = gamma dz and averages over a sample's group,
//   dx = rstd (g - avg(g) - xhat avg(g xhat)),  dgamma = sum dz xhat,  dbeta = sum dz.
//
// Bound by bytes: x (and dy) are needed twice, for the sums and for what follows from them. Samples of up to
// kTeamRows rows stay in registers in between (few_*). Larger ones are read twice, by a kernel that leaves
// the sums of chunks of rows and one that joins them and goes over the rows again (from the last chunk to
// the first, so that it begins with what the L2 still holds); a batch whose tensors pass the L2 goes
// through in groups of samples that fit.
//
// Variances are never differences of large sums: a thread takes up to kRows rows, their mean, the squares about
// that mean, and joins (count, mean, squares) with what it has, as do the joins above it. All sums run
// in a fixed order: two calls on the same inputs give the same bits.
#include <cuda_runtime.h>
#include <math.h>

#include <type_traits>

#include "layer_status.cuh"
#include "checks.h"
#include "linear_internal.h"
#include "tc_ptx.cuh"
#include "vectors.cuh"

namespace flarepp {
namespace {

using namespace vec;

constexpr int kThreads = 256;
// Rows that a thread has in flight: of the forward's sums, and of the backward (x and dy).
template <typename E, int W>
constexpr int sum_rows() { return sizeof(E) * W >= 8 ? 8 : 16; }
template <typename E, int W>
constexpr int back_rows() { return sizeof(E) * W >= 8 ? 4 : 8; }
constexpr int kTeamRows = 4;
constexpr int64_t kWsAlign = 256;

// One call, and how it is cut.
struct Norm {
    const void* x;
    const void* dy;
    void* y;  // y or dx
    const void* gamma;
    const void* beta;
    int param_f32;
    const int* lengths;
    float* stats;       // [B][2][G]: read by the backward, written by the forward (or null)
    int64_t B, N;
    int C, G, w;
    int act;
    float eps;
    int* status;
    // threads: tx vectors of W channels by ty rows; tiles of tc = tx W channels
    int tx, ty, tc, tiles, segs;
    int cell;           // channels that go into a group's sums as one: W, or 1 where groups cut vectors
    int b0, bn;         // samples of this launch
    int chunks, rows;   // chunks of rows a sample, rows of each
    int per;            // samples that a block of the sums takes (1 unless chunks is 1)
    float2* part;       // [B][chunks][G][segs]: (mean, squares) or (sum g, sum g xhat)
    float2* channels;   // [blocks][C]: (sum dz xhat, sum dz)
    int channel_rows;
};

__device__ __forceinline__ int live_rows(const Norm& p, int64_t b) {
    if (!p.lengths) return (int)p.N;
    const int n = p.lengths[b];
    if (n < 0 || n > p.N) {
        if (threadIdx.x == 0) record_status(p.status, FLAREPP_ERR_INVALID_ARGUMENT);
        return n < 0 ? 0 : (int)p.N;
    }
    return n;
}

__device__ __forceinline__ float param(const void* t, int f32, int c, float none) {
    if (!t) return none;
    return f32 ? ((const float*)t)[c] : widen(((const __nv_bfloat16*)t)[c]);
}

// ---- the activation and its slope: 16-bit results from the linear layer's approximations in pairs,
// 32-bit ones from the functions themselves, but for SiLU's exponential and reciprocal: with expf and a
// division the errors of Y, dX, dgamma and dbeta are the same but for a few per cent (8e-8 to 1.6e-7 of their
// norms, which are the sums'), and the backward of 6 x 99,991 x 250 takes 695 us instead of 590. The choice is
// outside the loops over a vector, whose values then go through the exponentials together: inside them it took
// the backward of 65,536 rows of 256 99 us instead of 56.
// 1 / (1 + exp(-z)): the exponential's relative error is |z| 2^-24 and two units more, and the result's the
// same for z far below 0, where it goes to 0, and less elsewhere.
__device__ __forceinline__ float logistic(float z) {
    return rcp_approx(1.f + ex2_approx(-1.44269504f * z));
}
template <int ACT, int W>
__device__ __forceinline__ void value_pairs(float* z) {
#pragma unroll
    for (int i = 0; i < W; i += 2) {
        const float2 v = halves(act_value2(ACT, pair(z[i], W > 1 ? z[(i + 1) % W] : 0.f)));
        z[i] = v.x;
        if (W > 1) z[(i + 1) % W] = v.y;
    }
}
template <int ACT, int W>
__device__ __forceinline__ void slope_pairs(float* z) {
#pragma unroll
    for (int i = 0; i < W; i += 2) {
        const float2 v = halves(act_slope2(ACT, pair(z[i], W > 1 ? z[(i + 1) % W] : 0.f)));
        z[i] = v.x;
        if (W > 1) z[(i + 1) % W] = v.y;
    }
}
template <typename E, int W>
__device__ __forceinline__ void act_value(int act, float* z) {
    constexpr bool exact = std::is_same<E, float>::value;
    if (act == FLAREPP_ACT_RELU) {
        value_pairs<FLAREPP_ACT_RELU, W>(z);
    } else if (act == FLAREPP_ACT_GELU) {
        if (!exact) value_pairs<FLAREPP_ACT_GELU, W>(z);
        else
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] *= normcdff(z[i]);
    } else if (act == FLAREPP_ACT_SILU) {
        if (!exact) value_pairs<FLAREPP_ACT_SILU, W>(z);
        else
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] *= logistic(z[i]);
    }
}
// z becomes act'(z)
template <typename E, int W>
__device__ __forceinline__ void act_slope(int act, float* z) {
    constexpr bool exact = std::is_same<E, float>::value;
    if (act == FLAREPP_ACT_RELU) {
        slope_pairs<FLAREPP_ACT_RELU, W>(z);
    } else if (act == FLAREPP_ACT_GELU) {
        if (!exact) slope_pairs<FLAREPP_ACT_GELU, W>(z);
        else
#pragma unroll
            for (int i = 0; i < W; ++i)
                z[i] = normcdff(z[i]) + z[i] * 0.39894228f * expf(-0.5f * z[i] * z[i]);
    } else if (act == FLAREPP_ACT_SILU) {
        if (!exact) slope_pairs<FLAREPP_ACT_SILU, W>(z);
        else
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float s = logistic(z[i]);
                z[i] = s * (1.f + z[i] * (1.f - s));
            }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) z[i] = 1.f;
    }
}

__device__ __forceinline__ float warp_sum(float v, int lanes = 32) {
    for (int k = lanes >> 1; k; k >>= 1) v += __shfl_xor_sync(0xffffffffu, v, k);
    return v;
}

// The rows that thread y of `ty` takes of `rows`: y, y + ty, ...
__device__ __forceinline__ int rows_of(int rows, int y, int ty) {
    return rows > y ? (rows - y - 1) / ty + 1 : 0;
}

// The part of group g that lies in the tile's channels [c0, c1).
__device__ __forceinline__ void segment(const Norm& p, int g, int c0, int c1, int& from, int& to) {
    from = max(c0, g * p.w);
    to = min(c1, (g + 1) * p.w);
}
__device__ __forceinline__ float2* slot(const Norm& p, int64_t b, int chunk, int g, int tile) {
    const int first = g * p.w / p.tc;
    return p.part + ((b * p.chunks + chunk) * p.G + g) * p.segs + (tile - first);
}

// Lanes that share a group of so many entries: a power of two, so that small groups share a warp.
__device__ __forceinline__ int lanes_for(int entries) {
    int n = 1;
    while (n < 32 && n < entries) n *= 2;
    return n;
}

// What a block is of a launch: a tile of channels, and a chunk of rows of a sample (or several samples).
struct Place {
    int tile, c0, c1;  // channels
    int tx, ty, c;     // the thread's column of vectors, its row, its first channel
    bool on;           // whether the thread has a column
    int unit;          // chunk of the launch
};
template <int W>
__device__ __forceinline__ Place place_of(const Norm& p, int64_t block) {
    Place a;
    a.unit = (int)(block / p.tiles);
    a.tile = (int)(block - (int64_t)a.unit * p.tiles);
    a.c0 = a.tile * p.tc;
    a.c1 = min(p.C, a.c0 + p.tc);
    a.ty = threadIdx.x / p.tx;
    a.tx = threadIdx.x - a.ty * p.tx;
    a.c = a.c0 + a.tx * W;
    a.on = a.ty < p.ty && a.c < a.c1;
    return a;
}

// ------------------------------------------------------------------ sums of the forward
// Bound by reading X once: 8 rows of 8 or 16 bytes (or 16 of less) in flight a thread.
template <typename E, int W>
__global__ void __launch_bounds__(kThreads, 4) stats_kernel(const Norm p) {
    __shared__ float sm[2][kThreads * W];
    constexpr int kRows = sum_rows<E, W>();
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, blockIdx.x);
    const int64_t b = p.b0 + a.unit / p.chunks;
    const int chunk = a.unit % p.chunks;
    const int live = live_rows(p, b);
    const int r0 = chunk * p.rows, r1 = min(live, r0 + p.rows);
    const int rows = max(0, r1 - r0);
    float mean[W], sq[W];
#pragma unroll
    for (int i = 0; i < W; ++i) mean[i] = sq[i] = 0.f;
    if (a.on) {
        const int mine = rows_of(rows, a.ty, p.ty);
        const E* x = (const E*)p.x + (b * p.N + r0 + a.ty) * p.C + a.c;
        const int64_t step = (int64_t)p.ty * p.C;
        int k = 0;
        for (; k + kRows <= mine; k += kRows, x += kRows * step) {
            Pack<E, W> v[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) v[j] = load<E, W>(x + j * step);
            const float f = (float)kRows / (k + kRows), q = f * k;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                float m = 0.f, s = 0.f;
#pragma unroll
                for (int j = 0; j < kRows; ++j) m += widen(v[j].v[i]);
                m *= 1.f / kRows;
#pragma unroll
                for (int j = 0; j < kRows; ++j) {
                    const float d = widen(v[j].v[i]) - m;
                    s = fmaf(d, d, s);
                }
                const float d = m - mean[i];
                mean[i] = fmaf(d, f, mean[i]);
                sq[i] += fmaf(d * d, q, s);
            }
        }
        for (; k < mine; ++k, x += step) {
            const Pack<E, W> v = load<E, W>(x);
            const float f = 1.f / (k + 1), q = f * k;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float d = widen(v.v[i]) - mean[i];
                mean[i] = fmaf(d, f, mean[i]);
                sq[i] = fmaf(d * d, q, sq[i]);
            }
        }
        if (p.cell == W) {  // the vector's channels are one group's
            float m = 0.f, q = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) m += mean[i];
            m *= 1.f / W;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float d = mean[i] - m;
                q += fmaf(d * d, (float)mine, sq[i]);
            }
            sm[0][a.ty * p.tx + a.tx] = m;
            sm[1][a.ty * p.tx + a.tx] = q;
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) {
                sm[0][a.ty * p.tc + a.c - a.c0 + i] = mean[i];
                sm[1][a.ty * p.tc + a.c - a.c0 + i] = sq[i];
            }
        }
    }
    __shared__ float count[kThreads];
    if (threadIdx.x < p.ty) count[threadIdx.x] = (float)(rows_of(rows, threadIdx.x, p.ty) * p.cell);
    __syncthreads();
    // some lanes take a group: the mean of the means, then the squares about it
    const int row = p.tc / p.cell, most = min(p.w, a.c1 - a.c0) / p.cell * p.ty;
    const int lanes = lanes_for(most), lane = threadIdx.x % lanes;
    const int g0 = a.c0 / p.w, groups = (a.c1 - 1) / p.w - g0 + 1;
    for (int k = threadIdx.x / lanes; k - threadIdx.x % 32 / lanes < groups; k += kThreads / lanes) {
        const int g = g0 + k;
        int from = 0, to = 0;
        if (k < groups) segment(p, g, a.c0, a.c1, from, to);
        const int per = (to - from) / p.cell, at0 = (from - a.c0) / p.cell;
        float n = 0.f, m = 0.f;
        for (int e = lane; e < per * p.ty; e += lanes) {
            const int y = per == 1 ? e : e / per, at = y * row + at0 + e - y * per;
            n += count[y];
            m = fmaf(count[y], sm[0][at], m);
        }
        n = warp_sum(n, lanes);
        m = warp_sum(m, lanes);
        m = n > 0.f ? m / n : 0.f;
        float q = 0.f;
        for (int e = lane; e < per * p.ty; e += lanes) {
            const int y = per == 1 ? e : e / per, at = y * row + at0 + e - y * per;
            const float d = sm[0][at] - m;
            q += fmaf(d * d, count[y], sm[1][at]);
        }
        q = warp_sum(q, lanes);
        if (lane == 0 && k < groups) *slot(p, b, chunk, g, a.tile) = make_float2(m, q);
    }
}

// What a block's threads make of the chunks' parts, before they go over the rows again: `lanes` lanes take a
// group, all of the tile's groups at once where they can, so that the parts' latency is met once. Up to
// kHeld parts of a lane stay in registers between the mean and the squares.
constexpr int kHeld = 16;
__device__ __forceinline__ int join_lanes(int groups, int entries) {
    int n = 32;
    while (n > 1 && (n / 2 >= entries || groups * n > kThreads)) n /= 2;
    return n;
}
struct Parts {
    const float2* at;
    int64_t step;  // from a chunk's to the next's
    int first, segs, entries;
};
__device__ __forceinline__ Parts parts_of(const Norm& p, int64_t b, int g) {
    Parts q;
    q.first = g * p.w / p.tc;
    q.segs = ((g + 1) * p.w - 1) / p.tc - q.first + 1;
    q.at = p.part + (b * p.chunks * p.G + g) * (int64_t)p.segs;
    q.step = (int64_t)p.G * p.segs;
    q.entries = p.chunks * q.segs;
    return q;
}
// Entry e and how many values it stands for.
__device__ __forceinline__ float2 part_of(const Norm& p, const Parts& q, int g, int live, int e, float& n) {
    const int k = q.segs == 1 ? e : e / q.segs, s = e - k * q.segs;
    int width = p.w;
    if (q.segs > 1) {
        int from, to;
        segment(p, g, (q.first + s) * p.tc, (q.first + s + 1) * p.tc, from, to);
        width = to - from;
    }
    n = (float)max(0, min(live - k * p.rows, p.rows)) * width;
    return q.at[k * q.step + s];
}
// (mean, 1 / deviation) of group g of sample b
__device__ __forceinline__ float2 join_stats(const Norm& p, int64_t b, int g, int live, int lane, int lanes) {
    const Parts q = parts_of(p, b, g);
    float2 v[kHeld];
    float c[kHeld], n = 0.f, m = 0.f;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        v[j] = make_float2(0.f, 0.f);
        c[j] = 0.f;
        if (lane + j * lanes < q.entries) v[j] = part_of(p, q, g, live, lane + j * lanes, c[j]);
    }
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        n += c[j];
        m = fmaf(c[j], v[j].x, m);
    }
    for (int e = lane + kHeld * lanes; e < q.entries; e += lanes) {
        float k;
        const float2 u = part_of(p, q, g, live, e, k);
        n += k;
        m = fmaf(k, u.x, m);
    }
    n = warp_sum(n, lanes);
    m = warp_sum(m, lanes);
    m = n > 0.f ? m / n : 0.f;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
        const float d = v[j].x - m;
        s += fmaf(d * d, c[j], v[j].y);
    }
    for (int e = lane + kHeld * lanes; e < q.entries; e += lanes) {
        float k;
        const float2 u = part_of(p, q, g, live, e, k);
        const float d = u.x - m;
        s += fmaf(d * d, k, u.y);
    }
    s = warp_sum(s, lanes);
    return make_float2(m, rsqrtf((n > 0.f ? s / n : 0.f) + p.eps));
}

// ------------------------------------------------------------------ the forward's second pass
template <typename E, int W, bool ONE>
__global__ void __launch_bounds__(kThreads, 3) apply_kernel(const Norm p) {
    __shared__ float2 sm[kThreads * W];  // of the tile's groups
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, gridDim.x - 1 - (int64_t)blockIdx.x);
    const int64_t b = p.b0 + a.unit / p.chunks;
    const int chunk = a.unit % p.chunks;
    const int live = live_rows(p, b);
    const int g0 = a.c0 / p.w, groups = (a.c1 - 1) / p.w - g0 + 1;
    const int lanes = join_lanes(groups, p.chunks * p.segs), lane = threadIdx.x % lanes;
    for (int k = threadIdx.x / lanes; k - threadIdx.x % 32 / lanes < groups; k += kThreads / lanes) {
        const int g = min(g0 + k, g0 + groups - 1);  // (all lanes take part)
        const float2 v = join_stats(p, b, g, live, lane, lanes);
        if (lane == 0 && k < groups) {
            sm[g - g0] = v;
            if (p.stats && chunk == 0 && g * p.w >= a.c0) {
                p.stats[b * 2 * p.G + g] = v.x;
                p.stats[(b * 2 + 1) * p.G + g] = v.y;
            }
        }
    }
    __syncthreads();
    if (!a.on) return;
    constexpr int M = ONE ? 1 : W;
    float m[M], f[W], s[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 v = sm[(a.c + i % M) / p.w - g0];
        m[i % M] = v.x;
        f[i] = v.y * param(p.gamma, p.param_f32, a.c + i, 1.f);
        s[i] = param(p.beta, p.param_f32, a.c + i, 0.f);
    }
    const int r0 = chunk * p.rows, r1 = (int)min(p.N, (int64_t)r0 + p.rows);
    const int64_t at = (b * p.N + r0 + a.ty) * p.C + a.c, step = (int64_t)p.ty * p.C;
    const E* x = (const E*)p.x + at;
    E* y = (E*)p.y + at;
    const int all = rows_of(r1 - r0, a.ty, p.ty), mine = rows_of(max(0, live - r0), a.ty, p.ty);
    constexpr int U = 8;
    for (int k = 0; k < all; k += U, x += U * step, y += U * step) {
        Pack<E, W> v[U];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (k + j < mine) v[j] = load<E, W>(x + j * step);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (k + j >= all) break;
            float z[W];
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] = k + j < mine ? fmaf(widen(v[j].v[i]) - m[i % M], f[i], s[i]) : 0.f;
            if (k + j < mine) act_value<E, W>(p.act, z);
#pragma unroll
            for (int i = 0; i < W; ++i) narrow(v[j].v[i], z[i]);
            store<E, W>(y + j * step, v[j]);
        }
    }
}

// ------------------------------------------------------------------ the backward
// A thread's channels: xhat = (x - m) r, z = gamma xhat + beta. Where groups do not cut vectors (ONE) the vector
// has one m and one r, which spares 14 registers of 8 channels (and as many averages').
template <int W, bool ONE>
struct Channels {
    float r[ONE ? 1 : W], m[ONE ? 1 : W], gamma[W], beta[W];
    __device__ __forceinline__ float rstd(int i) const { return r[ONE ? 0 : i]; }
    __device__ __forceinline__ float mean(int i) const { return m[ONE ? 0 : i]; }
};
template <int W, bool ONE>
__device__ __forceinline__ void params_of(const Norm& p, int c, Channels<W, ONE>& h) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        h.gamma[i] = param(p.gamma, p.param_f32, c + i, 1.f);
        h.beta[i] = param(p.beta, p.param_f32, c + i, 0.f);
    }
}
template <int W, bool ONE>
__device__ __forceinline__ void stats_of(const Norm& p, int64_t b, int c, Channels<W, ONE>& h) {
#pragma unroll
    for (int i = 0; i < (ONE ? 1 : W); ++i) {
        const int g = (c + i) / p.w;
        h.r[i] = p.stats[(b * 2 + 1) * p.G + g];
        h.m[i] = p.stats[b * 2 * p.G + g];
    }
}
// xhat and dz of a row's vector
template <typename E, int W, bool ONE>
__device__ __forceinline__ void row_of(const Norm& p, const Channels<W, ONE>& h, const Pack<E, W>& x,
                                       const Pack<E, W>& dy, float* xhat, float* dz) {
#pragma unroll
    for (int i = 0; i < W; ++i) xhat[i] = (widen(x.v[i]) - h.mean(i)) * h.rstd(i);
    if (p.act == FLAREPP_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < W; ++i) dz[i] = widen(dy.v[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) dz[i] = fmaf(h.gamma[i], xhat[i], h.beta[i]);
    act_slope<E, W>(p.act, dz);
#pragma unroll
    for (int i = 0; i < W; ++i) dz[i] *= widen(dy.v[i]);
}

// The sums over a chunk of rows (or over all rows of several samples): by group, sum g and sum g xhat, for
// dx; by channel, sum dz xhat and sum dz, for dgamma and dbeta.
template <typename E, int W, bool ONE>
__global__ void __launch_bounds__(kThreads, 3) back_sums_kernel(const Norm p) {
    __shared__ float sm[2][kThreads * W];
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, blockIdx.x);
    const int64_t from_b = p.b0 + (p.chunks > 1 ? a.unit / p.chunks : (int64_t)a.unit * p.per);
    const int64_t to_b = p.chunks > 1 ? from_b + 1 : min((int64_t)p.b0 + p.bn, from_b + p.per);
    const int chunk = p.chunks > 1 ? a.unit % p.chunks : 0;
    constexpr int kBackRows = back_rows<E, W>();
    Channels<W, ONE> h;
    __shared__ float all[2][kThreads * W];  // of the block's samples, by channel and row of threads
    if (a.on) params_of<W, ONE>(p, a.c, h);
    for (int64_t b = from_b; b < to_b; ++b) {
        const int live = live_rows(p, b);
        const int r0 = chunk * p.rows, rows = max(0, min(live, r0 + p.rows) - r0);
        float u[W], v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) u[i] = v[i] = 0.f;
        if (a.on) {
            stats_of<W, ONE>(p, b, a.c, h);
            const int mine = rows_of(rows, a.ty, p.ty);
            const int64_t at = (b * p.N + r0 + a.ty) * p.C + a.c, step = (int64_t)p.ty * p.C;
            const E* x = (const E*)p.x + at;
            const E* dy = (const E*)p.dy + at;
            for (int k = 0; k < mine; k += kBackRows, x += kBackRows * step, dy += kBackRows * step) {
                Pack<E, W> px[kBackRows], pd[kBackRows];
#pragma unroll
                for (int j = 0; j < kBackRows; ++j)
                    if (k + j < mine) {
                        px[j] = load<E, W>(x + j * step);
                        pd[j] = load<E, W>(dy + j * step);
                    }
#pragma unroll
                for (int j = 0; j < kBackRows; ++j)
                    if (k + j < mine) {
                        float xhat[W], dz[W];
                        row_of<E, W, ONE>(p, h, px[j], pd[j], xhat, dz);
#pragma unroll
                        for (int i = 0; i < W; ++i) {
                            u[i] = fmaf(dz[i], xhat[i], u[i]);
                            v[i] += dz[i];
                        }
                    }
            }
            float s0 = 0.f, s1 = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float g0 = v[i] * h.gamma[i], g1 = u[i] * h.gamma[i];
                if (p.channels) {
                    const int at = a.ty * p.tc + a.c - a.c0 + i;
                    all[0][at] = b > from_b ? all[0][at] + u[i] : u[i];
                    all[1][at] = b > from_b ? all[1][at] + v[i] : v[i];
                }
                s0 += g0;
                s1 += g1;
                if (p.cell != W) {
                    sm[0][a.ty * p.tc + a.c - a.c0 + i] = g0;
                    sm[1][a.ty * p.tc + a.c - a.c0 + i] = g1;
                }
            }
            if (p.cell == W) {
                sm[0][a.ty * p.tx + a.tx] = s0;
                sm[1][a.ty * p.tx + a.tx] = s1;
            }
        }
        __syncthreads();
        const int row = p.tc / p.cell, most = min(p.w, a.c1 - a.c0) / p.cell * p.ty;
        const int lanes = lanes_for(most), lane = threadIdx.x % lanes;
        const int g0 = a.c0 / p.w, groups = (a.c1 - 1) / p.w - g0 + 1;
        for (int k = threadIdx.x / lanes; k - threadIdx.x % 32 / lanes < groups; k += kThreads / lanes) {
            const int g = g0 + k;
            int from = 0, to = 0;
            if (k < groups) segment(p, g, a.c0, a.c1, from, to);
            const int per = (to - from) / p.cell, at0 = (from - a.c0) / p.cell;
            float s0 = 0.f, s1 = 0.f;
            for (int e = lane; e < per * p.ty; e += lanes) {
                const int y = per == 1 ? e : e / per, at = y * row + at0 + e - y * per;
                s0 += sm[0][at];
                s1 += sm[1][at];
            }
            s0 = warp_sum(s0, lanes);
            s1 = warp_sum(s1, lanes);
            if (lane == 0 && k < groups) *slot(p, b, chunk, g, a.tile) = make_float2(s0, s1);
        }
        __syncthreads();
    }
    if (!p.channels) return;
    float2* out = p.channels + (int64_t)(p.channel_rows + a.unit) * p.C;
    for (int c = a.c0 + threadIdx.x; c < a.c1; c += kThreads) {
        float s0 = 0.f, s1 = 0.f;
        for (int y = 0; y < p.ty; ++y) {
            s0 += all[0][y * p.tc + c - a.c0];
            s1 += all[1][y * p.tc + c - a.c0];
        }
        out[c] = make_float2(s0, s1);
    }
}

template <typename E, int W, bool ONE>
__global__ void __launch_bounds__(kThreads, 3) back_apply_kernel(const Norm p) {
    __shared__ float2 sm[kThreads * W];
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, gridDim.x - 1 - (int64_t)blockIdx.x);
    const int64_t b = p.b0 + a.unit / p.chunks;
    const int chunk = a.unit % p.chunks;
    const int live = live_rows(p, b);
    const int g0 = a.c0 / p.w;
    constexpr int kBackRows = back_rows<E, W>();
    const float each = 1.f / fmaxf(1.f, (float)live * p.w);
    const int groups = (a.c1 - 1) / p.w - g0 + 1;
    const int lanes = join_lanes(groups, p.chunks * p.segs), lane = threadIdx.x % lanes;
    for (int k = threadIdx.x / lanes; k - threadIdx.x % 32 / lanes < groups; k += kThreads / lanes) {
        const int g = min(g0 + k, g0 + groups - 1);
        const Parts q = parts_of(p, b, g);
        float s0 = 0.f, s1 = 0.f;
#pragma unroll 8
        for (int e = lane; e < q.entries; e += lanes) {
            const int c = q.segs == 1 ? e : e / q.segs;
            const float2 v = q.at[c * q.step + e - c * q.segs];
            s0 += v.x;
            s1 += v.y;
        }
        s0 = warp_sum(s0, lanes);
        s1 = warp_sum(s1, lanes);
        if (lane == 0 && k < groups) sm[g - g0] = make_float2(s0 * each, s1 * each);
    }
    __syncthreads();
    if (!a.on) return;
    Channels<W, ONE> h;
    params_of<W, ONE>(p, a.c, h);
    stats_of<W, ONE>(p, b, a.c, h);
    constexpr int M = ONE ? 1 : W;
    float m0[M], m1[M];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const float2 v = sm[(a.c + i) / p.w - g0];
        m0[i] = v.x;
        m1[i] = v.y;
    }
    const int r0 = chunk * p.rows, r1 = (int)min(p.N, (int64_t)r0 + p.rows);
    const int64_t at = (b * p.N + r0 + a.ty) * p.C + a.c, step = (int64_t)p.ty * p.C;
    const E* x = (const E*)p.x + at;
    const E* dy = (const E*)p.dy + at;
    E* dx = (E*)p.y + at;
    const int all = rows_of(r1 - r0, a.ty, p.ty), mine = rows_of(max(0, live - r0), a.ty, p.ty);
    for (int k = 0; k < all; k += kBackRows, x += kBackRows * step, dy += kBackRows * step,
             dx += kBackRows * step) {
        Pack<E, W> px[kBackRows], pd[kBackRows];
#pragma unroll
        for (int j = 0; j < kBackRows; ++j)
            if (k + j < mine) {
                px[j] = load<E, W>(x + j * step);
                pd[j] = load<E, W>(dy + j * step);
            }
#pragma unroll
        for (int j = 0; j < kBackRows; ++j) {
            if (k + j >= all) break;
            float xhat[W], dz[W];
            if (k + j < mine) {
                row_of<E, W, ONE>(p, h, px[j], pd[j], xhat, dz);
#pragma unroll
                for (int i = 0; i < W; ++i)
                    dz[i] = h.rstd(i) * (fmaf(dz[i], h.gamma[i], -m0[i % M]) - xhat[i] * m1[i % M]);
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) dz[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) narrow(px[j].v[i], dz[i]);
            store<E, W>(dx + j * step, px[j]);
        }
    }
}

// dgamma and dbeta from rows [R][C] of (sum dz xhat, sum dz): a block takes 8 channels, each of 128 threads
// every 128th row of one, in order; then their sums by halves.
constexpr int kReduceThreads = 1024, kReduceChannels = 8, kReduceRows = kReduceThreads / kReduceChannels;
template <typename P>
__global__ void __launch_bounds__(kReduceThreads)
    channels_kernel(const float2* rows, int R, int C, P* dgamma, P* dbeta) {
    __shared__ float2 sm[kReduceRows][kReduceChannels];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int x = threadIdx.x % kReduceChannels, y = threadIdx.x / kReduceChannels;
    const int c = blockIdx.x * kReduceChannels + x;
    float2 s = make_float2(0.f, 0.f);
    if (c < C)
#pragma unroll 4
        for (int r = y; r < R; r += kReduceRows) {
            const float2 v = rows[(int64_t)r * C + c];
            s.x += v.x;
            s.y += v.y;
        }
    sm[y][x] = s;
    for (int k = kReduceRows / 2; k; k >>= 1) {
        __syncthreads();
        if (y >= k) continue;
        s.x += sm[y + k][x].x;
        s.y += sm[y + k][x].y;
        sm[y][x] = s;
    }
    if (y || c >= C) return;
    if (dgamma) narrow(dgamma[c], s.x);
    if (dbeta) narrow(dbeta[c], s.y);
}

// ------------------------------------------------------------------ few rows a sample
// `lanes` lanes (a power of two) take a sample's group, its K rows of V vectors a lane staying in registers:
// one pass over the data and one launch. A block's 256 / lanes such teams and all blocks' together are a
// multiple of G, so that a team walks the samples with the same channels.
struct Team {
    int g, lane;
    int64_t row, rows;  // of the teams with this g: the team's place, their number
};
__device__ __forceinline__ Team team_of(const Norm& p, int lanes) {
    const int per = kThreads / lanes;
    const int64_t id = (int64_t)blockIdx.x * per + threadIdx.x / lanes;
    Team t;
    t.lane = threadIdx.x % lanes;
    t.row = id / p.G;
    t.g = (int)(id - t.row * p.G);
    t.rows = (int64_t)gridDim.x * per / p.G;
    return t;
}
__device__ __forceinline__ int live_rows_few(const Norm& p, int64_t b, bool on) {
    if (!on) return 0;
    if (!p.lengths) return (int)p.N;
    const int n = p.lengths[b];
    if (n >= 0 && n <= p.N) return n;
    record_status(p.status, FLAREPP_ERR_INVALID_ARGUMENT);
    return n < 0 ? 0 : (int)p.N;
}

template <typename E, int W, int K, int V>
__global__ void __launch_bounds__(kThreads) few_kernel(const Norm p, int lanes) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const Team t = team_of(p, lanes);
    const int vectors = p.w / W;
    float f[V * W], s[V * W];
    bool has[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        has[v] = v * lanes + t.lane < vectors;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int c = t.g * p.w + (v * lanes + t.lane) * W + i;
            f[v * W + i] = has[v] ? param(p.gamma, p.param_f32, c, 1.f) : 0.f;
            s[v * W + i] = has[v] ? param(p.beta, p.param_f32, c, 0.f) : 0.f;
        }
    }
    const int64_t turns = (p.B + t.rows - 1) / t.rows;
    for (int64_t k = 0; k < turns; ++k) {  // all lanes take part in the sums
        const int64_t b = k * t.rows + t.row;
        const bool on = b < p.B;
        const int live = live_rows_few(p, b, on);
        const int64_t at = b * p.N * p.C + t.g * p.w + t.lane * W;
        Pack<E, W> x[K][V];
        float m = 0.f, q = 0.f;
#pragma unroll
        for (int r = 0; r < K; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r < live && has[v]) x[r][v] = load<E, W>((const E*)p.x + at + (int64_t)r * p.C + v * lanes * W);
#pragma unroll
        for (int r = 0; r < K; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r < live && has[v])
#pragma unroll
                    for (int i = 0; i < W; ++i) m += widen(x[r][v].v[i]);
        const float each = 1.f / fmaxf(1.f, (float)live * p.w);
        m = warp_sum(m, lanes) * each;
#pragma unroll
        for (int r = 0; r < K; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r < live && has[v])
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float d = widen(x[r][v].v[i]) - m;
                        q = fmaf(d, d, q);
                    }
        q = rsqrtf(warp_sum(q, lanes) * each + p.eps);
        if (!on) continue;
        if (p.stats && t.lane == 0) {
            p.stats[b * 2 * p.G + t.g] = m;
            p.stats[(b * 2 + 1) * p.G + t.g] = q;
        }
#pragma unroll
        for (int r = 0; r < K; ++r) {
            if (r >= p.N) break;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!has[v]) continue;
                float z[W];
#pragma unroll
                for (int i = 0; i < W; ++i)
                    z[i] = r < live ? fmaf(widen(x[r][v].v[i]) - m, q * f[v * W + i], s[v * W + i]) : 0.f;
                if (r < live) act_value<E, W>(p.act, z);
#pragma unroll
                for (int i = 0; i < W; ++i) narrow(x[r][v].v[i], z[i]);
                store<E, W>((E*)p.y + at + (int64_t)r * p.C + v * lanes * W, x[r][v]);
            }
        }
    }
}

template <typename E, int W, int K, int V>
__global__ void __launch_bounds__(kThreads) back_few_kernel(const Norm p, int lanes) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const Team t = team_of(p, lanes);
    const int vectors = p.w / W;
    Channels<W, true> h[V];
    float u[V * W], w[V * W];
    bool has[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        has[v] = v * lanes + t.lane < vectors;
        if (has[v]) params_of<W, true>(p, t.g * p.w + (v * lanes + t.lane) * W, h[v]);
#pragma unroll
        for (int i = 0; i < W; ++i) u[v * W + i] = w[v * W + i] = 0.f;
    }
    const int64_t turns = (p.B + t.rows - 1) / t.rows;
    for (int64_t k = 0; k < turns; ++k) {
        const int64_t b = k * t.rows + t.row;
        const bool on = b < p.B;
        const int live = live_rows_few(p, b, on);
        if (on)
#pragma unroll
            for (int v = 0; v < V; ++v) stats_of<W, true>(p, b, t.g * p.w, h[v]);
        const int64_t at = b * p.N * p.C + t.g * p.w + t.lane * W;
        Pack<E, W> x[K][V], dy[K][V];
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int r = 0; r < K; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r < live && has[v]) {
                    x[r][v] = load<E, W>((const E*)p.x + at + (int64_t)r * p.C + v * lanes * W);
                    dy[r][v] = load<E, W>((const E*)p.dy + at + (int64_t)r * p.C + v * lanes * W);
                }
#pragma unroll
        for (int r = 0; r < K; ++r)
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (r < live && has[v]) {
                    float xhat[W], dz[W];
                    row_of<E, W, true>(p, h[v], x[r][v], dy[r][v], xhat, dz);
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        u[v * W + i] = fmaf(dz[i], xhat[i], u[v * W + i]);
                        w[v * W + i] += dz[i];
                        const float g = dz[i] * h[v].gamma[i];
                        s0 += g;
                        s1 = fmaf(g, xhat[i], s1);
                    }
                }
        const float each = 1.f / fmaxf(1.f, (float)live * p.w);
        s0 = warp_sum(s0, lanes) * each;
        s1 = warp_sum(s1, lanes) * each;
        if (!on) continue;
#pragma unroll
        for (int r = 0; r < K; ++r) {
            if (r >= p.N) break;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!has[v]) continue;
                float xhat[W], dz[W];
                if (r < live) {
                    row_of<E, W, true>(p, h[v], x[r][v], dy[r][v], xhat, dz);
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        dz[i] = h[v].rstd(i) * (fmaf(dz[i], h[v].gamma[i], -s0) - xhat[i] * s1);
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) dz[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < W; ++i) narrow(x[r][v].v[i], dz[i]);
                store<E, W>((E*)p.y + at + (int64_t)r * p.C + v * lanes * W, x[r][v]);
            }
        }
    }
    if (!p.channels) return;
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (has[v])
#pragma unroll
            for (int i = 0; i < W; ++i)
                p.channels[t.row * p.C + t.g * p.w + (v * lanes + t.lane) * W + i] =
                    make_float2(u[v * W + i], w[v * W + i]);
}

// Statistics of samples without rows: those of one whose length is 0.
__global__ void __launch_bounds__(kThreads) empty_kernel(float* stats, int64_t n, int G, float eps) {
    tc::pdl_trigger();
    tc::pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads)
        stats[i] = i / G % 2 ? rsqrtf(eps) : 0.f;
}

// ------------------------------------------------------------------ host side
template <typename... Args>
cudaError_t launch(void (*kernel)(Args...), int64_t blocks, int threads, cudaStream_t st,
                   const std::common_type_t<Args>&... args) {
    if (blocks <= 0 || blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(threads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Args(args)...);
}

size_t up(size_t n) { return (n + kWsAlign - 1) / kWsAlign * kWsAlign; }

// How a call is cut: the same for sizing its workspace and for running it.
struct Plan {
    int W, tx, ty, tc, tiles, segs, cell;
    int lanes, each;  // > 0: few rows, groups of that many lanes of `each` vectors a row
    int chunks, rows, per;
    int64_t group;    // samples that go through together
    int64_t units;    // rows of `channels` that a call leaves
    int64_t blocks;   // with few rows
    size_t off_channels, total;
};

int64_t elem_of(const flarepp_norm_shape& s) { return s.dtype == FLAREPP_BF16 ? 2 : 4; }

Plan plan_of(const flarepp_norm_shape& s, bool backward) {
    Plan p{};
    const int64_t e = elem_of(s);
    p.W = 4;
    while (s.C % p.W) p.W /= 2;
    const int64_t vectors = s.C / p.W, w = s.C / s.G;
    // Few rows, whose vectors do not cut groups: a warp or a part of one takes a group, if it has room
    // (1,024 channels of one row; a layer norm of more goes the long way).
    if (s.N <= kTeamRows && w % p.W == 0) {
        const int64_t vectors_of = w / p.W;
        p.lanes = 1;
        while (p.lanes < 32 && p.lanes < vectors_of) p.lanes *= 2;
        p.each = 1;
        while (p.each * p.lanes < vectors_of) p.each *= 2;
        if (p.each > (s.N == 1 && p.W == 4 ? 8 : 1)) p.lanes = 0;
    }
    p.tiles = (int)cdiv(vectors, kThreads);
    p.tx = (int)cdiv(vectors, p.tiles);
    p.tiles = (int)cdiv(vectors, p.tx);
    p.ty = kThreads / p.tx;
    p.tc = p.tx * p.W;
    p.cell = w % p.W == 0 ? p.W : 1;
    // the most tiles that w channels side by side can touch
    p.segs = (int)(w < 2 ? 1 : (w - 2) / p.tc + 2);
    if (p.segs > p.tiles) p.segs = p.tiles;
    p.per = 1;
    if (p.lanes) {
        // blocks in steps of as many as hold whole sets of G teams; 4 an SM at most
        const int64_t teams = kThreads / p.lanes;
        int64_t step = s.G;
        for (int64_t d = teams; d > 1 && step % 2 == 0; d /= 2) step /= 2;
        int64_t blocks = cdiv(s.B * s.G, teams);
        if (blocks > kNumSMs * 4) blocks = kNumSMs * 4;
        p.blocks = cdiv(blocks, step) * step;
        p.units = p.blocks * teams / s.G;
        p.chunks = 1;
        p.rows = (int)s.N;
        p.group = s.B;
    } else {
        // samples whose tensors stay in the L2 between the passes
        const int64_t bytes = s.N * s.C * e * (backward ? 2 : 1);
        p.group = (int64_t)(64 << 20) / (bytes ? bytes : 1);
        if (p.group < 1) p.group = 1;
        if (p.group > s.B) p.group = s.B;
        p.group = cdiv(s.B, cdiv(s.B, p.group));
        // Three blocks an SM, with 8 rows a thread at least where there are so many: a block's own sums take as long
        // as some ten rows of its threads.
        const int64_t wanted = cdiv(kNumSMs * 3, p.group * p.tiles);
        const int64_t least = (int64_t)p.ty * 8;
        p.chunks = (int)(wanted < cdiv(s.N, least) ? wanted : cdiv(s.N, least));
        if (p.chunks < 1) p.chunks = 1;
        p.rows = (int)cdiv(s.N, p.chunks);
        p.chunks = (int)cdiv(s.N, p.rows);
        if (p.chunks == 1) {
            const int64_t blocks = cdiv(kNumSMs * 3, p.tiles);
            p.per = (int)cdiv(p.group, blocks);
        }
        const int64_t whole = s.B / p.group, rest = s.B - whole * p.group;
        p.units = p.chunks > 1 ? s.B * p.chunks : whole * cdiv(p.group, p.per) + cdiv(rest, p.per);
    }
    size_t at = p.lanes ? 0 : up((size_t)s.B * p.chunks * s.G * p.segs * sizeof(float2));
    p.off_channels = at;
    if (backward) at += up((size_t)p.units * s.C * sizeof(float2));
    p.total = at;
    return p;
}

// The kernel for few rows: of one row and up to 8 vectors a lane, or of up to four rows.
#define FLAREPP_FEW(kernel)                                                                   \
    (a.N > 1         ? launch(kernel<E, W, kTeamRows, 1>, p.blocks, kThreads, st, a, p.lanes) \
     : p.each == 1   ? launch(kernel<E, W, 1, 1>, p.blocks, kThreads, st, a, p.lanes)         \
     : p.each == 2   ? launch(kernel<E, W, 1, W == 4 ? 2 : 1>, p.blocks, kThreads, st, a, p.lanes) \
     : p.each == 4   ? launch(kernel<E, W, 1, W == 4 ? 4 : 1>, p.blocks, kThreads, st, a, p.lanes) \
                     : launch(kernel<E, W, 1, W == 4 ? 8 : 1>, p.blocks, kThreads, st, a, p.lanes))

template <typename E, int W>
cudaError_t forward(Norm a, const Plan& p, cudaStream_t st) {
    if (p.lanes) return FLAREPP_FEW(few_kernel);
    for (int64_t b = 0; b < a.B; b += p.group) {
        a.b0 = (int)b;
        a.bn = (int)(a.B - b < p.group ? a.B - b : p.group);
        const int64_t blocks = (int64_t)a.bn * p.chunks * p.tiles;
        cudaError_t e = launch(stats_kernel<E, W>, blocks, kThreads, st, a);
        if (e == cudaSuccess)
            e = launch(a.cell == W ? apply_kernel<E, W, true> : apply_kernel<E, W, W == 1>, blocks, kThreads, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename E, int W>
cudaError_t backward(Norm a, const Plan& p, cudaStream_t st) {
    if (p.lanes) return FLAREPP_FEW(back_few_kernel);
    int rows = 0;
    for (int64_t b = 0; b < a.B; b += p.group) {
        a.b0 = (int)b;
        a.bn = (int)(a.B - b < p.group ? a.B - b : p.group);
        a.channel_rows = rows;
        const int64_t units = p.chunks > 1 ? (int64_t)a.bn * p.chunks : cdiv(a.bn, p.per);
        rows += (int)units;
        cudaError_t e = launch(a.cell == W ? back_sums_kernel<E, W, true> : back_sums_kernel<E, W, W == 1>,
                               units * p.tiles, kThreads, st, a);
        if (e == cudaSuccess)
            e = launch(a.cell == W ? back_apply_kernel<E, W, true> : back_apply_kernel<E, W, W == 1>,
                       (int64_t)a.bn * p.chunks * p.tiles, kThreads, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

// Vectors of 4 channels for 16 bits, too: with 8 the constants of the activations and two vectors' values and
// sums do not fit the registers of 3 blocks an SM.
template <typename E>
cudaError_t run(bool back, const Norm& a, const Plan& p, cudaStream_t st) {
    switch (p.W) {
        case 4: return back ? backward<E, 4>(a, p, st) : forward<E, 4>(a, p, st);
        case 2: return back ? backward<E, 2>(a, p, st) : forward<E, 2>(a, p, st);
        default: return back ? backward<E, 1>(a, p, st) : forward<E, 1>(a, p, st);
    }
}

flarepp_status check(const flarepp_norm_shape* s) {
    if (!s || s->B < 0 || s->N < 0 || s->C < 1 || s->G < 1) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->C % s->G) return FLAREPP_ERR_INVALID_ARGUMENT;
    for (int t : {s->dtype, s->param_dtype})
        if (t != FLAREPP_F32 && t != FLAREPP_BF16) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->act < FLAREPP_ACT_NONE || s->act > FLAREPP_ACT_SILU) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!isfinite(s->eps) || s->eps <= 0.f) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->C > (1 << 20) || s->N > (int64_t(1) << 30) || s->B > (int64_t(1) << 30))
        return FLAREPP_ERR_UNSUPPORTED;
    if (s->B && s->N > (int64_t(1) << 47) / s->B / s->C) return FLAREPP_ERR_UNSUPPORTED;
    // the launches' blocks and the sums' rows are counted in 31 bits
    if (s->B * cdiv(s->C, kThreads) > (int64_t(1) << 30)) return FLAREPP_ERR_UNSUPPORTED;
    return FLAREPP_OK;
}

flarepp_status group_norm(bool back, const flarepp_norm_shape* shape, const void* x, const void* dy,
                          const void* gamma, const void* beta, const int32_t* lengths, float* stats,
                          void* y, void* dgamma, void* dbeta, void* workspace, size_t workspace_bytes,
                          int32_t* status, cudaStream_t st) {
    const flarepp_status bad = check(shape);
    if (bad != FLAREPP_OK) return bad;
    const flarepp_norm_shape s = *shape;
    const size_t n = (size_t)(s.B * s.N * s.C * elem_of(s));
    const size_t pn = (size_t)s.C * (s.param_dtype == FLAREPP_BF16 ? 2 : 4);
    const size_t sn = (size_t)s.B * 2 * s.G * 4;
    for (const void* t : {(const void*)gamma, (const void*)beta, (const void*)dgamma,
                          (const void*)dbeta, (const void*)stats, (const void*)lengths,
                          (const void*)status})
        if (t && !aligned4(t)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const Plan p = n ? plan_of(s, back) : Plan{};
    const bool sums = back && (dgamma || dbeta);
    if (n) {
        if (!x || !y || (back && (!dy || !stats))) return FLAREPP_ERR_INVALID_ARGUMENT;
        for (const void* t : {x, (const void*)y, dy})
            if (t && !aligned16(t)) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (p.total && (!workspace || (uintptr_t)workspace % kWsAlign || workspace_bytes < p.total))
            return FLAREPP_ERR_WORKSPACE;
    }
    const Span outs[6] = {{y, n},           {back ? nullptr : stats, sn}, {dgamma, pn},
                          {dbeta, pn},      {workspace, n ? p.total : 0}, {status, 4}};
    const Span ins[6] = {{x, n},        {dy, n},
                         {gamma, pn},   {beta, pn},
                         {lengths, (size_t)s.B * 4}, {back ? stats : nullptr, sn}};
    if (!disjoint(outs, 6, ins, 6)) return FLAREPP_ERR_INVALID_ARGUMENT;
    cudaError_t e = cudaSuccess;
    if (n == 0) {
        const int64_t values = s.B * 2 * s.G;
        if (!back && stats && values)
            e = launch(empty_kernel, values < kNumSMs * kThreads ? cdiv(values, kThreads) : kNumSMs, kThreads, st,
                       stats, values, (int)s.G, s.eps);
        if (back && dgamma) e = cudaMemsetAsync(dgamma, 0, pn, st);
        if (back && dbeta && e == cudaSuccess) e = cudaMemsetAsync(dbeta, 0, pn, st);
        return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
    }
    Norm a{};
    a.x = x, a.dy = dy, a.y = y, a.gamma = gamma, a.beta = beta;
    a.param_f32 = s.param_dtype == FLAREPP_F32;
    a.lengths = lengths, a.stats = stats;
    a.B = s.B, a.N = s.N, a.C = (int)s.C, a.G = (int)s.G, a.w = (int)(s.C / s.G);
    a.act = s.act, a.eps = s.eps, a.status = status;
    a.tx = p.tx, a.ty = p.ty, a.tc = p.tc, a.cell = p.cell, a.tiles = p.tiles, a.segs = p.segs;
    a.chunks = p.chunks, a.rows = p.rows, a.per = p.per;
    a.part = (float2*)workspace;
    a.channels = sums ? (float2*)((char*)workspace + p.off_channels) : nullptr;
    e = s.dtype == FLAREPP_BF16 ? run<__nv_bfloat16>(back, a, p, st) : run<float>(back, a, p, st);
    if (e == cudaSuccess && sums) {
        const int64_t blocks = cdiv(s.C, kReduceChannels);
        if (s.param_dtype == FLAREPP_F32)
            e = launch(channels_kernel<float>, blocks, kReduceThreads, st, (const float2*)a.channels,
                       (int)p.units, (int)s.C, (float*)dgamma, (float*)dbeta);
        else
            e = launch(channels_kernel<__nv_bfloat16>, blocks, kReduceThreads, st,
                       (const float2*)a.channels, (int)p.units, (int)s.C, (__nv_bfloat16*)dgamma,
                       (__nv_bfloat16*)dbeta);
    }
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

size_t workspace_bytes(const flarepp_norm_shape* s, bool back) {
    if (check(s) != FLAREPP_OK || s->B == 0 || s->N == 0) return 0;
    return plan_of(*s, back).total;
}

}  // namespace

cudaError_t take_norm_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

}  // namespace flarepp

extern "C" {

size_t flarepp_group_norm_workspace_bytes(const flarepp_norm_shape* shape) {
    return flarepp::workspace_bytes(shape, false);
}

flarepp_status flarepp_group_norm_fwd(const flarepp_norm_shape* shape, const void* X,
                                      const void* gamma, const void* beta, const int32_t* lengths,
                                      void* Y, float* stats, void* workspace, size_t workspace_bytes,
                                      int32_t* status, void* stream) {
    return flarepp::group_norm(false, shape, X, nullptr, gamma, beta, lengths, stats, Y, nullptr, nullptr,
                               workspace, workspace_bytes, status, (cudaStream_t)stream);
}

size_t flarepp_group_norm_bwd_workspace_bytes(const flarepp_norm_shape* shape) {
    return flarepp::workspace_bytes(shape, true);
}

flarepp_status flarepp_group_norm_bwd(const flarepp_norm_shape* shape, const void* X, const void* dY,
                                      const void* gamma, const void* beta, const int32_t* lengths,
                                      const float* stats, void* dX, void* dgamma, void* dbeta,
                                      void* workspace, size_t workspace_bytes, int32_t* status,
                                      void* stream) {
    return flarepp::group_norm(true, shape, X, dY, gamma, beta, lengths, const_cast<float*>(stats), dX,
                               dgamma, dbeta, workspace, workspace_bytes, status, (cudaStream_t)stream);
}

}  // extern "C"
