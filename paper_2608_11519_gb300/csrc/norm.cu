// Group norm with an activation, channels last (flarepp_group_norm_*): X [B, N, C], statistics of every
// sample and group over its N rows and w = C / G channels,
//   xhat = (x - mean) rstd,  z = gamma xhat + beta,  y = act(z),
// and the gradients, with dz = dy act'(z), g = gamma dz and averages over a sample's group,
//   dx = rstd (g - avg(g) - xhat avg(g xhat)),  dgamma = sum dz xhat,  dbeta = sum dz.
//
// Bound by bytes: x (and dy) are needed twice, for the sums and for what follows from them. Samples of up to
// kFewRows rows stay in registers in between (few_*). Larger ones are read twice, by a kernel that leaves
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
constexpr int kRows = 8;      // rows that a thread of the forward's sums has in flight
constexpr int kBackRows = 4;  // of the backward's: x and dy
constexpr int kFewRows = 4;
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
// 32-bit ones from the functions themselves
template <typename E, int W>
__device__ __forceinline__ void act_value(int act, float* z) {
    if (act == FLAREPP_ACT_NONE) return;
    if (std::is_same<E, float>::value) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (act == FLAREPP_ACT_RELU) z[i] = z[i] < 0.f ? 0.f : z[i];
            else if (act == FLAREPP_ACT_GELU) z[i] *= normcdff(z[i]);
            else z[i] /= 1.f + expf(-z[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            const float2 v = halves(act_value2(act, pair(z[i], W > 1 ? z[(i + 1) % W] : 0.f)));
            z[i] = v.x;
            if (W > 1) z[(i + 1) % W] = v.y;
        }
    }
}
// z becomes act'(z)
template <typename E, int W>
__device__ __forceinline__ void act_slope(int act, float* z) {
    if (std::is_same<E, float>::value) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if (act == FLAREPP_ACT_NONE) z[i] = 1.f;
            else if (act == FLAREPP_ACT_RELU) z[i] = z[i] > 0.f ? 1.f : 0.f;
            else if (act == FLAREPP_ACT_GELU)
                z[i] = normcdff(z[i]) + z[i] * 0.39894228f * expf(-0.5f * z[i] * z[i]);
            else {
                const float s = 1.f / (1.f + expf(-z[i]));
                z[i] = s * (1.f + z[i] * (1.f - s));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; i += 2) {
            const float2 v = halves(act_slope2(act, pair(z[i], W > 1 ? z[(i + 1) % W] : 0.f)));
            z[i] = v.x;
            if (W > 1) z[(i + 1) % W] = v.y;
        }
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
// Bound by reading X once: 8 rows of 16 bytes in flight a thread.
template <typename E, int W>
__global__ void __launch_bounds__(kThreads) stats_kernel(const Norm p) {
    __shared__ float sm[2][kThreads * W];
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
#pragma unroll
        for (int i = 0; i < W; ++i) {
            sm[0][a.ty * p.tc + a.c - a.c0 + i] = mean[i];
            sm[1][a.ty * p.tc + a.c - a.c0 + i] = sq[i];
        }
    }
    __syncthreads();
    // a warp takes a group: the mean of the means, then the squares about it
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int g = a.c0 / p.w + warp; g * p.w < a.c1; g += kThreads / 32) {
        int from, to;
        segment(p, g, a.c0, a.c1, from, to);
        const int width = to - from;
        float n = 0.f, m = 0.f;
        for (int e = lane; e < width * p.ty; e += 32) {
            const int y = e / width, at = y * p.tc + from - a.c0 + e - y * width;
            const float k = (float)rows_of(rows, y, p.ty);
            n += k;
            m = fmaf(k, sm[0][at], m);
        }
        n = warp_sum(n);
        m = warp_sum(m);
        m = n > 0.f ? m / n : 0.f;
        float s = 0.f;
        for (int e = lane; e < width * p.ty; e += 32) {
            const int y = e / width, at = y * p.tc + from - a.c0 + e - y * width;
            const float d = sm[0][at] - m;
            s += fmaf(d * d, (float)rows_of(rows, y, p.ty), sm[1][at]);
        }
        s = warp_sum(s);
        if (lane == 0) *slot(p, b, chunk, g, a.tile) = make_float2(m, s);
    }
}

// The chunks' parts of group g of sample b, joined by a warp: (mean, 1 / deviation).
__device__ __forceinline__ float2 join_stats(const Norm& p, int64_t b, int g, int live, int lane) {
    const int first = g * p.w / p.tc, segs = ((g + 1) * p.w - 1) / p.tc - first + 1;
    const float2* part = p.part + (b * p.chunks * p.G + g) * (int64_t)p.segs;
    const int64_t step = (int64_t)p.G * p.segs;
    float n = 0.f, m = 0.f;
    for (int e = lane; e < p.chunks * segs; e += 32) {
        const int k = e / segs, s = e - k * segs;
        int from, to;
        segment(p, g, (first + s) * p.tc, (first + s + 1) * p.tc, from, to);
        const float c = (float)max(0, min(live - k * p.rows, p.rows)) * (to - from);
        n += c;
        m = fmaf(c, part[k * step + s].x, m);
    }
    n = warp_sum(n);
    m = warp_sum(m);
    m = n > 0.f ? m / n : 0.f;
    float q = 0.f;
    for (int e = lane; e < p.chunks * segs; e += 32) {
        const int k = e / segs, s = e - k * segs;
        int from, to;
        segment(p, g, (first + s) * p.tc, (first + s + 1) * p.tc, from, to);
        const float c = (float)max(0, min(live - k * p.rows, p.rows)) * (to - from);
        const float2 v = part[k * step + s];
        const float d = v.x - m;
        q += fmaf(d * d, c, v.y);
    }
    q = warp_sum(q);
    return make_float2(m, rsqrtf((n > 0.f ? q / n : 0.f) + p.eps));
}

// ------------------------------------------------------------------ the forward's second pass
template <typename E, int W>
__global__ void __launch_bounds__(kThreads) apply_kernel(const Norm p) {
    __shared__ float2 sm[kThreads * W];  // of the tile's groups
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, gridDim.x - 1 - (int64_t)blockIdx.x);
    const int64_t b = p.b0 + a.unit / p.chunks;
    const int chunk = a.unit % p.chunks;
    const int live = live_rows(p, b);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g0 = a.c0 / p.w;
    for (int g = g0 + warp; g * p.w < a.c1; g += kThreads / 32) {
        const float2 v = join_stats(p, b, g, live, lane);
        if (lane == 0) {
            sm[g - g0] = v;
            if (p.stats && chunk == 0 && g * p.w >= a.c0) {
                p.stats[b * 2 * p.G + g] = v.x;
                p.stats[(b * 2 + 1) * p.G + g] = v.y;
            }
        }
    }
    __syncthreads();
    if (!a.on) return;
    float m[W], f[W], s[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 v = sm[(a.c + i) / p.w - g0];
        m[i] = v.x;
        f[i] = v.y * param(p.gamma, p.param_f32, a.c + i, 1.f);
        s[i] = param(p.beta, p.param_f32, a.c + i, 0.f);
    }
    const int r0 = chunk * p.rows, r1 = (int)min(p.N, (int64_t)r0 + p.rows);
    const int64_t at = (b * p.N + r0 + a.ty) * p.C + a.c, step = (int64_t)p.ty * p.C;
    const E* x = (const E*)p.x + at;
    E* y = (E*)p.y + at;
    const int all = rows_of(r1 - r0, a.ty, p.ty), mine = rows_of(max(0, live - r0), a.ty, p.ty);
    constexpr int U = 4;
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
            for (int i = 0; i < W; ++i) z[i] = k + j < mine ? fmaf(widen(v[j].v[i]) - m[i], f[i], s[i]) : 0.f;
            if (k + j < mine) act_value<E, W>(p.act, z);
#pragma unroll
            for (int i = 0; i < W; ++i) narrow(v[j].v[i], z[i]);
            store<E, W>(y + j * step, v[j]);
        }
    }
}

// ------------------------------------------------------------------ the backward
// A thread's channels: xhat = (x - m) r, z = gamma xhat + beta.
template <int W>
struct Channels {
    float r[W], m[W], gamma[W], beta[W];
};
template <int W>
__device__ __forceinline__ void params_of(const Norm& p, int c, Channels<W>& h) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        h.gamma[i] = param(p.gamma, p.param_f32, c + i, 1.f);
        h.beta[i] = param(p.beta, p.param_f32, c + i, 0.f);
    }
}
template <int W>
__device__ __forceinline__ void stats_of(const Norm& p, int64_t b, int c, Channels<W>& h) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int g = (c + i) / p.w;
        h.r[i] = p.stats[(b * 2 + 1) * p.G + g];
        h.m[i] = p.stats[b * 2 * p.G + g];
    }
}
// xhat and dz of a row's vector
template <typename E, int W>
__device__ __forceinline__ void row_of(const Norm& p, const Channels<W>& h, const Pack<E, W>& x,
                                       const Pack<E, W>& dy, float* xhat, float* dz) {
#pragma unroll
    for (int i = 0; i < W; ++i) xhat[i] = (widen(x.v[i]) - h.m[i]) * h.r[i];
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
template <typename E, int W>
__global__ void __launch_bounds__(kThreads) back_sums_kernel(const Norm p) {
    __shared__ float sm[2][kThreads * W];
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, blockIdx.x);
    const int64_t from_b = p.b0 + (p.chunks > 1 ? a.unit / p.chunks : (int64_t)a.unit * p.per);
    const int64_t to_b = p.chunks > 1 ? from_b + 1 : min((int64_t)p.b0 + p.bn, from_b + p.per);
    const int chunk = p.chunks > 1 ? a.unit % p.chunks : 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Channels<W> h;
    float all_u[W], all_v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) all_u[i] = all_v[i] = 0.f;
    if (a.on) params_of<W>(p, a.c, h);
    for (int64_t b = from_b; b < to_b; ++b) {
        const int live = live_rows(p, b);
        const int r0 = chunk * p.rows, rows = max(0, min(live, r0 + p.rows) - r0);
        float u[W], v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) u[i] = v[i] = 0.f;
        if (a.on) {
            stats_of<W>(p, b, a.c, h);
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
                        row_of<E, W>(p, h, px[j], pd[j], xhat, dz);
#pragma unroll
                        for (int i = 0; i < W; ++i) {
                            u[i] = fmaf(dz[i], xhat[i], u[i]);
                            v[i] += dz[i];
                        }
                    }
            }
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int at_s = a.ty * p.tc + a.c - a.c0 + i;
                sm[0][at_s] = v[i] * h.gamma[i];
                sm[1][at_s] = u[i] * h.gamma[i];
                all_u[i] += u[i];
                all_v[i] += v[i];
            }
        }
        __syncthreads();
        for (int g = a.c0 / p.w + warp; g * p.w < a.c1; g += kThreads / 32) {
            int from, to;
            segment(p, g, a.c0, a.c1, from, to);
            const int width = to - from;
            float s0 = 0.f, s1 = 0.f;
            for (int e = lane; e < width * p.ty; e += 32) {
                const int y = e / width, at = y * p.tc + from - a.c0 + e - y * width;
                s0 += sm[0][at];
                s1 += sm[1][at];
            }
            s0 = warp_sum(s0);
            s1 = warp_sum(s1);
            if (lane == 0) *slot(p, b, chunk, g, a.tile) = make_float2(s0, s1);
        }
        __syncthreads();
    }
    if (!p.channels) return;
    if (a.on)
#pragma unroll
        for (int i = 0; i < W; ++i) {
            sm[0][a.ty * p.tc + a.c - a.c0 + i] = all_u[i];
            sm[1][a.ty * p.tc + a.c - a.c0 + i] = all_v[i];
        }
    __syncthreads();
    float2* out = p.channels + (int64_t)(p.channel_rows + a.unit) * p.C;
    for (int c = a.c0 + threadIdx.x; c < a.c1; c += kThreads) {
        float s0 = 0.f, s1 = 0.f;
        for (int y = 0; y < p.ty; ++y) {
            s0 += sm[0][y * p.tc + c - a.c0];
            s1 += sm[1][y * p.tc + c - a.c0];
        }
        out[c] = make_float2(s0, s1);
    }
}

template <typename E, int W>
__global__ void __launch_bounds__(kThreads) back_apply_kernel(const Norm p) {
    __shared__ float2 sm[kThreads * W];
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, gridDim.x - 1 - (int64_t)blockIdx.x);
    const int64_t b = p.b0 + a.unit / p.chunks;
    const int chunk = a.unit % p.chunks;
    const int live = live_rows(p, b);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g0 = a.c0 / p.w;
    const float each = 1.f / fmaxf(1.f, (float)live * p.w);
    for (int g = g0 + warp; g * p.w < a.c1; g += kThreads / 32) {
        const int first = g * p.w / p.tc, segs = ((g + 1) * p.w - 1) / p.tc - first + 1;
        const float2* part = p.part + (b * p.chunks * p.G + g) * (int64_t)p.segs;
        float s0 = 0.f, s1 = 0.f;
        for (int e = lane; e < p.chunks * segs; e += 32) {
            const int k = e / segs;
            const float2 v = part[k * (int64_t)p.G * p.segs + e - k * segs];
            s0 += v.x;
            s1 += v.y;
        }
        s0 = warp_sum(s0);
        s1 = warp_sum(s1);
        if (lane == 0) sm[g - g0] = make_float2(s0 * each, s1 * each);
    }
    __syncthreads();
    if (!a.on) return;
    Channels<W> h;
    params_of<W>(p, a.c, h);
    stats_of<W>(p, b, a.c, h);
    float m0[W], m1[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
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
                row_of<E, W>(p, h, px[j], pd[j], xhat, dz);
#pragma unroll
                for (int i = 0; i < W; ++i)
                    dz[i] = h.r[i] * (fmaf(dz[i], h.gamma[i], -m0[i]) - xhat[i] * m1[i]);
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

// dgamma and dbeta from rows [R][C] of (sum dz xhat, sum dz): a block takes 32 channels, its 32 warps every
// 32nd row, in order; then the warps' sums in order.
constexpr int kReduceThreads = 1024;
template <typename P>
__global__ void __launch_bounds__(kReduceThreads)
    channels_kernel(const float2* rows, int R, int C, P* dgamma, P* dbeta) {
    __shared__ float2 sm[32][33];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float2 s = make_float2(0.f, 0.f);
    if (c < C)
        for (int r = warp; r < R; r += 32) {
            const float2 v = rows[(int64_t)r * C + c];
            s.x += v.x;
            s.y += v.y;
        }
    sm[warp][lane] = s;
    __syncthreads();
    if (warp || c >= C) return;
    for (int k = 1; k < 32; ++k) {
        s.x += sm[k][lane].x;
        s.y += sm[k][lane].y;
    }
    if (dgamma) narrow(dgamma[c], s.x);
    if (dbeta) narrow(dbeta[c], s.y);
}

// ------------------------------------------------------------------ few rows a sample
// A group's w channels are the vectors of `lanes` lanes (a power of two), a sample's K rows stay in their
// registers: one pass over the data and one launch. Blocks walk the samples.
template <typename E, int W, int K>
__global__ void __launch_bounds__(kThreads) few_kernel(const Norm p, int lanes) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, blockIdx.x);
    float f[W], s[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        f[i] = a.on ? param(p.gamma, p.param_f32, a.c + i, 1.f) : 0.f;
        s[i] = a.on ? param(p.beta, p.param_f32, a.c + i, 0.f) : 0.f;
    }
    const int64_t step = gridDim.x / p.tiles * (int64_t)p.ty;
    const int64_t turns = (p.B + step - 1) / step;
    for (int64_t t = 0; t < turns; ++t) {  // all lanes take part in the sums
        const int64_t b = t * step + (int64_t)a.unit * p.ty + a.ty;
        const bool on = a.on && b < p.B;
        int live = 0;
        if (on) {
            live = (int)p.N;
            if (p.lengths) {
                live = p.lengths[b];
                if (live < 0 || live > p.N) {
                    record_status(p.status, FLAREPP_ERR_INVALID_ARGUMENT);
                    live = live < 0 ? 0 : (int)p.N;
                }
            }
        }
        const int64_t at = b * p.N * p.C + a.c;
        Pack<E, W> x[K];
        float m = 0.f, q = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < live) {
                x[k] = load<E, W>((const E*)p.x + at + (int64_t)k * p.C);
#pragma unroll
                for (int i = 0; i < W; ++i) m += widen(x[k].v[i]);
            }
        const float each = 1.f / fmaxf(1.f, (float)live * p.w);
        m = warp_sum(m, lanes) * each;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < live)
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float d = widen(x[k].v[i]) - m;
                    q = fmaf(d, d, q);
                }
        q = rsqrtf(warp_sum(q, lanes) * each + p.eps);
        if (!on) continue;
        if (p.stats && a.c % p.w == 0) {
            p.stats[b * 2 * p.G + a.c / p.w] = m;
            p.stats[(b * 2 + 1) * p.G + a.c / p.w] = q;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k >= p.N) break;
            float z[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                z[i] = k < live ? fmaf(widen(x[k].v[i]) - m, q * f[i], s[i]) : 0.f;
            }
            if (k < live) act_value<E, W>(p.act, z);
#pragma unroll
            for (int i = 0; i < W; ++i) narrow(x[k].v[i], z[i]);
            store<E, W>((E*)p.y + at + (int64_t)k * p.C, x[k]);
        }
    }
}

template <typename E, int W, int K>
__global__ void __launch_bounds__(kThreads) back_few_kernel(const Norm p, int lanes) {
    __shared__ float sm[2][kThreads * W];
    tc::pdl_trigger();
    tc::pdl_wait();
    const Place a = place_of<W>(p, blockIdx.x);
    Channels<W> h;
    float u[W], v[W];
#pragma unroll
    for (int i = 0; i < W; ++i) u[i] = v[i] = h.r[i] = h.m[i] = h.gamma[i] = h.beta[i] = 0.f;
    if (a.on) params_of<W>(p, a.c, h);
    const int64_t step = gridDim.x / p.tiles * (int64_t)p.ty;
    const int64_t turns = (p.B + step - 1) / step;
    for (int64_t t = 0; t < turns; ++t) {
        const int64_t b = t * step + (int64_t)a.unit * p.ty + a.ty;
        const bool on = a.on && b < p.B;
        int live = 0;
        if (on) {
            live = (int)p.N;
            if (p.lengths) {
                live = p.lengths[b];
                if (live < 0 || live > p.N) {
                    record_status(p.status, FLAREPP_ERR_INVALID_ARGUMENT);
                    live = live < 0 ? 0 : (int)p.N;
                }
            }
            stats_of<W>(p, b, a.c, h);
        }
        const int64_t at = b * p.N * p.C + a.c;
        Pack<E, W> x[K], dy[K];
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < live) {
                x[k] = load<E, W>((const E*)p.x + at + (int64_t)k * p.C);
                dy[k] = load<E, W>((const E*)p.dy + at + (int64_t)k * p.C);
            }
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k < live) {
                float xhat[W], dz[W];
                row_of<E, W>(p, h, x[k], dy[k], xhat, dz);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    u[i] = fmaf(dz[i], xhat[i], u[i]);
                    v[i] += dz[i];
                    const float g = dz[i] * h.gamma[i];
                    s0 += g;
                    s1 = fmaf(g, xhat[i], s1);
                }
            }
        const float each = 1.f / fmaxf(1.f, (float)live * p.w);
        s0 = warp_sum(s0, lanes) * each;
        s1 = warp_sum(s1, lanes) * each;
        if (!on) continue;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (k >= p.N) break;
            float xhat[W], dz[W];
            if (k < live) {
                row_of<E, W>(p, h, x[k], dy[k], xhat, dz);
#pragma unroll
                for (int i = 0; i < W; ++i)
                    dz[i] = h.r[i] * (fmaf(dz[i], h.gamma[i], -s0) - xhat[i] * s1);
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) dz[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) narrow(x[k].v[i], dz[i]);
            store<E, W>((E*)p.y + at + (int64_t)k * p.C, x[k]);
        }
    }
    if (!p.channels) return;
    if (a.on)
#pragma unroll
        for (int i = 0; i < W; ++i) {
            sm[0][a.ty * p.tc + a.c - a.c0 + i] = u[i];
            sm[1][a.ty * p.tc + a.c - a.c0 + i] = v[i];
        }
    __syncthreads();
    float2* out = p.channels + (int64_t)a.unit * p.C;
    for (int c = a.c0 + threadIdx.x; c < a.c1; c += kThreads) {
        float s0 = 0.f, s1 = 0.f;
        for (int y = 0; y < p.ty; ++y) {
            s0 += sm[0][y * p.tc + c - a.c0];
            s1 += sm[1][y * p.tc + c - a.c0];
        }
        out[c] = make_float2(s0, s1);
    }
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
    int W, tx, ty, tc, tiles, segs;
    int lanes;        // > 0: few rows, groups of that many lanes
    int chunks, rows, per;
    int64_t group;    // samples that go through together
    int64_t units;    // rows of `channels` that a call leaves
    size_t off_channels, total;
};

int64_t elem_of(const flarepp_norm_shape& s) { return s.dtype == FLAREPP_BF16 ? 2 : 4; }

Plan plan_of(const flarepp_norm_shape& s, bool backward) {
    Plan p{};
    const int64_t e = elem_of(s);
    p.W = (int)(16 / e);
    while (s.C % p.W) p.W /= 2;
    const int64_t vectors = s.C / p.W, w = s.C / s.G;
    // Few rows: the groups' lanes must divide a warp. (A sample of one row and 512 channels: 1 launch.)
    if (s.N <= kFewRows && w % p.W == 0) {
        const int64_t lanes = w / p.W;
        if (lanes <= 32 && (lanes & (lanes - 1)) == 0) p.lanes = (int)lanes;
    }
    // tiles as even as can be, of whole groups' lanes where they matter
    p.tiles = (int)cdiv(vectors, kThreads);
    p.tx = (int)cdiv(vectors, p.tiles);
    if (p.lanes) p.tx = (int)cdiv(p.tx, p.lanes) * p.lanes;
    p.tiles = (int)cdiv(vectors, p.tx);
    p.ty = kThreads / p.tx;
    p.tc = p.tx * p.W;
    // the most tiles that w channels side by side can touch
    p.segs = (int)(w < 2 ? 1 : (w - 2) / p.tc + 2);
    if (p.segs > p.tiles) p.segs = p.tiles;
    p.per = 1;
    if (p.lanes) {
        p.units = cdiv(s.B, p.ty);
        const int64_t most = cdiv(kNumSMs * 4, p.tiles);
        if (p.units > most) p.units = most;
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
        const int64_t wanted = cdiv(kNumSMs * 6, p.group * p.tiles);
        const int64_t least = (int64_t)p.ty * kRows;  // rows that keep a block's threads busy
        p.chunks = (int)(wanted < cdiv(s.N, least) ? wanted : cdiv(s.N, least));
        if (p.chunks < 1) p.chunks = 1;
        p.rows = (int)cdiv(s.N, p.chunks);
        p.chunks = (int)cdiv(s.N, p.rows);
        if (p.chunks == 1) {
            const int64_t blocks = cdiv(kNumSMs * 6, p.tiles);
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

template <typename E, int W>
cudaError_t forward(Norm a, const Plan& p, cudaStream_t st) {
    if (p.lanes) {
        const int64_t blocks = p.units * p.tiles;
        return a.N == 1 ? launch(few_kernel<E, W, 1>, blocks, kThreads, st, a, p.lanes)
                        : launch(few_kernel<E, W, kFewRows>, blocks, kThreads, st, a, p.lanes);
    }
    for (int64_t b = 0; b < a.B; b += p.group) {
        a.b0 = (int)b;
        a.bn = (int)(a.B - b < p.group ? a.B - b : p.group);
        const int64_t blocks = (int64_t)a.bn * p.chunks * p.tiles;
        cudaError_t e = launch(stats_kernel<E, W>, blocks, kThreads, st, a);
        if (e == cudaSuccess) e = launch(apply_kernel<E, W>, blocks, kThreads, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename E, int W>
cudaError_t backward(Norm a, const Plan& p, cudaStream_t st) {
    if (p.lanes) {
        const int64_t blocks = p.units * p.tiles;
        a.channel_rows = 0;
        return a.N == 1 ? launch(back_few_kernel<E, W, 1>, blocks, kThreads, st, a, p.lanes)
                        : launch(back_few_kernel<E, W, kFewRows>, blocks, kThreads, st, a, p.lanes);
    }
    int rows = 0;
    for (int64_t b = 0; b < a.B; b += p.group) {
        a.b0 = (int)b;
        a.bn = (int)(a.B - b < p.group ? a.B - b : p.group);
        a.channel_rows = rows;
        const int64_t units = p.chunks > 1 ? (int64_t)a.bn * p.chunks : cdiv(a.bn, p.per);
        rows += (int)units;
        cudaError_t e = launch(back_sums_kernel<E, W>, units * p.tiles, kThreads, st, a);
        if (e == cudaSuccess)
            e = launch(back_apply_kernel<E, W>, (int64_t)a.bn * p.chunks * p.tiles, kThreads, st, a);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename E>
cudaError_t run(bool back, const Norm& a, const Plan& p, cudaStream_t st) {
    constexpr int M = 16 / sizeof(E);
    switch (p.W) {
        case M: return back ? backward<E, M>(a, p, st) : forward<E, M>(a, p, st);
        case M / 2: return back ? backward<E, M / 2>(a, p, st) : forward<E, M / 2>(a, p, st);
        case 2: return back ? backward<E, 2>(a, p, st) : forward<E, 2>(a, p, st);
        default: return back ? backward<E, 1>(a, p, st) : forward<E, 1>(a, p, st);
    }
}
template <>
cudaError_t run<float>(bool back, const Norm& a, const Plan& p, cudaStream_t st) {
    switch (p.W) {
        case 4: return back ? backward<float, 4>(a, p, st) : forward<float, 4>(a, p, st);
        case 2: return back ? backward<float, 2>(a, p, st) : forward<float, 2>(a, p, st);
        default: return back ? backward<float, 1>(a, p, st) : forward<float, 1>(a, p, st);
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
    const Plan p = plan_of(s, back);
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
    a.tx = p.tx, a.ty = p.ty, a.tc = p.tc, a.tiles = p.tiles, a.segs = p.segs;
    a.chunks = p.chunks, a.rows = p.rows, a.per = p.per;
    a.part = (float2*)workspace;
    a.channels = sums ? (float2*)((char*)workspace + p.off_channels) : nullptr;
    e = s.dtype == FLAREPP_BF16 ? run<__nv_bfloat16>(back, a, p, st) : run<float>(back, a, p, st);
    if (e == cudaSuccess && sums) {
        const int64_t blocks = cdiv(s.C, 32);
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
