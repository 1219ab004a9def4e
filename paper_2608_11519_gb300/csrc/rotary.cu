// Rotary positions with several axes (flarepp_rotary): pairs of a head's channels, (x, y), turned by the
// angle position[axis of the pair] * freq[pair],
//   x' = x cos - y sin,  y' = y cos + x sin   (the inverse, which is also the gradient's: sin negated).
//
// Bound by bytes: each value is read and written once; a head's values take one multiply-add pair each,
// and a position's sines and cosines, some 40 instructions a pair of channels, serve all heads of q and
// k, which one thread walks.
//
// The angle. Far positions leave no bits of position * freq behind the point in 32 bits (10^6 rad has
// a unit of 0.06), so it is taken in turns as a sum of products whose rounding errors are kept (each by
// a fused multiply-add) and whose whole turns are dropped one by one: freq / (2 pi) in three floats, the
// position in two (an int32 has 31 bits). What is left is off by a few 2^-25 turns, whatever
// the position.
#include <cuda_runtime.h>
#include <math.h>

#include "checks.h"
#include "flarepp_internal.h"
#include "heads.h"
#include "tc_ptx.cuh"
#include "vectors.cuh"

namespace flarepp {
namespace {

using namespace vec;

constexpr int kThreads = 256;
constexpr int kMaxAxes = FLAREPP_ROTARY_AXES;
constexpr int64_t kMaxDim = 1024;

struct Side {  // one of q and k
    const void* x;
    void* y;
    int64_t xb, xh, xn, yb, yh, yn;
};

struct Rotary {
    Side side[2];
    int Hq, H;  // heads of q; of q and k together
    int64_t B, N;
    int D, P;       // channels, pairs
    int ends[kMaxAxes];  // pairs up to each axis's last
    int axes, pairing;
    int per;        // heads that a thread walks
    int copies;     // whether channels that no pair holds are copied
    float sign;
    const void* positions;
    int64_t pos_stride;
    int real;       // positions are floats
    const float* freqs;
};

__device__ __forceinline__ float fraction(float x) { return x - rintf(x); }

// cos and sin of (p + q) f, p and q floats
__device__ __forceinline__ void turn_of(float p, float q, float f, float& c, float& s) {
    const float kHi = 0.159154937f, kLo = 6.42063824e-09f, kLast = 7.3427387e-17f;  // 1 / (2 pi)
    const float f0 = f * kHi, rest = fmaf(f, kHi, -f0), f1 = fmaf(f, kLo, rest);
    const float f2 = fmaf(f, kLast, fmaf(f, kLo, rest - f1));
    const float m = p * f0, n = q * f0, l = p * f1;
    const float r = fraction(m) + fraction(fmaf(p, f0, -m)) + fraction(n) + fraction(l) +
                    (fmaf(q, f0, -n) + fmaf(p, f1, -l) + p * f2 + q * f1);
    sincospif(2.f * fraction(r), &s, &c);
}

// The position of row n in two floats
__device__ __forceinline__ void position(const Rotary& a, int64_t b, int64_t n, int axis, float& p,
                                         float& q) {
    const int64_t at = b * a.pos_stride + n * a.axes + axis;
    if (a.real) {
        p = ((const float*)a.positions)[at];
        q = 0.f;
    } else {
        const int i = ((const int*)a.positions)[at];
        p = (float)i;
        q = (float)((int64_t)i - (int64_t)p);
    }
}

__device__ __forceinline__ int axis_of(const Rotary& a, int pair) {
    int k = 0;
    while (k < a.axes - 1 && pair >= a.ends[k]) ++k;
    return k;
}

__device__ __forceinline__ const Side& side_of(const Rotary& a, int h, int& local) {
    const bool k = h >= a.Hq;
    local = k ? h - a.Hq : h;
    return a.side[k];
}

// A thread holds W pairs (two vectors of W channels, or with W = 1 two channels) of a token, or a vector
// of channels that no pair holds, for `per` heads, four of them in flight. Pairs whose channels lie apart:
// channels first and second; adjacent ones: 2 W channels side by side.
template <typename E, int W>
__global__ void __launch_bounds__(kThreads) pairs_kernel(const Rotary a) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int blocks = a.P / W, units = blocks + (a.copies ? (a.D - 2 * a.P) / W : 0);
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (id >= a.B * a.N * units) return;
    const int64_t row = id / units;
    const int unit = (int)(id - row * units);
    const int64_t b = row / a.N, n = row - b * a.N;
    const int h0 = blockIdx.y * a.per, h1 = min(a.H, h0 + a.per);
    if (unit >= blocks) {
        const int c = 2 * a.P + (unit - blocks) * W;
        for (int h = h0; h < h1; ++h) {
            int hh;
            const Side& s = side_of(a, h, hh);
            store<E, W>((E*)s.y + b * s.yb + hh * s.yh + n * s.yn + c,
                        load<E, W>((const E*)s.x + b * s.xb + hh * s.xh + n * s.xn + c));
        }
        return;
    }
    const int p0 = unit * W;
    int first = 2 * p0, second = 2 * p0 + W;
    const bool adjacent = a.pairing == FLAREPP_ROTARY_ADJACENT;
    if (a.pairing == FLAREPP_ROTARY_HALVES) first = p0, second = p0 + a.P;
    if (a.pairing == FLAREPP_ROTARY_AXES_APART) {
        const int k = axis_of(a, p0), start = k ? a.ends[k - 1] : 0;
        first = p0 + start;
        second = first + a.ends[k] - start;
    }
    if (adjacent && W == 1) second = first + 1;
    float cs[W], sn[W];
    int held = -1;
    float p = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int k = axis_of(a, p0 + i);
        if (k != held) position(a, b, n, held = k, p, q);
        turn_of(p, q, a.freqs[p0 + i], cs[i], sn[i]);
        sn[i] *= a.sign;
    }
    constexpr int kFlight = 4;
    for (int h = h0; h < h1; h += kFlight) {
        Pack<E, W> u[kFlight], v[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (h + j < h1) {
                int hh;
                const Side& s = side_of(a, h + j, hh);
                const E* x = (const E*)s.x + b * s.xb + hh * s.xh + n * s.xn;
                u[j] = load<E, W>(x + first);
                v[j] = load<E, W>(x + second);
            }
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (h + j < h1) {
                int hh;
                const Side& s = side_of(a, h + j, hh);
                if (adjacent && W > 1) {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        E& ex = i < W / 2 ? u[j].v[2 * i % W] : v[j].v[2 * i % W];
                        E& ey = i < W / 2 ? u[j].v[(2 * i + 1) % W] : v[j].v[(2 * i + 1) % W];
                        const float x = widen(ex), y = widen(ey);
                        narrow(ex, x * cs[i] - y * sn[i]);
                        narrow(ey, y * cs[i] + x * sn[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float x = widen(u[j].v[i]), y = widen(v[j].v[i]);
                        narrow(u[j].v[i], x * cs[i] - y * sn[i]);
                        narrow(v[j].v[i], y * cs[i] + x * sn[i]);
                    }
                }
                E* o = (E*)s.y + b * s.yb + hh * s.yh + n * s.yn;
                store<E, W>(o + first, u[j]);
                store<E, W>(o + second, v[j]);
            }
    }
}

// Pairs that no vector divides (sections of 6, 5 and 5, say): a thread holds a vector of a token's channels
// as they lie, and their partners come through shared memory, four heads at a time. On a mesh of a million
// points and 16 heads of 32 channels the channels one by one would be 2-byte accesses.
template <typename E, int W>
__global__ void __launch_bounds__(kThreads) rows_kernel(const Rotary a, int tokens) {
    tc::pdl_trigger();
    tc::pdl_wait();
    constexpr int kFlight = 4;
    __shared__ __align__(16) E stage[2][kFlight][kThreads * W];
    const int vectors = a.D / W, t = threadIdx.x;
    const int token = t / vectors, c0 = (t - token * vectors) * W;
    const int64_t row = (int64_t)blockIdx.x * tokens + token;
    const bool live = token < tokens && row < a.B * a.N;
    const int64_t b = live ? row / a.N : 0, n = live ? row - b * a.N : 0;
    const int h0 = blockIdx.y * a.per, h1 = min(a.H, h0 + a.per);
    float cs[W], sn[W];  // a channel's own: its value times cs plus its partner's times sn
    int other[W];        // where its partner lies in a stage
    const int rows = token * a.D;
    {
        int held = -1;
        float p = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const int c = c0 + i;
            cs[i] = 1.f;
            sn[i] = 0.f;
            other[i] = rows + c;
            if (!live || c >= 2 * a.P) continue;
            int pair, partner;
            float sign = -a.sign;
            if (a.pairing == FLAREPP_ROTARY_HALVES) {
                pair = c < a.P ? c : c - a.P;
                partner = c < a.P ? c + a.P : c - a.P;
                if (c >= a.P) sign = a.sign;
            } else if (a.pairing == FLAREPP_ROTARY_ADJACENT) {
                pair = c >> 1;
                partner = c ^ 1;
                if (c & 1) sign = a.sign;
            } else {
                int k = 0;
                while (k < a.axes - 1 && c >= 2 * a.ends[k]) ++k;
                const int start = k ? a.ends[k - 1] : 0, size = a.ends[k] - start;
                const bool low = c - 2 * start < size;
                pair = low ? c - start : c - start - size;
                partner = low ? c + size : c - size;
                if (!low) sign = a.sign;
            }
            const int k = axis_of(a, pair);
            if (k != held) position(a, b, n, held = k, p, q);
            turn_of(p, q, a.freqs[pair], cs[i], sn[i]);
            sn[i] *= sign;
            other[i] = rows + partner;
        }
    }
    int buf = 0;
    for (int h = h0; h < h1; h += kFlight, buf ^= 1) {
        Pack<E, W> u[kFlight];
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (live && h + j < h1) {
                int hh;
                const Side& s = side_of(a, h + j, hh);
                u[j] = load<E, W>((const E*)s.x + b * s.xb + hh * s.xh + n * s.xn + c0);
            }
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (live && h + j < h1) store<E, W>(&stage[buf][j][rows + c0], u[j]);
        __syncthreads();  // the stage before is read by all once this one is passed
#pragma unroll
        for (int j = 0; j < kFlight; ++j)
            if (live && h + j < h1) {
                int hh;
                const Side& s = side_of(a, h + j, hh);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const float x = widen(u[j].v[i]), y = widen(stage[buf][j][other[i]]);
                    if (other[i] != rows + c0 + i) narrow(u[j].v[i], x * cs[i] + y * sn[i]);
                }
                store<E, W>((E*)s.y + b * s.yb + hh * s.yh + n * s.yn + c0, u[j]);
            }
    }
}

template <typename... Args>
cudaError_t launch(void (*kernel)(Args...), dim3 grid, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Heads for a thread to walk: all of them would spare sines, but a thread's loads are a few in flight, so
// as many threads as the card holds (2,048 a SM) come first.
int heads_per_thread(int64_t threads, int heads) {
    const int64_t full = (int64_t)kNumSMs * 2048;
    int64_t groups = cdiv(2 * full, threads > 0 ? threads : 1);
    if (groups > heads) groups = heads;
    int per = (int)cdiv(heads, groups);
    if (per > 4) per = (int)cdiv(per, 4) * 4;
    return per;
}

template <typename E>
cudaError_t enqueue(Rotary a, bool whole, bool pairs_whole, cudaStream_t st) {
    constexpr int W = 16 / sizeof(E);
    const int64_t rows = a.B * a.N;
    if (whole && !pairs_whole) {
        const int tokens = kThreads / (a.D / W);
        const int64_t blocks = cdiv(rows, tokens);
        a.per = heads_per_thread(blocks * kThreads, a.H);
        if (blocks > INT32_MAX) return cudaErrorInvalidValue;
        return launch(rows_kernel<E, W>, dim3((unsigned)blocks, (unsigned)cdiv(a.H, a.per)), st, a,
                      tokens);
    }
    const int w = whole ? W : 1;
    const int units = a.P / w + (a.copies ? (a.D - 2 * a.P) / w : 0);
    if (units == 0) return cudaSuccess;
    const int64_t blocks = cdiv(rows * units, kThreads);
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    a.per = heads_per_thread(blocks * kThreads, a.H);
    const dim3 grid((unsigned)blocks, (unsigned)cdiv(a.H, a.per));
    return whole ? launch(pairs_kernel<E, W>, grid, st, a) : launch(pairs_kernel<E, 1>, grid, st, a);
}

// One side's tensors: FLAREPP_OK, or what is wrong with them.
flarepp_status check_side(const HeadDims& d, const flarepp_heads* x, const flarepp_heads* y) {
    if (!x || !y) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (empty(d)) return FLAREPP_OK;
    if (!x->data || !y->data) return FLAREPP_ERR_INVALID_ARGUMENT;
    if ((uintptr_t)x->data % d.bytes || (uintptr_t)y->data % d.bytes) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!strides_ok(*x, d) || !strides_ok(*y, d)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!apart_within(*y, d)) return FLAREPP_ERR_INVALID_ARGUMENT;
    return FLAREPP_OK;
}

bool same(const flarepp_heads& x, const flarepp_heads& y) {
    return x.data == y.data && x.stride_b == y.stride_b && x.stride_h == y.stride_h &&
           x.stride_n == y.stride_n;
}

bool vectors_ok(const flarepp_heads& t, int64_t per) {
    return aligned16(t.data) && t.stride_b % per == 0 && t.stride_h % per == 0 && t.stride_n % per == 0;
}

flarepp_status rotary(const flarepp_rotary_shape* s, const void* positions, const float* freqs,
                      const flarepp_heads* q, const flarepp_heads* k, const flarepp_heads* q_out,
                      const flarepp_heads* k_out, cudaStream_t st) {
    if (!s) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->B < 0 || s->N < 0 || s->Hq < 0 || s->Hk < 0 || s->D < 1) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->dtype != FLAREPP_F32 && s->dtype != FLAREPP_BF16) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->axes < 1 || s->axes > kMaxAxes) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->pairing < FLAREPP_ROTARY_HALVES || s->pairing > FLAREPP_ROTARY_AXES_APART)
        return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->D > kMaxDim || s->Hq > 65535 || s->Hk > 65535 || s->B > INT32_MAX || s->N > INT32_MAX)
        return FLAREPP_ERR_UNSUPPORTED;
    Rotary a{};
    int64_t P = 0;
    for (int i = 0; i < s->axes; ++i) {
        if (s->sections[i] < 0 || s->sections[i] > s->D) return FLAREPP_ERR_INVALID_ARGUMENT;
        a.ends[i] = (int)(P += s->sections[i]);
    }
    if (2 * P > s->D) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->pos_stride_b < 0 || (s->B > 1 && s->pos_stride_b > (int64_t(1) << 47) / s->B))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const int64_t e = s->dtype == FLAREPP_BF16 ? 2 : 4;
    const flarepp_heads* in[2] = {q, k};
    const flarepp_heads* out[2] = {q_out, k_out};
    HeadDims d[2] = {{s->B, s->Hq, s->N, s->D, e}, {s->B, s->Hk, s->N, s->D, e}};
    for (int i = 0; i < 2; ++i) {
        if (d[i].H == 0) continue;
        const flarepp_status r = check_side(d[i], in[i], out[i]);
        if (r != FLAREPP_OK) return r;
    }
    if (s->B == 0 || s->N == 0 || s->Hq + s->Hk == 0) return FLAREPP_OK;
    if (P > 0 && (!positions || !freqs || !aligned4(positions) || !aligned4(freqs)))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const Span about[2] = {
        {positions, P > 0 ? (size_t)(((s->B - 1) * s->pos_stride_b + s->N * s->axes) * 4) : 0},
        {freqs, (size_t)P * 4}};
    for (int i = 0; i < 2; ++i) {
        if (d[i].H == 0) continue;
        const Span o = span_of(*out[i], d[i]);
        for (int j = 0; j < 2; ++j) {
            if (overlaps(o.p, o.bytes, about[j].p, about[j].bytes)) return FLAREPP_ERR_INVALID_ARGUMENT;
            if (d[j].H == 0) continue;
            if (!(i == j && same(*in[i], *out[i])) && !apart(*out[i], d[i], *in[j], d[j]))
                return FLAREPP_ERR_INVALID_ARGUMENT;
            if (j < i && !apart(*out[i], d[i], *out[j], d[j])) return FLAREPP_ERR_INVALID_ARGUMENT;
        }
    }
    a.B = s->B, a.N = s->N, a.D = (int)s->D, a.P = (int)P;
    a.Hq = (int)s->Hq, a.H = (int)(s->Hq + s->Hk);
    a.axes = s->axes, a.pairing = s->pairing;
    a.sign = s->inverse ? -1.f : 1.f;
    a.positions = positions, a.pos_stride = s->pos_stride_b, a.real = s->real_positions != 0;
    a.freqs = freqs;
    const int64_t per = 16 / e;
    bool whole = s->D % per == 0, in_place = true;
    for (int i = 0; i < 2; ++i) {
        if (d[i].H == 0) continue;
        whole = whole && vectors_ok(*in[i], per) && vectors_ok(*out[i], per);
        in_place = in_place && same(*in[i], *out[i]);
        a.side[i] = {in[i]->data,      out[i]->data,      in[i]->stride_b,  in[i]->stride_h,
                     in[i]->stride_n,  out[i]->stride_b,  out[i]->stride_h, out[i]->stride_n};
    }
    a.copies = !in_place && s->D > 2 * P;
    bool pairs_whole = P % per == 0;
    if (s->pairing == FLAREPP_ROTARY_AXES_APART)
        for (int i = 0; i < s->axes; ++i) pairs_whole = pairs_whole && s->sections[i] % per == 0;
    if (P == 0 && in_place) return FLAREPP_OK;
    const cudaError_t err = e == 2 ? enqueue<__nv_bfloat16>(a, whole, pairs_whole, st)
                                   : enqueue<float>(a, whole, pairs_whole, st);
    return err == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

}  // namespace
}  // namespace flarepp

extern "C" flarepp_status flarepp_rotary(const flarepp_rotary_shape* shape, const void* positions,
                                         const float* freqs, const flarepp_heads* q,
                                         const flarepp_heads* k, const flarepp_heads* q_out,
                                         const flarepp_heads* k_out, void* stream) {
    return flarepp::rotary(shape, positions, freqs, q, k, q_out, k_out, (cudaStream_t)stream);
}
