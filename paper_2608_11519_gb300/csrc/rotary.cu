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
// a fused multiply-add) and whose whole turns are dropped one by one: freq / (2 pi) in three floats (72 bits), the
// position in two (an int32 has 31 bits). What is left is off by four roundings of 2^-25 turns at most, 2^-20 rad
// with the sine's own, for any int32 position and real ones up to 2^40 rad. (With the third float rounded from the
// second one's rounded error, 51 bits in all, angles were off by 2^-17 rad at 2^31 and by 2^-9 at 2^40.)
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
constexpr int kMaxDim = 1024;

struct Side {  // one of q and k
    const void* x;
    void* y;
    int64_t xb, xh, xn, yb, yh, yn;
};

struct Rotary {
    Side side[2];
    int Hq, H;  // heads of q; of q and k together
    int rows, N;    // tokens of the batch, of an element
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

// f / (2 pi) as a sum of three floats. (The _rn forms are not contracted into multiply-adds.)
struct Turns {
    float hi, mid, lo;
};
__device__ __forceinline__ Turns turns_of(float f) {
    const float kHi = 0.159154937f, kLo = 6.42063824e-09f, kLast = 7.3427387e-17f;  // 1 / (2 pi)
    Turns t;
    t.hi = __fmul_rn(f, kHi);
    const float a = fmaf(f, kHi, -t.hi), b = __fmul_rn(f, kLo);
    t.mid = __fadd_rn(a, b);
    const float z = __fsub_rn(t.mid, b);  // what that sum leaves, exactly
    const float rest = __fadd_rn(__fsub_rn(b, __fsub_rn(t.mid, z)), __fsub_rn(a, z));
    t.lo = fmaf(f, kLast, __fadd_rn(rest, fmaf(f, kLo, -b)));
    return t;
}

// cos and sin of (p + q) f, p and q floats
__device__ __forceinline__ void turn_of(float p, float q, const Turns& f, float& c, float& s) {
    const float m = __fmul_rn(p, f.hi), n = __fmul_rn(q, f.hi), l = __fmul_rn(p, f.mid);
    const float r = fraction(fraction(m) + fraction(fmaf(p, f.hi, -m))) + fraction(fraction(n) + fraction(l));
    const float small = fmaf(q, f.hi, -n) + fmaf(p, f.mid, -l) + p * f.lo + q * f.mid;
    sincospif(2.f * fraction(r + small), &s, &c);
}

// The position of row n in two floats
__device__ __forceinline__ void position(const Rotary& a, int64_t b, int n, int axis, float& p,
                                         float& q) {
    const int64_t at = b * a.pos_stride + (int64_t)n * a.axes + axis;
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

// The part of one side's heads in [h0, h1): how many, and where the first one's row n of batch element b is.
template <typename E>
struct Rows {
    const E* x;
    E* y;
    int64_t xh, yh;
    int heads;
};
template <typename E>
__device__ __forceinline__ Rows<E> rows_on(const Rotary& a, int k, int64_t b, int64_t n, int h0, int h1) {
    const Side& s = a.side[k];
    const int first = k ? max(h0 - a.Hq, 0) : h0, last = k ? h1 - a.Hq : min(h1, a.Hq);
    Rows<E> r;
    r.heads = max(last - first, 0);
    r.xh = s.xh;
    r.yh = s.yh;
    r.x = (const E*)s.x + b * s.xb + first * s.xh + n * s.xn;
    r.y = (E*)s.y + b * s.yb + first * s.yh + n * s.yn;
    return r;
}

template <typename E, int W>
__device__ __forceinline__ void widen_all(const Pack<E, W>& v, float* x) {
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = widen(v.v[i]);
}
template <typename E>
__device__ __forceinline__ void narrow_all(Pack<E, 1>& v, const float* x) {
    narrow(v.v[0], x[0]);
}
__device__ __forceinline__ void narrow_all(Pack<float, 4>& v, const float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = x[i];
}
__device__ __forceinline__ void narrow_all(Pack<__nv_bfloat16, 8>& v, const float* x) {
#pragma unroll
    for (int i = 0; i < 8; i += 2)
        *reinterpret_cast<__nv_bfloat162*>(&v.v[i]) = __floats2bfloat162_rn(x[i], x[i + 1]);
}

// A thread holds W pairs (two vectors of W channels, or with W = 1 two channels) of a token, or a vector
// of channels that no pair holds, for `per` heads, four of them in flight. Pairs whose channels lie apart:
// channels first and second; adjacent ones: 2 W channels side by side.
template <typename E, int W, bool ADJACENT>
__global__ void __launch_bounds__(kThreads, 3) pairs_kernel(const Rotary a) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int blocks = a.P / W, units = blocks + (a.copies ? (a.D - 2 * a.P) / W : 0);
    // the block's first row and unit, and from there (units are at most 1,024)
    const int64_t id0 = (int64_t)blockIdx.x * kThreads;
    const int row0 = (int)(id0 / units), in0 = (int)(id0 - (int64_t)row0 * units) + threadIdx.x;
    const int row = row0 + in0 / units, unit = in0 % units;
    if (row >= a.rows) return;
    const int b = row / a.N, n = row - b * a.N;
    const int h0 = blockIdx.y * a.per, h1 = min(a.H, h0 + a.per);
    if (unit >= blocks) {
        const int c = 2 * a.P + (unit - blocks) * W;
        for (int k = 0; k < 2; ++k) {
            Rows<E> r = rows_on<E>(a, k, b, n, h0, h1);
            for (; r.heads > 0; --r.heads, r.x += r.xh, r.y += r.yh)
                store<E, W>(r.y + c, load<E, W>(r.x + c));
        }
        return;
    }
    const int p0 = unit * W;
    int first = 2 * p0, second = 2 * p0 + W;  // adjacent ones
    constexpr bool adjacent = ADJACENT && W > 1;
    if (a.pairing == FLAREPP_ROTARY_HALVES) first = p0, second = p0 + a.P;
    if (a.pairing == FLAREPP_ROTARY_AXES_APART) {
        const int k = axis_of(a, p0), start = k ? a.ends[k - 1] : 0;
        first = p0 + start;
        second = first + a.ends[k] - start;
    }
    float cs[W], sn[W];
    int held = -1;
    float p = 0.f, q = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int k = axis_of(a, p0 + i);
        if (k != held) position(a, b, n, held = k, p, q);
        turn_of(p, q, turns_of(a.freqs[p0 + i]), cs[i], sn[i]);
        sn[i] *= a.sign;
    }
    constexpr int kFlight = 4;
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        Rows<E> r = rows_on<E>(a, k, b, n, h0, h1);
#pragma unroll 1
        for (; r.heads > 0; r.heads -= kFlight) {
            Pack<E, W> u[kFlight], v[kFlight];
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (j < r.heads) {
                    u[j] = load<E, W>(r.x + first);
                    v[j] = load<E, W>(r.x + second);
                    r.x += r.xh;
                }
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (j < r.heads) {
                    float x[2 * W];
                    widen_all<E, W>(u[j], x);
                    widen_all<E, W>(v[j], x + W);
#pragma unroll
                    for (int i = 0; i < W; ++i) {  // adjacent pairs lie side by side in u and v
                        float& p0 = adjacent ? x[2 * i] : x[i];
                        float& p1 = adjacent ? x[2 * i + 1] : x[W + i];
                        const float q0 = p0, q1 = p1;
                        p0 = q0 * cs[i] - q1 * sn[i];
                        p1 = q1 * cs[i] + q0 * sn[i];
                    }
                    narrow_all(u[j], x);
                    narrow_all(v[j], x + W);
                    store<E, W>(r.y + first, u[j]);
                    store<E, W>(r.y + second, v[j]);
                    r.y += r.yh;
                }
        }
    }
}

// Pairs that no vector divides (sections of 6, 5 and 5, say): a thread holds a vector of a token's channels
// as they lie, and their partners come through shared memory, four heads at a time, within a warp. The warp's tokens' sines
// and cosines are taken once a pair, into a table that every thread reads its channels' from. (On a mesh of a
// million points and 16 heads of 32 channels a sine for every channel took 610 us instead of 441.)
// A stage holds vector v (16 bytes) with its words turned by v / 8: the threads of a warp ask for one value each
// of vectors side by side, which without that lie in 8 of 32 banks.
__device__ __forceinline__ uint32_t staged_at(int value, int size) {  // the byte where a value lies
    const uint32_t at = value * size, v = at / 16, w = at % 16 / 4;
    return v * 16 + ((w + v / 8) & 3) * 4 + at % 4;
}
__device__ __forceinline__ uint4 turned(uint4 d, int by) {
    if (by & 1) d = make_uint4(d.w, d.x, d.y, d.z);
    if (by & 2) d = make_uint4(d.z, d.w, d.x, d.y);
    return d;
}

template <typename E, int W>
__global__ void __launch_bounds__(kThreads, 3) rows_kernel(const Rotary a, int tokens) {
    tc::pdl_trigger();
    tc::pdl_wait();
    constexpr int kFlight = 4;
    constexpr uint32_t kHead = 32 * 16;  // bytes of a head's stage of a warp
    __shared__ __align__(16) uint8_t stages[kThreads / 32][kFlight * kHead];
    __shared__ int places[kMaxDim];  // by channel: its pair, its partner, and whether it is the first
    __shared__ Turns freqs[kMaxDim / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint8_t* const stage = stages[warp];
    float2* const table = reinterpret_cast<float2*>(stage);  // [tokens][P], before the stage is used
    for (int pair = threadIdx.x; pair < a.P; pair += kThreads) {
        int first = 2 * pair, second = 2 * pair + 1;
        if (a.pairing == FLAREPP_ROTARY_HALVES) first = pair, second = pair + a.P;
        if (a.pairing == FLAREPP_ROTARY_AXES_APART) {
            const int k = axis_of(a, pair), start = k ? a.ends[k - 1] : 0;
            first = pair + start;
            second = first + a.ends[k] - start;
        }
        freqs[pair] = turns_of(a.freqs[pair]);
        places[first] = pair << 16 | second << 1 | 1;
        places[second] = pair << 16 | first << 1;
    }
    __syncthreads();
    // the warp's tokens, and the lane's vector of one of them
    const int vectors = a.D / W, token = lane / vectors, c0 = (lane - token * vectors) * W;
    const int64_t first_row = ((int64_t)blockIdx.x * (kThreads / 32) + warp) * tokens;
    if (first_row >= a.rows) return;
    const int row0 = (int)first_row, row = row0 + token;
    const bool live = token < tokens && row < a.rows;
    const int b = live ? row / a.N : 0, n = live ? row - b * a.N : 0;
    const int h0 = blockIdx.y * a.per, h1 = min(a.H, h0 + a.per);
    for (int e = lane; e < tokens * a.P; e += 32) {
        const int k = e / a.P, pair = e - k * a.P, r = row0 + k;
        if (r >= a.rows) break;
        const int bk = r / a.N;
        float p, q, c, s;
        position(a, bk, r - bk * a.N, axis_of(a, pair), p, q);
        turn_of(p, q, freqs[pair], c, s);
        table[e] = make_float2(c, s * a.sign);
    }
    __syncwarp();
    float cs[W], sn[W];  // a channel's own: its value times cs plus its partner's times sn
    uint32_t from[W];    // where its partner lies in a stage
    const int rows = token * a.D;
    uint32_t own = 0;    // a bit for every channel that has no partner
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int c = c0 + i;
        cs[i] = 1.f;
        sn[i] = 0.f;
        from[i] = 0;
        if (!live || c >= 2 * a.P) {
            own |= 1u << i;
            continue;
        }
        const int place = places[c];
        const float2 v = table[token * a.P + (place >> 16)];
        cs[i] = v.x;
        sn[i] = place & 1 ? -v.y : v.y;
        from[i] = staged_at(rows + (place >> 1 & 0x7fff), sizeof(E));
    }
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
        Rows<E> r = rows_on<E>(a, k, b, n, h0, h1);
        r.x += c0;
        r.y += c0;
#pragma unroll 1
        for (int left = r.heads; left > 0; left -= kFlight) {
            Pack<E, W> u[kFlight];
            const int now = live ? left : 0;
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (j < now) {
                    u[j] = load<E, W>(r.x);
                    r.x += r.xh;
                }
            __syncwarp();  // the stage (or the table) is read
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (j < now)
                    *reinterpret_cast<uint4*>(stage + lane * 16 + j * kHead) =
                        turned(*reinterpret_cast<const uint4*>(&u[j]), lane / 8);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < kFlight; ++j)
                if (j < now) {
                    float x[W];
                    widen_all<E, W>(u[j], x);
#pragma unroll
                    for (int i = 0; i < W; ++i)
                        x[i] = fmaf(widen(*reinterpret_cast<const E*>(stage + from[i] + j * kHead)), sn[i],
                                    x[i] * cs[i]);
                    const Pack<E, W> old = u[j];
                    narrow_all(u[j], x);
                    if (own)
#pragma unroll
                        for (int i = 0; i < W; ++i)
                            if (own >> i & 1) u[j].v[i] = old.v[i];
                    store<E, W>(r.y, u[j]);
                    r.y += r.yh;
                }
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
    const int64_t rows = a.rows;
    if (whole && !pairs_whole && a.D / W > 32) whole = false;  // rows of more than a warp: channel by channel
    if (whole && !pairs_whole) {
        const int tokens = 32 / (a.D / W);  // of a warp
        const int64_t blocks = cdiv(rows, tokens * (kThreads / 32));
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
    if (!whole) return launch(pairs_kernel<E, 1, false>, grid, st, a);
    return a.pairing == FLAREPP_ROTARY_ADJACENT ? launch(pairs_kernel<E, W, true>, grid, st, a)
                                                : launch(pairs_kernel<E, W, false>, grid, st, a);
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

// Strides of dimensions of size 1 do not matter.
bool same(const flarepp_heads& x, const flarepp_heads& y, const HeadDims& d) {
    return x.data == y.data && (d.B <= 1 || x.stride_b == y.stride_b) && (d.H <= 1 || x.stride_h == y.stride_h) &&
           (d.N <= 1 || x.stride_n == y.stride_n);
}

bool vectors_ok(const flarepp_heads& t, const HeadDims& d, int64_t per) {
    return aligned16(t.data) && (d.B <= 1 || t.stride_b % per == 0) && (d.H <= 1 || t.stride_h % per == 0) &&
           (d.N <= 1 || t.stride_n % per == 0);
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
    if (s->D > kMaxDim || s->Hq > 65535 || s->Hk > 65535 ||
        s->N > INT32_MAX - 1024 || (s->N && s->B > (INT32_MAX - 1024) / s->N))
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
            if (!(i == j && same(*in[i], *out[i], d[i])) && !apart(*out[i], d[i], *in[j], d[j]))
                return FLAREPP_ERR_INVALID_ARGUMENT;
            if (j < i && !apart(*out[i], d[i], *out[j], d[j])) return FLAREPP_ERR_INVALID_ARGUMENT;
        }
    }
    a.rows = (int)(s->B * s->N), a.N = (int)s->N, a.D = (int)s->D, a.P = (int)P;
    a.Hq = (int)s->Hq, a.H = (int)(s->Hq + s->Hk);
    a.axes = s->axes, a.pairing = s->pairing;
    a.sign = s->inverse ? -1.f : 1.f;
    a.positions = positions, a.pos_stride = s->pos_stride_b, a.real = s->real_positions != 0;
    a.freqs = freqs;
    const int64_t per = 16 / e;
    bool whole = s->D % per == 0, in_place = true;
    for (int i = 0; i < 2; ++i) {
        if (d[i].H == 0) continue;
        whole = whole && vectors_ok(*in[i], d[i], per) && vectors_ok(*out[i], d[i], per);
        in_place = in_place && same(*in[i], *out[i], d[i]);
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
