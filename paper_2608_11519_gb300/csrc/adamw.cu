// The AdamW step over all tensors of a model (flarepp_adamw_step) and the values of its 8-bit
// states (flarepp_adamw_moments).
//
// The step is bound by its bytes: per value the weight and both moments are read and written and
// the gradient is read (28 bytes in 32 bits; 14 to 16 with bf16 gradients, a float32 master and
// 8-bit states), against some 20 operations. So one launch walks all tensors of a kind: the
// table of tensors is a kernel parameter (no copy to the device, nothing to keep until the kernel
// has run), a block takes 2,048 values of one tensor, which it finds by bisection of the tensors'
// first blocks, and a warp takes 256 of them, which is also the block that shares a scale in an 8-bit
// state: its largest value is a warp reduction, and a state is read and written once. (Warps that
// take several such blocks in turn measured slower, 192 M values with 8-bit states 939 us instead of
// 819 with the moments read back: each turn waits for its own loads.)
// Measured: 5.8 M values in 32 bits 26.7 us (6.2 TB/s, 0.91 of the copy rate); 192 M bf16 values with float32
// masters and 8-bit states 495 us (6.2 TB/s), and 278 us for the moments read back.
// With 8-bit states the memory leaves about 60 issue slots a value: the codes of sqrt(v) are those
// of a half-precision number of 4 exponent and 4 mantissa bits, so two shifts and a conversion read
// them, and only whole blocks skip the checks of a tensor's end.
//
// Every operation is rounded on its own (no contraction): the step is then a function of its inputs
// that any float32 implementation of the same formulas gives bit for bit, 8-bit codes included.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "checks.h"
#include "flarepp_internal.h"
#include "tc_ptx.cuh"

namespace flarepp {
namespace {

constexpr int kBlockVals = 256;               // values that share a scale
constexpr int kThreads = 256;
constexpr int kItem = kThreads * 8;           // values per thread block
constexpr float kMTop = 256.f;                // what the largest |m| of a block is stored as
constexpr float kRTop = 16384.f;              // what the largest sqrt(v) of a block is stored as
constexpr float kTiny = 7.8886090522101181e-31f;  // 2^-100

struct Entry {
    void* param;
    const void* grad;
    float* master;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    int64_t n;
};
constexpr int kHints = 64;
// CAP tensors of one kind; tensor i owns the thread blocks [first[i], first[i + 1])
template <int CAP>
struct Table {
    Entry e[CAP];
    uint32_t first[CAP + 1];
    int count;
    int shift;                       // block b looks from tensor hint[b >> shift] on,
    uint16_t hint[kHints + 1];       // at most to hint[(b >> shift) + 1]
};
struct Coef {
    float b1, c1, b2, c2, by_bias, eps, keep, rate;
    uint32_t seed;  // of the step (kUnbiased8)
};
// The moments: float32, or codes of 8 bits, rounded to nearest or without bias.
enum State { kFull, kNearest8, kUnbiased8 };

template <int CAP>
__device__ __forceinline__ int find_tensor(const Table<CAP>& t, uint32_t block) {
    int lo = t.hint[block >> t.shift], hi = t.hint[(block >> t.shift) + 1] + 1;
    while (hi - lo > 1) {  // first[lo] <= block < first[hi]
        const int mid = (lo + hi) / 2;
        if (t.first[mid] <= block) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Four values at p[i .. i + 4), those from n on as zeros (FULL: there are none).
template <bool FULL>
__device__ __forceinline__ void load4(const float* p, int64_t i, int64_t n, float* x) {
    if (FULL || i + 4 <= n) {
        const float4 v = *reinterpret_cast<const float4*>(p + i);
        x[0] = v.x;
        x[1] = v.y;
        x[2] = v.z;
        x[3] = v.w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = i + k < n ? p[i + k] : 0.f;
    }
}
template <bool FULL>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, int64_t i, int64_t n, float* x) {
    if (FULL || i + 4 <= n) {
        const uint2 v = *reinterpret_cast<const uint2*>(p + i);
        x[0] = __uint_as_float(v.x << 16);
        x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16);
        x[3] = __uint_as_float(v.y & 0xffff0000u);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = i + k < n ? __bfloat162float(p[i + k]) : 0.f;
    }
}
template <bool FULL>
__device__ __forceinline__ void store4(float* p, int64_t i, int64_t n, const float* x) {
    if (FULL || i + 4 <= n) {
        *reinterpret_cast<float4*>(p + i) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = x[k];
    }
}
template <bool FULL>
__device__ __forceinline__ void store4(__nv_bfloat16* p, int64_t i, int64_t n, const float* x) {
    if (FULL || i + 4 <= n) {
        __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
        *reinterpret_cast<uint2*>(p + i) = make_uint2(*reinterpret_cast<uint32_t*>(&a),
                                                      *reinterpret_cast<uint32_t*>(&b));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = __float2bfloat16_rn(x[k]);
    }
}
template <bool FULL>
__device__ __forceinline__ uint32_t load4_bytes(const void* p, int64_t i, int64_t n) {
    const uint8_t* b = reinterpret_cast<const uint8_t*>(p);
    if (FULL || i + 4 <= n) return *reinterpret_cast<const uint32_t*>(b + i);
    uint32_t v = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) v |= (uint32_t)b[i + k] << (8 * k);
    return v;
}
template <bool FULL>
__device__ __forceinline__ void store4_bytes(void* p, int64_t i, int64_t n, uint32_t v) {
    uint8_t* b = reinterpret_cast<uint8_t*>(p);
    if (FULL || i + 4 <= n) {
        *reinterpret_cast<uint32_t*>(b + i) = v;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) b[i + k] = (uint8_t)(v >> (8 * k));
    }
}

// Four e4m3 codes and their values (exact both ways but for the rounding of `pack`).
__device__ __forceinline__ void unpack_m(uint32_t code, float* x) {
    uint32_t lo, hi;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(code));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = f.x;
    x[1] = f.y;
    x[2] = g.x;
    x[3] = g.y;
}
__device__ __forceinline__ uint32_t pack_m(const float* x) {
    uint32_t code;
    asm("{\n\t.reg .b16 a, b;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 b, %4, %3;\n\t"
        "mov.b32 %0, {a, b};\n\t}"
        : "=r"(code)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
    return code;
}
// Four codes of sqrt(v) (c / 16 below 16, (1 + (c % 16) / 16) 2^(c / 16 - 1) from there on), times
// 2^-14: a code is the upper eight of the ten used bits of such a half-precision number.
__device__ __forceinline__ void unpack_r(uint32_t codes, float* x) {
    const uint32_t lo = __byte_perm(codes, 0, 0x4140) << 6, hi = __byte_perm(codes, 0, 0x4342) << 6;
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = f.x;
    x[1] = f.y;
    x[2] = g.x;
    x[3] = g.y;
}
// The code of y (in its low eight bits): y rounded to four mantissa bits, ties to even; below 1 the
// steps are sixteenths, which adding 2^19 rounds to. A y that is not zero never becomes zero.
__device__ __forceinline__ uint32_t pack_r(float y) {
    const uint32_t bits = __float_as_uint(y);
    const uint32_t high = (bits + (0x3FFFFu - (126u << 23)) + ((bits >> 19) & 1u)) >> 19;
    const uint32_t low = __float_as_uint(__fadd_rn(y, 524288.f)) - __float_as_uint(524288.f);
    return max(y < 1.f ? low : high, min(bits, 1u));
}

// Rounding without bias: a value goes up to the next code with a probability that is its distance from
// the code below in steps, so that changes of less than half a step (a second moment moves by (1 - beta2)
// of itself) are kept on average instead of lost. Random bits are a hash of the value's place in its
// tensor and of the step: xor-shifts and multiplications by odd numbers (the fractional digits of the
// square roots of 2 and 3), each output bit a function of all input bits; the lower half is for m, the
// upper for sqrt(v). The integer work shows: 192 M bf16 values with masters take 545 us, with codes
// rounded to nearest 475.
__host__ __device__ __forceinline__ uint32_t hashed(uint32_t x) {
    x ^= x >> 16;
    x *= 0x6A09E667u;
    x ^= x >> 15;
    x *= 0xBB67AE85u;
    return x ^ (x >> 16);
}
// The e4m3 value above or below y: 3 mantissa bits, steps of 2^-9 below 2^-6 (which adding 2^-6 gives).
__device__ __forceinline__ float dither_m(float y, uint32_t random) {
    const float a = fabsf(y), lift = a < 0x1p-6f ? 0x1p-6f : 0.f;
    const uint32_t bits = __float_as_uint(__fadd_rn(a, lift)) + ((random & 0xffffu) << 4);
    return copysignf(__fsub_rn(__uint_as_float(bits & 0xfff00000u), lift), y);
}
// The code above or below y, as pack_r's codes (sixteenths below 1, which adding 1 gives).
__device__ __forceinline__ uint32_t dither_r(float y, uint32_t random) {
    const bool small = y < 1.f;
    const uint32_t bits = __float_as_uint(small ? __fadd_rn(y, 1.f) : y) + (random >> 16 << 3);
    return max((bits >> 19) - (126u << 4) - (small ? 16u : 0u), min(__float_as_uint(y), 1u));
}

// The largest |x| over the warp, as bits (so that a NaN is the largest of all).
__device__ __forceinline__ float warp_most(const float (*x)[4]) {
    uint32_t most = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) most = max(most, __float_as_uint(x[h][k]) & 0x7fffffffu);
    return __uint_as_float(__reduce_max_sync(0xffffffffu, most));
}

// 256 values from `at` on, by one warp. P, G: types of the weights and the gradients. MASTER: the
// weights have a float32 master. S: the moments. FULL: all 256 exist. A lane holds values
// 4 lane + 128 h + (0..3).
template <typename P, typename G, bool MASTER, State S, bool FULL>
__device__ __forceinline__ void step_block(const Entry& e, const Coef& c, int64_t at) {
    constexpr bool Q8 = S != kFull;
    const int lane = threadIdx.x % 32;
    const int64_t n = e.n;
    const int64_t block = at / kBlockVals;
    float w[2][4], g[2][4], m[2][4], v[2][4];
    uint32_t mc[2], vc[2];
    float ms, vs;
    if (Q8) {
        ms = e.m_scale[block];
        vs = e.v_scale[block] * kRTop;  // exact, like the codes' 2^-14
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t i = at + 128 * h + 4 * lane;
        load4<FULL>(reinterpret_cast<const G*>(e.grad), i, n, g[h]);
        if (MASTER) load4<FULL>(e.master, i, n, w[h]);
        else load4<FULL>(reinterpret_cast<const P*>(e.param), i, n, w[h]);
        if (Q8) {
            mc[h] = load4_bytes<FULL>(e.m, i, n);
            vc[h] = load4_bytes<FULL>(e.v, i, n);
        } else {
            load4<FULL>(reinterpret_cast<const float*>(e.m), i, n, m[h]);
            load4<FULL>(reinterpret_cast<const float*>(e.v), i, n, v[h]);
        }
    }
    float r[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (Q8) {
            unpack_m(mc[h], m[h]);
            unpack_r(vc[h], v[h]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                m[h][k] = __fmul_rn(m[h][k], ms);
                const float root = __fmul_rn(v[h][k], vs);
                v[h][k] = __fmul_rn(root, root);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float gr = g[h][k];
            m[h][k] = __fadd_rn(__fmul_rn(m[h][k], c.b1), __fmul_rn(gr, c.c1));
            v[h][k] = __fadd_rn(__fmul_rn(v[h][k], c.b2), __fmul_rn(__fmul_rn(gr, gr), c.c2));
            r[h][k] = __fsqrt_rn(v[h][k]);
            const float over = __fadd_rn(__fmul_rn(r[h][k], c.by_bias), c.eps);
            w[h][k] = __fsub_rn(__fmul_rn(w[h][k], c.keep),
                                __fmul_rn(__fdiv_rn(m[h][k], over), c.rate));
        }
        const int64_t i = at + 128 * h + 4 * lane;
        if (MASTER) store4<FULL>(e.master, i, n, w[h]);
        store4<FULL>(reinterpret_cast<P*>(e.param), i, n, w[h]);
        if (!Q8) {
            store4<FULL>(reinterpret_cast<float*>(e.m), i, n, m[h]);
            store4<FULL>(reinterpret_cast<float*>(e.v), i, n, v[h]);
        }
    }
    if (!Q8) return;
    // values from n on are zeros and do not count
    const float m_most = warp_most(m), r_most = warp_most(r);
    const bool m_live = !(m_most < kTiny), r_live = !(r_most < kTiny);
    const float m_by = m_live ? __fdiv_rn(kMTop, m_most) : 0.f;
    const float r_by = r_live ? __fdiv_rn(kRTop, r_most) : 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t i = at + 128 * h + 4 * lane;
        float y[4];
        uint32_t rc[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[k] = __fmul_rn(m[h][k], m_by);
            const float root = __fmul_rn(r[h][k], r_by);
            if (S == kUnbiased8) {
                const uint64_t j = (uint64_t)(i + k);
                const uint32_t random = hashed(((uint32_t)j + (uint32_t)(j >> 32) * 0x9E3779B9u) ^ c.seed);
                y[k] = dither_m(y[k], random);
                rc[k] = dither_r(root, random);
            } else {
                rc[k] = pack_r(root);
            }
        }
        const uint32_t code = __byte_perm(__byte_perm(rc[0], rc[1], 0x0040),
                                          __byte_perm(rc[2], rc[3], 0x0040), 0x5410);
        store4_bytes<FULL>(e.m, i, n, pack_m(y));
        store4_bytes<FULL>(e.v, i, n, code);
    }
    if (lane == 0) {
        e.m_scale[block] = m_live ? m_most * (1.f / kMTop) : 0.f;
        e.v_scale[block] = r_live ? r_most * (1.f / kRTop) : 0.f;
    }
}

template <typename P, typename G, bool MASTER, State S, int CAP>
__global__ void __launch_bounds__(kThreads, 5)
    adamw_kernel(const __grid_constant__ Table<CAP> table, const Coef c) {
    const int t = find_tensor(table, blockIdx.x);
    const Entry& e = table.e[t];
    const int64_t n = e.n;
    const int64_t at = (int64_t)(blockIdx.x - table.first[t]) * kItem + threadIdx.x / 32 * kBlockVals;
    if (at + kBlockVals <= n) step_block<P, G, MASTER, S, true>(e, c, at);
    else if (at < n) step_block<P, G, MASTER, S, false>(e, c, at);
}

// The values of 8-bit states; e.param and e.master are the outputs for m and v.
template <bool FULL>
__device__ __forceinline__ void moments_block(const Entry& e, int64_t at) {
    const int lane = threadIdx.x % 32;
    const float ms = e.m_scale[at / kBlockVals], vs = e.v_scale[at / kBlockVals] * kRTop;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t i = at + 128 * h + 4 * lane;
        const uint32_t mc = load4_bytes<FULL>(e.m, i, e.n), vc = load4_bytes<FULL>(e.v, i, e.n);
        float m[4], v[4];
        unpack_m(mc, m);
        unpack_r(vc, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] = __fmul_rn(m[k], ms);
            const float root = __fmul_rn(v[k], vs);
            v[k] = __fmul_rn(root, root);
        }
        store4<FULL>(reinterpret_cast<float*>(e.param), i, e.n, m);
        store4<FULL>(e.master, i, e.n, v);
    }
}

template <int CAP>
__global__ void __launch_bounds__(kThreads)
    moments_kernel(const __grid_constant__ Table<CAP> table) {
    const int t = find_tensor(table, blockIdx.x);
    const Entry& e = table.e[t];
    const int64_t n = e.n;
    const int64_t at = (int64_t)(blockIdx.x - table.first[t]) * kItem + threadIdx.x / 32 * kBlockVals;
    if (at + kBlockVals <= n) moments_block<true>(e, at);
    else if (at < n) moments_block<false>(e, at);
}

// ------------------------------------------------------------------ host side

// Tensors per launch: a table of kFew stays within the 4 KB of parameters that every launch
// carries cheaply; one of kMany takes most of the 32 KB that a launch may carry.
constexpr int kFew = 48;
constexpr int kMany = 384;

bool type_ok(int32_t t) { return t == FLAREPP_F32 || t == FLAREPP_BF16; }

// 0..5 for the type combinations of the step
int kind_of(const flarepp_adamw_tensor& t) {
    const int g = t.grad_dtype == FLAREPP_BF16;
    if (t.param_dtype == FLAREPP_F32) return g;
    return 2 + 2 * (t.master != nullptr) + g;
}

flarepp_status check_tensor(const flarepp_adamw_tensor& t, bool q8) {
    if (t.n < 0 || !type_ok(t.param_dtype) || !type_ok(t.grad_dtype))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    if (t.n == 0) return FLAREPP_OK;
    const void* need[4] = {t.param, t.grad, t.m, t.v};
    for (const void* p : need)
        if (!p || !aligned16(p)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!aligned16(t.master) || (t.master && t.param_dtype == FLAREPP_F32))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    // the scales, one value at a time, may start anywhere in a buffer of all tensors' scales
    if (q8 && (!t.m_scale || !t.v_scale || !aligned4(t.m_scale) || !aligned4(t.v_scale)))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const size_t n = (size_t)t.n, sb = (size_t)cdiv(t.n, kBlockVals) * 4;
    const size_t state = n * (q8 ? 1 : 4);
    const Span outs[6] = {{t.param, n * (t.param_dtype == FLAREPP_BF16 ? 2 : 4)},
                          {t.master, n * 4},
                          {t.m, state},
                          {t.v, state},
                          {q8 ? t.m_scale : nullptr, sb},
                          {q8 ? t.v_scale : nullptr, sb}};
    const Span in{t.grad, n * (t.grad_dtype == FLAREPP_BF16 ? 2 : 4)};
    return disjoint(outs, 6, &in, 1) ? FLAREPP_OK : FLAREPP_ERR_INVALID_ARGUMENT;
}

template <int CAP>
void set_hints(Table<CAP>* t, uint32_t blocks) {
    t->shift = 0;
    while ((blocks - 1) >> t->shift >= kHints) ++t->shift;
    int i = 0;
    for (int h = 0; h <= kHints; ++h) {  // the tensor of block h << shift, or the last one
        const uint64_t b = (uint64_t)h << t->shift;
        while (i + 1 < t->count && t->first[i + 1] <= b) ++i;
        t->hint[h] = (uint16_t)i;
    }
}

// Launch once per CAP tensors that `pick` accepts; `fill` makes a tensor's entry.
template <int CAP, typename Pick, typename Fill, typename Go>
cudaError_t each_table(int64_t n_tensors, Pick pick, Fill fill, Go go) {
    Table<CAP> t;
    t.count = 0;
    uint64_t blocks = 0;
    for (int64_t i = 0; i <= n_tensors; ++i) {
        const bool end = i == n_tensors;
        if (!end && !pick(i)) continue;
        Entry e{};
        uint64_t more = 0;
        if (!end) {
            e = fill(i);
            more = (uint64_t)cdiv(e.n, kItem);
        }
        if (t.count && (end || t.count == CAP || blocks + more > 0x7fffffffull)) {
            t.first[t.count] = (uint32_t)blocks;
            set_hints(&t, (uint32_t)blocks);
            const cudaError_t err = go(t, (unsigned)blocks);
            if (err != cudaSuccess) return err;
            t.count = 0;
            blocks = 0;
        }
        if (end) break;
        if (more > 0x7fffffffull) return cudaErrorInvalidValue;
        t.first[t.count] = (uint32_t)blocks;
        t.e[t.count++] = e;
        blocks += more;
    }
    return cudaSuccess;
}

template <typename P, typename G, bool MASTER, State S, int CAP>
cudaError_t go_step(const Table<CAP>& t, unsigned blocks, const Coef& c, cudaStream_t st) {
    adamw_kernel<P, G, MASTER, S, CAP><<<blocks, kThreads, 0, st>>>(t, c);
    return cudaGetLastError();
}

template <State S, int CAP>
cudaError_t step_all(const flarepp_adamw_tensor* ts, int64_t n, const Coef& c, cudaStream_t st) {
    for (int kind = 0; kind < 6; ++kind) {
        const cudaError_t e = each_table<CAP>(
            n, [&](int64_t i) { return ts[i].n > 0 && kind_of(ts[i]) == kind; },
            [&](int64_t i) {
                const flarepp_adamw_tensor& t = ts[i];
                return Entry{t.param, t.grad, t.master, t.m, t.v, t.m_scale, t.v_scale, t.n};
            },
            [&](const Table<CAP>& t, unsigned blocks) {
                using B = __nv_bfloat16;
                switch (kind) {
                    case 0: return go_step<float, float, false, S, CAP>(t, blocks, c, st);
                    case 1: return go_step<float, B, false, S, CAP>(t, blocks, c, st);
                    case 2: return go_step<B, float, false, S, CAP>(t, blocks, c, st);
                    case 3: return go_step<B, B, false, S, CAP>(t, blocks, c, st);
                    case 4: return go_step<B, float, true, S, CAP>(t, blocks, c, st);
                }
                return go_step<B, B, true, S, CAP>(t, blocks, c, st);
            });
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <int CAP>
cudaError_t step_any(State s, const flarepp_adamw_tensor* ts, int64_t n, const Coef& c,
                     cudaStream_t st) {
    return s == kFull       ? step_all<kFull, CAP>(ts, n, c, st)
           : s == kNearest8 ? step_all<kNearest8, CAP>(ts, n, c, st)
                            : step_all<kUnbiased8, CAP>(ts, n, c, st);
}

flarepp_status adamw_step(const flarepp_adamw_tensor* ts, int64_t n, const flarepp_adamw_hyper* h,
                          bool unbiased, cudaStream_t st) {
    if (!h || n < 0 || (n && !ts)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if ((h->state_bits != 32 || unbiased) && h->state_bits != 8) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!isfinite(h->lr) || !isfinite(h->weight_decay) || !(h->eps >= 0) || !isfinite(h->eps) ||
        !(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1) || h->step < 1)
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const bool q8 = h->state_bits == 8;
    for (int64_t i = 0; i < n; ++i) {
        const flarepp_status s = check_tensor(ts[i], q8);
        if (s != FLAREPP_OK) return s;
    }
    Coef c;
    c.b1 = (float)h->beta1;
    c.c1 = (float)(1 - h->beta1);
    c.b2 = (float)h->beta2;
    c.c2 = (float)(1 - h->beta2);
    c.by_bias = (float)(1 / sqrt(1 - pow(h->beta2, (double)h->step)));
    c.eps = (float)h->eps;
    c.keep = (float)(1 - h->lr * h->weight_decay);
    c.rate = (float)(h->lr / (1 - pow(h->beta1, (double)h->step)));
    c.seed = hashed((uint32_t)(uint64_t)h->step * 0x9E3779B9u + (uint32_t)((uint64_t)h->step >> 32));
    const State s = !q8 ? kFull : unbiased ? kUnbiased8 : kNearest8;
    const cudaError_t e = n <= kFew ? step_any<kFew>(s, ts, n, c, st) : step_any<kMany>(s, ts, n, c, st);
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

template <int CAP>
cudaError_t moments_all(const flarepp_adamw_tensor* ts, int64_t n, float* const* m_out,
                        float* const* v_out, cudaStream_t st) {
    return each_table<CAP>(
        n, [&](int64_t i) { return ts[i].n > 0; },
        [&](int64_t i) {
            const flarepp_adamw_tensor& t = ts[i];
            return Entry{m_out[i], nullptr, v_out[i], t.m, t.v, t.m_scale, t.v_scale, t.n};
        },
        [&](const Table<CAP>& t, unsigned blocks) {
            moments_kernel<CAP><<<blocks, kThreads, 0, st>>>(t);
            return cudaGetLastError();
        });
}

flarepp_status adamw_moments(const flarepp_adamw_tensor* ts, int64_t n, float* const* m_out,
                             float* const* v_out, cudaStream_t st) {
    if (n < 0 || (n && (!ts || !m_out || !v_out))) return FLAREPP_ERR_INVALID_ARGUMENT;
    for (int64_t i = 0; i < n; ++i) {
        const flarepp_adamw_tensor& t = ts[i];
        if (t.n < 0) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (t.n == 0) continue;
        const void* need[4] = {t.m, t.v, m_out[i], v_out[i]};
        for (const void* p : need)
            if (!p || !aligned16(p)) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (!t.m_scale || !t.v_scale || !aligned4(t.m_scale) || !aligned4(t.v_scale))
            return FLAREPP_ERR_INVALID_ARGUMENT;
        const size_t sb = (size_t)cdiv(t.n, kBlockVals) * 4;
        const Span outs[2] = {{m_out[i], (size_t)t.n * 4}, {v_out[i], (size_t)t.n * 4}};
        const Span ins[4] = {{t.m, (size_t)t.n}, {t.v, (size_t)t.n}, {t.m_scale, sb}, {t.v_scale, sb}};
        if (!disjoint(outs, 2, ins, 4)) return FLAREPP_ERR_INVALID_ARGUMENT;
    }
    const cudaError_t e = n <= kFew ? moments_all<kFew>(ts, n, m_out, v_out, st)
                                    : moments_all<kMany>(ts, n, m_out, v_out, st);
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

}  // namespace
}  // namespace flarepp

extern "C" {

flarepp_status flarepp_adamw_step(const flarepp_adamw_tensor* tensors, int64_t n_tensors,
                                  const flarepp_adamw_hyper* hyper, void* stream) {
    return flarepp::adamw_step(tensors, n_tensors, hyper, false, (cudaStream_t)stream);
}

flarepp_status flarepp_adamw_step_unbiased(const flarepp_adamw_tensor* tensors, int64_t n_tensors,
                                           const flarepp_adamw_hyper* hyper, void* stream) {
    return flarepp::adamw_step(tensors, n_tensors, hyper, true, (cudaStream_t)stream);
}

flarepp_status flarepp_adamw_moments(const flarepp_adamw_tensor* tensors, int64_t n_tensors,
                                     float* const* m_out, float* const* v_out, void* stream) {
    return flarepp::adamw_moments(tensors, n_tensors, m_out, v_out, (cudaStream_t)stream);
}

}  // extern "C"
