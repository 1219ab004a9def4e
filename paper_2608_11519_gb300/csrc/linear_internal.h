// Declarations shared by the translation units of the linear layer (not installed).
#pragma once
#include <cuda_bf16.h>

#include "flarepp_internal.h"

namespace flarepp {

// One matrix operand of a product D[M][N] = sum_k A(m, k) B(n, k), bf16. `mn` = 0: the
// contraction is innermost, memory [rows][k]; `mn` = 1: the rows are innermost, memory
// [k][rows]. `pitch` is the distance of two lines in elements (a multiple of 8).
struct LinOperand {
    const void* t;
    int64_t pitch;
    int mn;
};

// What happens to the sums. Either the epilogue: z = sum + bias[n] (kept in Z when it is not
// null), Y = act(z) + R, all [M][N] bf16; or, when `part` is set, the float32 sums of each
// chunk of the contraction go to part[chunk][M][ldp].
struct LinEpilogue {
    int act;
    const void* bias;
    const void* R;
    void* Y;
    void* Z;
    float* part;
    int64_t ldp;
    int backward;  // take the rows from the last to the first
};

// How a product is cut: tiles of 256 rows x NT columns, `chunks` parts of the contraction.
struct LinPlan {
    int NT;
    int chunks;
};
LinPlan lin_plan(int64_t M, int64_t N, int64_t K);

// Enqueue the product (tc_linear.cu). M, N, K below 2^31.
cudaError_t lin_gemm(const LinPlan& plan, int64_t M, int64_t N, int64_t K, const LinOperand& a,
                     const LinOperand& b, const LinEpilogue& e, int* status, cudaStream_t st);

// The product of up to kFewRows rows of x (contraction innermost) with w: [rows][cols], with the
// epilogue, in one launch.
constexpr int64_t kFewRows = 256;
cudaError_t lin_few(int64_t rows, int64_t cols, int64_t K, const LinOperand& x,
                    const LinOperand& w, const LinEpilogue& e, int* status, cudaStream_t st);

// dX = (dY o act'(Z)) W for a layer of up to kFusedIn inputs (a multiple of 8) and kFusedOut outputs (a
// multiple of 8) with an activation, in one pass that also leaves dZ (when it is not null, lines of `ldz`)
// and per CTA the column sums of dZ (db_part[ctas][ldz], at most kNumSMs rows, when it is not null). w: W
// with its inputs innermost.
constexpr int64_t kFusedIn = 256, kFusedOut = 512;
cudaError_t lin_fused(int64_t T, int64_t K, int64_t N, int act, const void* dY, const void* Z,
                      const LinOperand& w, void* dX, void* dZ, float* db_part, int64_t ldz,
                      int* ctas, int* status, cudaStream_t st);

// ---- activations (flarepp_activation) and their slopes, float32
__device__ __forceinline__ float rcp_approx(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float ex2_approx(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// Two floats as one operand of the packed float32 instructions.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(uint64_t v) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
    return f;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// 1 / (1 + 2^-u) of both halves: 2 exponentials, 2 reciprocals, one packed addition.
__device__ __forceinline__ uint64_t sigmoid2(uint64_t minus_u) {
    const float2 u = halves(minus_u);
    const float2 d = halves(add2(pair(ex2_approx(u.x), ex2_approx(u.y)), pair(1.f, 1.f)));
    return pair(rcp_approx(d.x), rcp_approx(d.y));
}
// The normal distribution function as 1 / (1 + 2^-u), u(z) = log2(Phi(z) / Phi(-z)): odd and smooth,
// so an odd polynomial of degree 13 does, fitted for the least largest error of z Phi(z) over
// |z| <= 5 (2.3e-7; 5e-7 with float32 arithmetic; beyond 5 it grows faster than u, and z Phi(z)
// is below 1.5e-6 from its limits). Down to z = -5 Phi keeps a relative precision of 2.2e-3 (half a unit of
// the bf16 result); below that only an absolute one: z Phi(z) is off by 1.8e-8 at most, which is 4 % of it at
// -5.25 and all of it from -6.5 on. It takes about 8 issue slots a value in pairs, where the epilogue of a
// memory-bound layer has about 16 for everything.
__device__ __forceinline__ uint64_t normal_cdf2(uint64_t z) {
    const uint64_t s = mul2(z, z);
    uint64_t p = pair(-4.122593377786643e-09f, -4.122593377786643e-09f);
    p = fma2(p, s, pair(3.340366276916029e-07f, 3.340366276916029e-07f));
    p = fma2(p, s, pair(-1.0618686246743891e-05f, -1.0618686246743891e-05f));
    p = fma2(p, s, pair(1.5339275705628097e-04f, 1.5339275705628097e-04f));
    p = fma2(p, s, pair(1.15053633635398e-04f, 1.15053633635398e-04f));
    p = fma2(p, s, pair(-1.0486429184675217e-01f, -1.0486429184675217e-01f));
    p = fma2(p, s, pair(-2.3021974563598633f, -2.3021974563598633f));
    return sigmoid2(mul2(p, z));
}
__device__ __forceinline__ uint64_t logistic2(uint64_t z) {
    return sigmoid2(mul2(z, pair(-1.44269504f, -1.44269504f)));
}
// act of both halves. Every operation is an instruction of its own, so that a value has the same
// bits wherever it is computed.
__device__ __forceinline__ uint64_t act_value2(int act, uint64_t z) {
    switch (act) {
        case FLAREPP_ACT_RELU: {
            const float2 f = halves(z);
            return pair(f.x < 0.f ? 0.f : f.x, f.y < 0.f ? 0.f : f.y);  // keeps a NaN
        }
        case FLAREPP_ACT_GELU: return mul2(z, normal_cdf2(z));
        case FLAREPP_ACT_SILU: return mul2(z, logistic2(z));
    }
    return z;
}
// act' of both halves: 1 or 0; Phi(z) + z phi(z); s (1 + z (1 - s)) with s = logistic(z).
__device__ __forceinline__ uint64_t act_slope2(int act, uint64_t z) {
    switch (act) {
        case FLAREPP_ACT_RELU: {
            const float2 f = halves(z);
            return pair(f.x > 0.f ? 1.f : 0.f, f.y > 0.f ? 1.f : 0.f);
        }
        case FLAREPP_ACT_GELU: {
            const float2 q = halves(mul2(mul2(z, z), pair(-0.72134752f, -0.72134752f)));
            const uint64_t e = pair(ex2_approx(q.x), ex2_approx(q.y));  // exp(-z^2 / 2)
            return fma2(mul2(z, pair(0.39894228f, 0.39894228f)), e, normal_cdf2(z));
        }
        case FLAREPP_ACT_SILU: {
            const uint64_t s = logistic2(z), one = pair(1.f, 1.f);
            const uint64_t t = fma2(s, pair(-1.f, -1.f), one);
            return mul2(s, fma2(z, t, one));
        }
    }
    return pair(1.f, 1.f);
}
__device__ __forceinline__ uint32_t pack_bf16x2(uint64_t v) {
    const float2 f = halves(v);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint64_t unpack_bf16x2(uint32_t v) {
    return pair(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

}  // namespace flarepp
