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
// chunk of the contraction go to part[chunk][M][ldp] (transposed: part[chunk][N][ldp], for
// products whose rows are the output's columns).
struct LinEpilogue {
    int act;
    const void* bias;
    const void* R;
    void* Y;
    void* Z;
    float* part;
    int64_t ldp;
};

// How a product is cut: tiles of 128 * cg rows x NT columns, `chunks` parts of the contraction.
struct LinPlan {
    int cg;       // CTAs that share a tile: 1, or 2 (cta_group::2)
    int NT;
    int chunks;
    bool transposed;
};
LinPlan lin_plan(int64_t M, int64_t N, int64_t K, bool few_columns);

// Enqueue the product (tc_linear.cu). M, N, K below 2^31.
cudaError_t lin_gemm(const LinPlan& plan, int64_t M, int64_t N, int64_t K, const LinOperand& a,
                     const LinOperand& b, const LinEpilogue& e, int* status, cudaStream_t st);

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
// The normal distribution function Phi(z), and e = exp(-z^2 / 2). Abramowitz and Stegun's
// rational approximation 7.1.26 of erf (absolute error 1.5e-7, against the 2^-8 of the bf16 result)
// at |z| / sqrt 2, taken as the lower tail so that a large negative z keeps its digits: six
// multiply-adds, one reciprocal and one exponential, which the slope uses again.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float a = fabsf(z);
    const float t = rcp_approx(fmaf(a, 0.3275911f * 0.70710678f, 1.f));
    e = ex2_approx(z * z * -0.72134752f);  // log2(e) / 2
    float p = fmaf(t, 1.061405429f, -1.453152027f);
    p = fmaf(t, p, 1.421413741f);
    p = fmaf(t, p, -0.284496736f);
    p = fmaf(t, p, 0.254829592f);
    const float tail = 0.5f * t * p * e;
    return z > 0.f ? 1.f - tail : tail;
}
__device__ __forceinline__ float logistic(float z) {
    return rcp_approx(1.f + ex2_approx(z * -1.44269504f));
}
// (The last product is rounded on its own: fused into the residual's addition in one of the
// compiler's copies of a loop and not in another, the same call would not give the same bits with
// and without Z.)
__device__ __forceinline__ float act_value(int act, float z) {
    float e;
    switch (act) {
        case FLAREPP_ACT_RELU: return z < 0.f ? 0.f : z;  // keeps a NaN
        case FLAREPP_ACT_GELU: return __fmul_rn(z, normal_cdf(z, e));
        case FLAREPP_ACT_SILU: return __fmul_rn(z, logistic(z));
    }
    return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
    float e;
    switch (act) {
        case FLAREPP_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case FLAREPP_ACT_GELU: {
            const float cdf = normal_cdf(z, e);
            return fmaf(z * 0.39894228f, e, cdf);
        }
        case FLAREPP_ACT_SILU: {
            const float s = logistic(z);
            return s * fmaf(z, 1.f - s, 1.f);
        }
    }
    return 1.f;
}

}  // namespace flarepp
