// The single-token step of the decay attention (flarepp_decay_attention_step): for every sequence and query
// head, S = g S + k v^T [Dk, Dv] in place and y = scale q S, in float32.
//
// Bound by the states' bytes, read once and written once: 4 Dk Dv values each way for 2 (Dk + Dv) of the token.
// A block takes kCols columns of one state (whole 128-byte lines), so that one sequence's eight heads
// are already 16 blocks or more; a thread four of the columns and every 32nd row, so y's sums end in a
// warp's shuffles and one row of eight warps' sums.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "decay.h"
#include "layer_status.cuh"
#include "tc_ptx.cuh"

namespace flarepp {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 32;
constexpr int kRowGroups = kThreads / (kCols / 4);  // 32
constexpr int kMaxDim = 128;
constexpr int kTurns = kMaxDim / kRowGroups;  // rows of a thread, at most

struct Step {
    const __nv_bfloat16 *q, *k, *v;
    __nv_bfloat16* y;
    int64_t qb, qh, kb, kh, vb, vh, yb, yh;
    const float* log_decay;
    float* state;
    int Hq, group, Dk, Dv, tiles;
    float scale;
    int* status;
};

__global__ void __launch_bounds__(kThreads) step_kernel(const Step p) {
    __shared__ float4 sums[kThreads / 32][kCols / 4];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int64_t item = blockIdx.x / p.tiles;
    const int tile = (int)(blockIdx.x - item * p.tiles);
    const int64_t b = item / p.Hq;
    const int h = (int)(item - b * p.Hq), hk = h / p.group;
    const int x = threadIdx.x % (kCols / 4), r0 = threadIdx.x / (kCols / 4);
    const int c = tile * kCols + 4 * x;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < p.Dv) {
        float* S = p.state + (item * p.Dk + r0) * p.Dv + c;
        float4 s[kTurns];
        float k[kTurns], q[kTurns];
#pragma unroll
        for (int i = 0; i < kTurns; ++i)
            if (r0 + i * kRowGroups < p.Dk)
                s[i] = *reinterpret_cast<const float4*>(S + (int64_t)i * kRowGroups * p.Dv);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int r = r0 + i * kRowGroups;
            k[i] = r < p.Dk ? __bfloat162float(p.k[b * p.kb + hk * p.kh + r]) : 0.f;
            q[i] = r < p.Dk ? __bfloat162float(p.q[b * p.qb + h * p.qh + r]) : 0.f;
        }
        const uint2 raw = *reinterpret_cast<const uint2*>(p.v + b * p.vb + hk * p.vh + c);
        const float v0 = __uint_as_float(raw.x << 16), v1 = __uint_as_float(raw.x & 0xffff0000u);
        const float v2 = __uint_as_float(raw.y << 16), v3 = __uint_as_float(raw.y & 0xffff0000u);
        float ld = p.log_decay[h];
        if (!(ld <= 0.f)) {
            if (threadIdx.x == 0) record_status(p.status, FLAREPP_ERR_INVALID_ARGUMENT);
            ld = ld > 0.f ? 0.f : -INFINITY;
        }
        const float g = expf(ld);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            if (r0 + i * kRowGroups >= p.Dk) break;
            // g = 0 forgets a state that is not finite, too
            s[i].x = fmaf(k[i], v0, g > 0.f ? g * s[i].x : 0.f);
            s[i].y = fmaf(k[i], v1, g > 0.f ? g * s[i].y : 0.f);
            s[i].z = fmaf(k[i], v2, g > 0.f ? g * s[i].z : 0.f);
            s[i].w = fmaf(k[i], v3, g > 0.f ? g * s[i].w : 0.f);
            *reinterpret_cast<float4*>(S + (int64_t)i * kRowGroups * p.Dv) = s[i];
            acc.x = fmaf(q[i], s[i].x, acc.x);
            acc.y = fmaf(q[i], s[i].y, acc.y);
            acc.z = fmaf(q[i], s[i].z, acc.z);
            acc.w = fmaf(q[i], s[i].w, acc.w);
        }
    }
#pragma unroll
    for (int k = kCols / 4; k < 32; k <<= 1) {
        acc.x += __shfl_xor_sync(0xffffffffu, acc.x, k);
        acc.y += __shfl_xor_sync(0xffffffffu, acc.y, k);
        acc.z += __shfl_xor_sync(0xffffffffu, acc.z, k);
        acc.w += __shfl_xor_sync(0xffffffffu, acc.w, k);
    }
    if (threadIdx.x % 32 < kCols / 4) sums[threadIdx.x / 32][x] = acc;
    __syncthreads();
    if (threadIdx.x >= kCols / 4 || c >= p.Dv) return;
    acc = sums[0][x];
    for (int w = 1; w < kThreads / 32; ++w) {
        const float4 o = sums[w][x];
        acc.x += o.x;
        acc.y += o.y;
        acc.z += o.z;
        acc.w += o.w;
    }
    const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * p.scale, acc.y * p.scale);
    const __nv_bfloat162 hi = __floats2bfloat162_rn(acc.z * p.scale, acc.w * p.scale);
    uint2 out;
    out.x = *reinterpret_cast<const uint32_t*>(&lo);
    out.y = *reinterpret_cast<const uint32_t*>(&hi);
    *reinterpret_cast<uint2*>(p.y + b * p.yb + h * p.yh + c) = out;
}

}  // namespace

cudaError_t take_decay_step_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

cudaError_t decay_step(const flarepp_decay_shape& s, const flarepp_heads& Q, const flarepp_heads& K,
                       const flarepp_heads& V, const float* log_decay, float* state,
                       const flarepp_heads& Y, int32_t* status, cudaStream_t st) {
    Step p{};
    p.q = (const __nv_bfloat16*)Q.data, p.k = (const __nv_bfloat16*)K.data;
    p.v = (const __nv_bfloat16*)V.data, p.y = (__nv_bfloat16*)Y.data;
    p.qb = Q.stride_b, p.qh = Q.stride_h, p.kb = K.stride_b, p.kh = K.stride_h;
    p.vb = V.stride_b, p.vh = V.stride_h, p.yb = Y.stride_b, p.yh = Y.stride_h;
    p.log_decay = log_decay, p.state = state;
    p.Hq = (int)s.Hq, p.group = (int)(s.Hq / s.Hk), p.Dk = (int)s.Dk, p.Dv = (int)s.Dv;
    p.tiles = (int)cdiv(s.Dv, kCols);
    p.scale = s.scale;
    p.status = status;
    const int64_t blocks = s.B * s.Hq * p.tiles;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, step_kernel, p);
}

}  // namespace flarepp
