// The entry points of the decay attention: checks of the arguments and the launches
// (flarepp_decay_attention_*). The kernels are in tc_decay.cu and decay_step.cu.
#include <cuda_runtime.h>
#include <math.h>

#include "checks.h"
#include "decay.h"

namespace flarepp {
namespace {

constexpr int64_t kMaxDim = 128;

flarepp_status check_shape(const flarepp_decay_shape* s) {
    if (!s || s->B < 0 || s->Hq < 0 || s->Hk < 0 || s->N < 0 || s->Dk < 1 || s->Dv < 1 || s->sequences < 0)
        return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->dtype != FLAREPP_F32 && s->dtype != FLAREPP_BF16) return FLAREPP_ERR_INVALID_ARGUMENT;
    if ((s->Hq > 0) != (s->Hk > 0) || (s->Hk > 0 && s->Hq % s->Hk)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->sequences > 0 && s->B != 1) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!isfinite(s->scale)) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (s->dtype != FLAREPP_BF16 || s->Dk % 8 || s->Dv % 8 || s->Dk > kMaxDim || s->Dv > kMaxDim)
        return FLAREPP_ERR_UNSUPPORTED;
    // tokens, and the units of work that they make, are counted in 31 bits
    const int64_t n = s->sequences ? s->sequences : s->B;
    if (s->N > INT32_MAX - 256 || s->Hq > 65535 || n > INT32_MAX / 64) return FLAREPP_ERR_UNSUPPORTED;
    if (n * (s->sequences ? 1 : s->N / kDecayChunk + 1) > (INT32_MAX - (1 << 20)) / (s->Hq ? s->Hq : 1))
        return FLAREPP_ERR_UNSUPPORTED;
    if (s->sequences && n * (1 + kDecayFront) + s->N / kDecayChunk > (INT32_MAX - (1 << 20)) / (s->Hq ? s->Hq : 1))
        return FLAREPP_ERR_UNSUPPORTED;
    return FLAREPP_OK;
}

bool nothing(const flarepp_decay_shape& s) { return s.B == 0 || s.Hq == 0; }
size_t state_bytes(const flarepp_decay_shape& s) {
    return (size_t)(s.sequences ? s.sequences : s.B) * s.Hq * s.Dk * s.Dv * 4;
}

// An operand: there, aligned, with strides that TMA takes (16 bytes, below 2^40); rows that do not overlap.
flarepp_status check_heads(const flarepp_heads* t, const HeadDims& d, bool out) {
    if (!t) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (empty(d)) return FLAREPP_OK;
    if (!t->data || !aligned16(t->data) || !strides_ok(*t, d)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const int64_t n[3] = {d.B, d.H, d.N}, s[3] = {t->stride_b, t->stride_h, t->stride_n};
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (s[i] % 8) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (s[i] >= int64_t(1) << 38) return FLAREPP_ERR_UNSUPPORTED;
    }
    if (d.N > 1 && t->stride_n < d.D) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (out && !apart_within(*t, d)) return FLAREPP_ERR_INVALID_ARGUMENT;
    return FLAREPP_OK;
}

struct Tensor {
    const flarepp_heads* t;
    HeadDims d;
    bool out;
};

// Every tensor of a call by itself, and what it writes apart from everything else.
flarepp_status check_tensors(const Tensor* t, int n, const Span* outs, int n_outs, const Span* ins,
                             int n_ins) {
    for (int i = 0; i < n; ++i) {
        const flarepp_status bad = check_heads(t[i].t, t[i].d, t[i].out);
        if (bad != FLAREPP_OK) return bad;
    }
    for (int i = 0; i < n; ++i) {
        const Span a = span_of(*t[i].t, t[i].d);
        for (int j = 0; j < n_outs; ++j)
            if (overlaps(a.p, a.bytes, outs[j].p, outs[j].bytes)) return FLAREPP_ERR_INVALID_ARGUMENT;
        if (!t[i].out) continue;
        for (int j = 0; j < n_ins; ++j)
            if (overlaps(a.p, a.bytes, ins[j].p, ins[j].bytes)) return FLAREPP_ERR_INVALID_ARGUMENT;
        for (int j = 0; j < n; ++j)
            if (j != i && (!t[j].out || j < i) && !empty(t[i].d) && !empty(t[j].d) &&
                !apart(*t[i].t, t[i].d, *t[j].t, t[j].d))
                return FLAREPP_ERR_INVALID_ARGUMENT;
    }
    return FLAREPP_OK;
}

bool words_ok(const void* a, const void* b, const void* c, const void* d, const void* e) {
    return aligned4(a) && aligned4(b) && aligned4(c) && aligned4(d) && aligned4(e);
}

// Sequences without tokens: the state goes on as it came.
flarepp_status pass_state(const flarepp_decay_shape& s, const float* from, float* to, cudaStream_t st) {
    if (!to || from == to) return FLAREPP_OK;
    const size_t n = state_bytes(s);
    const cudaError_t e = from ? cudaMemcpyAsync(to, from, n, cudaMemcpyDeviceToDevice, st)
                               : cudaMemsetAsync(to, 0, n, st);
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

struct Call {
    const flarepp_heads *Q, *K, *V, *Y, *dY, *dQ, *dK, *dV;
    const float* log_decay;
    const int32_t* offsets;
    const float *state, *dstate_out;
    float *state_out, *dstate;
    int32_t* status;
};

flarepp_status attention(const flarepp_decay_shape* shape, bool back, const Call& c, void* workspace,
                         size_t workspace_bytes, cudaStream_t st) {
    const flarepp_status bad = check_shape(shape);
    if (bad != FLAREPP_OK) return bad;
    const flarepp_decay_shape s = *shape;
    if (nothing(s)) return FLAREPP_OK;
    if (!words_ok(c.log_decay, c.offsets, c.state, c.dstate_out, c.status) || !aligned4(c.state_out) ||
        !aligned4(c.dstate))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    if (!c.log_decay || (s.sequences > 0) != (c.offsets != nullptr)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const HeadDims q{s.B, s.Hq, s.N, s.Dk, 2}, k{s.B, s.Hk, s.N, s.Dk, 2}, v{s.B, s.Hk, s.N, s.Dv, 2},
        y{s.B, s.Hq, s.N, s.Dv, 2};
    const DecayPlan plan = decay_plan(s, back);
    const size_t sb = state_bytes(s);
    // a state that goes on in place is no overlap: each of its values is read before it is written
    float* out_state = back ? c.dstate : c.state_out;
    const float* in_state = back ? c.dstate_out : c.state;
    const Span outs[3] = {{out_state, sb}, {s.N ? workspace : nullptr, plan.total}, {c.status, 4}};
    const Span ins[4] = {{c.log_decay, (size_t)s.Hq * 4},
                         {c.offsets, (size_t)(s.sequences + 1) * 4},
                         {c.state, sb},
                         {c.dstate_out, sb}};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j) {
            if (i == 0 && ins[j].p == in_state && in_state == out_state) continue;
            if (overlaps(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes))
                return FLAREPP_ERR_INVALID_ARGUMENT;
        }
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
                return FLAREPP_ERR_INVALID_ARGUMENT;
    }
    flarepp_status r;
    if (back) {
        const Tensor t[7] = {{c.Q, q, false},  {c.K, k, false}, {c.V, v, false}, {c.dY, y, false},
                             {c.dQ, q, true},  {c.dK, k, true}, {c.dV, v, true}};
        r = check_tensors(t, 7, outs, 3, ins, 4);
    } else {
        const Tensor t[4] = {{c.Q, q, false}, {c.K, k, false}, {c.V, v, false}, {c.Y, y, true}};
        r = check_tensors(t, 4, outs, 3, ins, 4);
    }
    if (r != FLAREPP_OK) return r;
    if (s.N == 0) return pass_state(s, in_state, out_state, st);
    if (plan.total && (!workspace || (uintptr_t)workspace % 256 || workspace_bytes < plan.total))
        return FLAREPP_ERR_WORKSPACE;
    char* ws = (char*)workspace;
    cudaError_t e = cudaSuccess;
    if (s.sequences) {
        e = decay_cut(s, plan, c.offsets, ws, c.status, st);
        const flarepp_heads* y_of[3] = {back ? c.dQ : c.Y, back ? c.dK : nullptr, back ? c.dV : nullptr};
        const HeadDims d_of[3] = {back ? q : y, k, v};
        for (int i = 0; i < 3 && e == cudaSuccess; ++i)
            if (y_of[i] && (i == 0 || s.Hq == s.Hk))
                e = decay_blank(s, plan, ws, *y_of[i], d_of[i].H, d_of[i].D, st);
    }
    if (e != cudaSuccess) return FLAREPP_ERR_CUDA;
    DecayWalk w{};
    w.shape = &s;
    w.log_decay = c.log_decay;
    w.status = c.status;
    const DecayOperand oq{c.Q, s.Hq}, ok{c.K, s.Hk}, ov{c.V, s.Hk}, og{c.dY, s.Hq};
    if (!back) {
        w.Da = s.Dk, w.Dv = s.Dv;
        w.x = oq, w.a = ok, w.v = ov, w.y = c.Y;
        w.state = c.state, w.state_out = c.state_out;
        e = decay_walk(plan, ws, w, st);
        return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
    }
    // dq_t = scale S_t dy_t: a walk with keys and values (and the state's sides) exchanged
    w.Da = s.Dv, w.Dv = s.Dk;
    w.x = og, w.a = ov, w.v = ok, w.y = c.dQ;
    w.state = c.state, w.turned = 1;
    e = decay_walk(plan, ws, w, st);
    // dv_t = G_t^T k_t and dk_t = G_t v_t, with G the state of a walk from the end
    float* sums = s.Hq != s.Hk ? (float*)(ws + plan.off_sums) : nullptr;
    w.back = 1;
    w.state = c.dstate_out;
    if (e == cudaSuccess) {
        w.Da = s.Dv, w.Dv = s.Dk;
        w.x = ov, w.a = og, w.v = oq, w.y = c.dK, w.y32 = sums, w.turned = 1;
        e = decay_walk(plan, ws, w, st);
    }
    if (e == cudaSuccess && sums) {
        e = decay_group_sum(s, sums, *c.dK, s.Dk, st);
        if (e == cudaSuccess && s.sequences) e = decay_blank(s, plan, ws, *c.dK, s.Hk, s.Dk, st);
    }
    if (e == cudaSuccess) {
        w.Da = s.Dk, w.Dv = s.Dv;
        w.x = ok, w.a = oq, w.v = og, w.y = c.dV, w.y32 = sums, w.turned = 0, w.again = 1;
        w.state_out = c.dstate;
        e = decay_walk(plan, ws, w, st);
    }
    if (e == cudaSuccess && sums) {
        e = decay_group_sum(s, sums, *c.dV, s.Dv, st);
        if (e == cudaSuccess && s.sequences) e = decay_blank(s, plan, ws, *c.dV, s.Hk, s.Dv, st);
    }
    return e == cudaSuccess ? FLAREPP_OK : FLAREPP_ERR_CUDA;
}

flarepp_status step(const flarepp_decay_shape* shape, const flarepp_heads* Q, const flarepp_heads* K,
                    const flarepp_heads* V, const float* log_decay, float* state, const flarepp_heads* Y,
                    int32_t* status, cudaStream_t st) {
    const flarepp_status bad = check_shape(shape);
    if (bad != FLAREPP_OK) return bad;
    const flarepp_decay_shape s = *shape;
    if (s.N != 1 || s.sequences) return FLAREPP_ERR_INVALID_ARGUMENT;
    if (nothing(s)) return FLAREPP_OK;
    if (!log_decay || !state || !aligned4(log_decay) || !aligned16(state) || !aligned4(status))
        return FLAREPP_ERR_INVALID_ARGUMENT;
    const HeadDims q{s.B, s.Hq, 1, s.Dk, 2}, k{s.B, s.Hk, 1, s.Dk, 2}, v{s.B, s.Hk, 1, s.Dv, 2},
        y{s.B, s.Hq, 1, s.Dv, 2};
    const Span outs[2] = {{state, state_bytes(s)}, {status, 4}};
    const Span ins[1] = {{log_decay, (size_t)s.Hq * 4}};
    if (!disjoint(outs, 2, ins, 1)) return FLAREPP_ERR_INVALID_ARGUMENT;
    const Tensor t[4] = {{Q, q, false}, {K, k, false}, {V, v, false}, {Y, y, true}};
    const flarepp_status r = check_tensors(t, 4, outs, 2, ins, 1);
    if (r != FLAREPP_OK) return r;
    return decay_step(s, *Q, *K, *V, log_decay, state, *Y, status, st) == cudaSuccess ? FLAREPP_OK
                                                                                     : FLAREPP_ERR_CUDA;
}

size_t workspace_bytes_of(const flarepp_decay_shape* s, bool back) {
    if (check_shape(s) != FLAREPP_OK || nothing(*s) || s->N == 0) return 0;
    return decay_plan(*s, back).total;
}

}  // namespace
}  // namespace flarepp

extern "C" {

size_t flarepp_decay_attention_workspace_bytes(const flarepp_decay_shape* shape) {
    return flarepp::workspace_bytes_of(shape, false);
}

flarepp_status flarepp_decay_attention_fwd(const flarepp_decay_shape* shape, const flarepp_heads* Q,
                                           const flarepp_heads* K, const flarepp_heads* V,
                                           const float* log_decay, const int32_t* offsets,
                                           const float* state, const flarepp_heads* Y, float* state_out,
                                           void* workspace, size_t workspace_bytes, int32_t* status,
                                           void* stream) {
    flarepp::Call c{};
    c.Q = Q, c.K = K, c.V = V, c.Y = Y;
    c.log_decay = log_decay, c.offsets = offsets;
    c.state = state, c.state_out = state_out;
    c.status = status;
    return flarepp::attention(shape, false, c, workspace, workspace_bytes, (cudaStream_t)stream);
}

size_t flarepp_decay_attention_bwd_workspace_bytes(const flarepp_decay_shape* shape) {
    return flarepp::workspace_bytes_of(shape, true);
}

flarepp_status flarepp_decay_attention_bwd(const flarepp_decay_shape* shape, const flarepp_heads* Q,
                                           const flarepp_heads* K, const flarepp_heads* V,
                                           const float* log_decay, const int32_t* offsets,
                                           const float* state, const flarepp_heads* dY,
                                           const float* dstate_out, const flarepp_heads* dQ,
                                           const flarepp_heads* dK, const flarepp_heads* dV,
                                           float* dstate, void* workspace, size_t workspace_bytes,
                                           int32_t* status, void* stream) {
    flarepp::Call c{};
    c.Q = Q, c.K = K, c.V = V, c.dY = dY, c.dQ = dQ, c.dK = dK, c.dV = dV;
    c.log_decay = log_decay, c.offsets = offsets;
    c.state = state, c.dstate_out = dstate_out, c.dstate = dstate;
    c.status = status;
    return flarepp::attention(shape, true, c, workspace, workspace_bytes, (cudaStream_t)stream);
}

flarepp_status flarepp_decay_attention_step(const flarepp_decay_shape* shape, const flarepp_heads* Q,
                                            const flarepp_heads* K, const flarepp_heads* V,
                                            const float* log_decay, float* state,
                                            const flarepp_heads* Y, int32_t* status, void* stream) {
    return flarepp::step(shape, Q, K, V, log_decay, state, Y, status, (cudaStream_t)stream);
}

}  // extern "C"
