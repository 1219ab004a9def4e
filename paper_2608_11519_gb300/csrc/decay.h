// Declarations shared by the translation units of the decay attention (not installed).
#pragma once
#include "flarepp_internal.h"
#include "heads.h"

namespace flarepp {

// A head's decay as a base-2 logarithm per token, and whether it was one. -inf becomes a number that
// leaves nothing of the token before (2^-1e6 = 0) and may be multiplied by 0.
__device__ __forceinline__ float decay_log2(float log_decay, bool* bad) {
    if (log_decay > 0.f) {
        *bad = true;
        return 0.f;
    }
    if (!(log_decay <= 0.f)) *bad = true;
    return log_decay > -1e6f ? log_decay * 1.44269504f : -1e6f;
}
// Whether nothing is left of the token before (2^lg is 0 in float32): then nothing is left of what is not finite
// either, which a product with 0 would keep.
__device__ __forceinline__ bool forgets(float lg) { return lg <= -150.f; }

constexpr int kDecayChunk = 128;  // tokens
// A packed sequence's head counts as so many chunks more than it has, in front: what it takes to begin with it
// and to end. (At least one, so that an empty sequence has a place. Training on 45 sequences of 8 heads in
// 131,072 tokens, some of a chunk or two: 785 us without, 733 with one, 699 with two, 705 with three.)
constexpr int kDecayFront = 2;

// One walk over the sequences (tc_decay.cu): for every query head, from the state S [Da, Dv],
//   forward:   S_t = g S_(t-1) + a_t v_t^T,  y_t = scale x_t S_t
//   backward:  the sequences from their ends, and S enters undecayed and leaves decayed:
//              S_t = g S_(t+1) + scale a_t v_t^T (no g for the first),  y_t = x_t S_t
// with x, a [.., N, Da], v, y [.., N, Dv]. The head of an operand is the query head / its group.
struct DecayOperand {
    const flarepp_heads* t;
    int64_t heads;
};
struct DecayWalk {
    const flarepp_decay_shape* shape;
    int64_t Da, Dv;
    int back;
    DecayOperand x, a, v;
    const flarepp_heads* y;  // bf16 [B, Hq, N, Dv], or
    float* y32;              // dense float32
    const float* log_decay;
    // states between calls, [sequences][Hq] of Da x Dv or (turned) Dv x Da; NULL: zeros, not kept
    const float* state;
    float* state_out;
    int turned;
    // the walk before this one had the same state, turned: what it found in front of cut sequences' parts holds
    int again;
    int32_t* status;
};

// How the walk is shared among the blocks (tc_decay.cu), and the workspace that goes with it.
struct DecayPlan {
    int64_t sequences, chunks;  // chunks of a sequence (the longest possible one)
    bool whole;                 // whether no sequence is cut
    int64_t blocks, share;      // share: heads or chunks of a block, 0 if the lengths tell
    size_t off_first, off_cuts, off_starts, off_left, off_slots, off_sums, total;
};
DecayPlan decay_plan(const flarepp_decay_shape& s, bool backward);

// Packed sequences: the cuts (checked), the places before each and the blocks' first places into the workspace.
cudaError_t decay_cut(const flarepp_decay_shape& s, const DecayPlan& p, const int32_t* offsets, char* ws,
                      int32_t* status, cudaStream_t st);
// The rows that no sequence holds become 0.
cudaError_t decay_blank(const flarepp_decay_shape& s, const DecayPlan& p, char* ws, const flarepp_heads& y,
                        int64_t heads, int64_t D, cudaStream_t st);
cudaError_t decay_walk(const DecayPlan& p, char* ws, const DecayWalk& w, cudaStream_t st);
// y[b][k] = sum over the group's query heads of the float32 sums[b][h]
cudaError_t decay_group_sum(const flarepp_decay_shape& s, const float* sums, const flarepp_heads& y, int64_t D,
                            cudaStream_t st);
cudaError_t decay_step(const flarepp_decay_shape& s, const flarepp_heads& Q, const flarepp_heads& K,
                       const flarepp_heads& V, const float* log_decay, float* state,
                       const flarepp_heads& Y, int32_t* status, cudaStream_t st);

}  // namespace flarepp
