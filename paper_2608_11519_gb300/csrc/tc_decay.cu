// The walk of the decay attention over a sequence (tcgen05 / TMEM / TMA): y_t = x_t S_t with
// S_t = g S_(t-1) + a_t v_t^T, in chunks of 128 tokens. Within a chunk, from the state S in front of it,
//   Y = (X A^T o W) V + r o (X S),   S' = g^n S + A^T (w o V)
// with W_ij = g^(i-j) for j <= i (0 above), r_i = g^(i+1), w_j = g^(n-1-j): four products of 128 rows. The
// same walk from the sequence's end makes the gradients of keys and values (DecayWalk says how).
//
// The floor is bytes at every width: a chunk reads three tiles and writes one, 64 KB at 64 channels, 1.45 us of
// an SM's share of HBM. So one block walks a sequence of one head, with the state staying in TMEM, and
// nothing is read twice; where heads and sequences do not fill the SMs evenly, sequences are cut, and a
// first walk (only A and V, only S, only in front of the cuts) and a join over the blocks find the states
// there. What bounds it is shared memory and the state's way round. By count a chunk's products, whose operands
// are read from it, its tiles, decayed values and state move 580 KB through it at 128 channels, 4,500 of the
// 6,300 cycles that a chunk takes (no counter has the tensor pipe's reads; threads' accesses alone are 23 % of
// it); of keys and values of 64 channels it takes 3,800, of 128 and 64 5,000, of 64 and 128 6,000. And a
// chunk's state is scaled, multiplied and added to before the next one's. 4 x 32 heads of 8,192 tokens and 128 channels take 203 us (3.3 TB/s of what has to move), the
// gradients of 8 heads of 131,072 tokens, 64 and 128 channels, 664 (HBM at 54 to 68 % in each of the walks).
//
// W o (X A^T) is rounded to bf16 as an operand, w o V and S are two bf16 each (Cfg says why and where not); sums,
// states and what r multiplies are float32.
//
// Roles (24 warps, a block an SM): warp 0 loads tiles (A, X, V of each chunk, a ring of each), warps 1 and 2 issue the
// products, warps 4 to 11 make W o (X A^T), warps 12 to 15 write Y, warps 16 to 19 keep the state, warps 20 to
// 23 make w o V. A chunk passes through them like through a pipeline; the longest way round is
// the state's (scale it, add to it). Every wait is bounded.
#include "decay.h"
#include "tc_linear_common.cuh"

namespace flarepp {
namespace {

constexpr int kThreads = 768;
constexpr int kChunk = kDecayChunk;
constexpr int kAtomBytes = kChunk * 128;  // 128 tokens of 64 channels
constexpr size_t kWsAlign = 256;

// Where an operand's values are, for what is not loaded as tiles; in values.
struct Source {
    const __nv_bfloat16* t;
    int64_t b, h, n;
};

struct Walk {
    int Hq, N, Da, Dv;
    int back;
    int gx, ga, gv;       // query heads that share a head of x, a, v
    int mx, ma, mv;       // whether a batch element has its own
    // The list of all sequences' heads' chunks in the order in which they are walked (or of the sequences'
    // heads, where none is cut), of which every block takes `share` places.
    int whole;            // the list's places are sequences' heads
    int sequences, chunks;  // chunks of a sequence, if they are all alike
    int share;            // 0: from the list's length
    const int* cuts;      // packed sequences' first tokens, else NULL
    const int* first;     // places of the sequences before each, of packed ones
    int front;            // places that a sequence's head has in front of its chunks
    const int2* starts;   // and the sequence and head of every block's first place, where they are cut
    float scale_p, scale_w, scale_r;  // what scores, decayed values and X S are multiplied by
    float gentle;                     // decays above it (base 2, per token) make powers by products along a row
    int lead;                         // r_i = g^(i + lead), w_j = g^(n - lead - j)
    const float* log_decay;
    Source x, a, v;
    void* y;
    int64_t yb, yh, yn;
    int y_f32;
    // States in front of every block's first chunk, [blocks] of Da x Dv, and of its last piece's first if the
    // sequence begins there and goes on in the next block: a copy of `state`, since the block that ends the
    // sequence may have written state_out, which may be the same buffer, before this one begins.
    const float *slots, *begins;
    int slot_row, slot_col;  // their strides
    float* slots_out;     // of the first walk: the state that a block's last piece leaves
    const float* state;   // in front of every sequence, or NULL
    float* state_out;
    int64_t row_stride, col_stride;  // of a state between calls
    Waits waits;
};

// STATES: the first walk over what lies in front of the cuts, which only finds states. (A choice at run time
// in one kernel left it with the shallow rings of the other and both with more code: the long backward took
// 680 us instead of 650.)
template <int TK, int TV, bool STATES>
struct Cfg {
    // TMEM columns: scores (W o scores as bf16 over a half of them), (W o scores) V, X S, the state. Values of
    // up to 64 channels leave room for two sets of scores and of X S. (With what a chunk adds in columns of
    // its own, so that the next one's is multiplied before this one's is added, and (W o scores) V in the
    // scores' other half to make room, a walk took longer: 712 us instead of 677 for the long backward.)
    static constexpr int kSets = TV == 64 ? 2 : 1;
    static constexpr uint32_t kColY = kSets * 128;
    static constexpr uint32_t kColX = kColY + TV;
    static constexpr uint32_t kColS = kColX + kSets * TV;
    static constexpr uint32_t kTmem = 512;
    static_assert(kColS + TV <= kTmem, "TMEM");
    // Shared memory: rings of tiles, as many as there is room for; of A, X and V each, so that a ring's slot
    // only ever holds one kind.
    static constexpr bool kWide = TK == 128 && TV == 128;
    static constexpr int kA = STATES ? (TK == 64 && TV == 64 ? 5 : TV == 64 ? 4 : 3) : TK == 64 && TV == 64 ? 3 : 2;
    static constexpr int kX = kWide || STATES ? 1 : kA, kV = kA;  // (of X no use is made then)
    static constexpr int kTileK = TK * kChunk * 2, kTileV = TV * kChunk * 2;
    // Decayed values and the state go into their products as two bf16 each, the second what the first's
    // rounding left: so a state is as good as its 32 bits but for some 2^-17, and X S as good as the state
    // (with both widths above 64 there is no room for the state's second: X S then carries its rounding).
    // Decayed values pass in parts of a chunk's tokens, so that some are made while others are multiplied.
    static constexpr bool kStTwo = !kWide;
    static constexpr int kParts = TV == 128 ? 4 : TK == 128 ? 2 : 1;
    static constexpr int kBufs = TV == 128 ? (kWide ? 2 : 4) : 2;
    static constexpr int kPart = kChunk / kParts;      // tokens
    static constexpr int kVw = kPart * TV * 2;         // bytes of one of the two
    static constexpr int kSt = STATES ? 0 : TK * TV * 2;
    static constexpr int kOffX = kA * kTileK, kOffV = kOffX + (STATES ? 0 : kX) * kTileK, kOffVw = kOffV + kV * kTileV;
    static constexpr int kOffSt = kOffVw + kBufs * 2 * kVw;
    static constexpr int kBody = kOffSt + (kStTwo ? 2 : 1) * kSt;
    // barriers
    static constexpr int kFullA = 0, kFullX = kA, kFullV = kFullX + kX, kEmptyA = kFullV + kV,
                         kEmptyX = kEmptyA + kA, kEmptyV = kEmptyX + kX, kOut = kEmptyV + kV,
                         kVFull = kOut + kV, kVFree = kVFull + kBufs, kOther = kVFree + kBufs;
    static constexpr int kBars = kOther + 18;
    static constexpr int kSmem = 1024 + kBody + kBars * 8 + 16;
    static_assert(kSmem <= kMaxSmem, "shared memory");
};

// A part of a sequence of one head, as a block walks it: chunks c0 to c1 of `total`, counted as walked.
struct Piece {
    int sequence, h;
    int start, rows;  // the sequence's tokens
    int c0, c1, total;
    int begun;        // whether the block before has begun with it
};
// Where a block is in its part of the list.
struct Feed {
    int at, end;      // places
    int sequence, h;  // of the next place
};

__device__ __forceinline__ int tokens_of(const Walk& p, int sequence, int& start) {
    start = p.cuts ? p.cuts[sequence] : 0;
    return p.cuts ? p.cuts[sequence + 1] - start : p.N;
}
// The places before a sequence's first head, and of each of its heads.
__device__ __forceinline__ int places_before(const Walk& p, int sequence) {
    if (p.whole) return sequence * p.Hq;
    return (p.cuts ? p.first[sequence] : sequence * p.chunks) * p.Hq;
}
__device__ __forceinline__ int places_of(const Walk& p, int sequence) {
    if (p.whole) return 1;
    return p.cuts ? p.first[sequence + 1] - p.first[sequence] : p.chunks;
}
__device__ __noinline__ void begin_feed(const Walk& p, int block, int blocks, Feed& f) {
    const int all = places_before(p, p.sequences);
    const int share = p.share ? p.share : (all + blocks - 1) / blocks;
    f.at = min(block * share, all);  // (at most 2^31: the host has seen to it)
    f.end = min(f.at + share, all);
    if (f.at >= f.end) return;
    if (p.starts) {  // (a search of the packed sequences by every block would be one load after another)
        const int2 s = p.starts[block];
        f.sequence = s.x;
        f.h = s.y;
    } else {
        const int head = f.at / (p.whole ? 1 : p.chunks);
        f.sequence = head / p.Hq;
        f.h = head - f.sequence * p.Hq;
    }
}
// The next piece; false after the last.
__device__ __noinline__ bool next_piece(const Walk& p, Feed& f, Piece& x) {
    if (f.at >= f.end) return false;
    const int each = places_of(p, f.sequence);
    const int base = places_before(p, f.sequence) + f.h * each;
    x.sequence = f.sequence;
    x.h = f.h;
    x.rows = tokens_of(p, f.sequence, x.start);
    x.total = (x.rows + kChunk - 1) / kChunk;
    x.c0 = p.whole ? 0 : min(max(f.at - base - p.front, 0), x.total);
    x.c1 = p.whole ? x.total : min(max(f.end - base - p.front, 0), x.total);
    x.begun = f.at > base;
    f.at = base + each;
    if (++f.h == p.Hq) {
        f.h = 0;
        ++f.sequence;
    }
    return true;
}
// The pieces of a block's walk: all of its part of the list, or, for the states alone, the last
// one if its sequence goes on in the next block.
template <bool STATES>
__device__ __forceinline__ bool next_walked(const Walk& p, Feed& f, Piece& x) {
    while (next_piece(p, f, x))
        if (!STATES || x.c1 < x.total) return true;
    return false;
}
// The first token of chunk c, and its tokens.
__device__ __forceinline__ int chunk_at(const Walk& p, const Piece& x, int c, int& rows) {
    const int k = p.back ? x.total - 1 - c : c;
    rows = min(kChunk, x.rows - k * kChunk);
    return x.start + k * kChunk;
}
// Whether a chunk's outputs are stored as whole tiles: what lies behind a packed sequence is another's (behind
// the last token of others TMA leaves it).
__device__ __forceinline__ bool staged(const Walk& p, int rows) {
    return !p.y_f32 && (rows == kChunk || !p.cuts);
}
__device__ __forceinline__ float head_decay(const Walk& p, int h, bool record) {
    bool bad = false;
    const float lg = decay_log2(p.log_decay[h], &bad);
    if (bad && record) record_status(p.waits.status, FLAREPP_ERR_INVALID_ARGUMENT);
    return lg;
}

// warp_wait whose tries sleep in the barrier (up to a millisecond each) instead of polling: most of a block's
// warps wait most of the time. What follows a first try in vain is kept out of line: in line, in some thirty
// places, it was half of the kernel's code, and instructions came late.
__device__ __noinline__ bool wait_longer(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                         uint64_t limit_ns, int* status) {
    const uint64_t t0 = globaltimer_ns();
    const uint32_t nap = limit_ns < 4000000u ? (uint32_t)(limit_ns / 4) : 1000000u;
    while (!mbar_sleep_wait(bar, parity, nap)) {
        if (*abort_flag) return false;
        if (globaltimer_ns() - t0 > limit_ns) {
            *abort_flag = 1;
            record_status(status, FLAREPP_ERR_TIMEOUT);
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                         const Waits& w) {
    bool got = mbar_sleep_wait(bar, parity, 1000000u);
    if (__all_sync(0xffffffffu, got)) return true;
    if (!got) got = wait_longer(bar, parity, abort_flag, w.limit_ns, w.status);
    return __all_sync(0xffffffffu, got);
}

template <int T>
__device__ __forceinline__ void load_rows(uint32_t dst, const CUtensorMap* m, int token, int head, int b,
                                          uint32_t bar) {
#pragma unroll
    for (int k = 0; k < T / 64; ++k) tma_load_4d(dst + k * kAtomBytes, m, 64 * k, token, head, b, bar);
}

// The operands of a product lie in tiles of 128-byte rows, swizzled. The upper halves of their descriptors
// (8 rows every 1,024 bytes, version, swizzle) are all the same, the lower ones a start and a stride:
// with the upper half a constant a step costs one addition, and a chunk's products are issued in a few
// hundred cycles (whole descriptors took three times that, and their issue was what bounded a chunk).
constexpr uint32_t kUpper = (1024u >> 4) | (1u << 14) | ((uint32_t)kSw128 << 29);
__device__ __forceinline__ uint32_t lower(uint32_t start, uint32_t stride) {
    return (start >> 4) | (stride >> 4) << 16;
}
// what step s (16 contraction values) adds: of a tile whose channels are contracted, whose rows are
__device__ __forceinline__ uint32_t by_channel(int s) { return (uint32_t)(s / 4 * kAtomBytes + s % 4 * 32) >> 4; }
__device__ __forceinline__ uint32_t by_row(int s) { return (uint32_t)(s * 16 * 128) >> 4; }

__device__ __forceinline__ void product_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                           uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 x, {%1, %4};\n\tmov.b64 y, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(kUpper), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                           uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 y, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}\n" ::"r"(d),
        "r"(a), "r"(b), "r"(idesc), "r"(kUpper), "r"(accumulate)
        : "memory");
}

// Two values as a pair of bf16, and a pair of what its rounding leaves.
__device__ __forceinline__ uint32_t split_pair(uint64_t v, uint32_t& rest) {
    const uint32_t hi = pack_bf16x2(v);
    rest = pack_bf16x2(fma2(unpack_bf16x2(hi), pair(-1.f, -1.f), v));
    return hi;
}
// 8 bf16 values times w, in two
__device__ __forceinline__ uint4 scaled(uint4 d, float w, uint4& rest) {
    const uint64_t w2 = pair(w, w);
    uint4 hi;
    hi.x = split_pair(mul2(unpack_bf16x2(d.x), w2), rest.x);
    hi.y = split_pair(mul2(unpack_bf16x2(d.y), w2), rest.y);
    hi.z = split_pair(mul2(unpack_bf16x2(d.z), w2), rest.z);
    hi.w = split_pair(mul2(unpack_bf16x2(d.w), w2), rest.w);
    return hi;
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// tcgen05.wait::ld that names the 8 registers of a load before it
__device__ __forceinline__ void wait_ld8(uint32_t* r) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7])
                 :
                 : "memory");
}

// Of 16 bf16 values in 8 words those whose bit is set; the others become 0, whatever they were. The
// shifts put the bits of two values that share a byte into its top place, from where a byte permute
// spreads them over a word.
__device__ __forceinline__ void keep_keys(uint32_t* w, uint32_t bits) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int b = j / 4, i = 2 * j % 8;  // values 8 b + i and the next
        uint32_t mask;                       // a selector of 8 and more takes the byte's top bit eight times
        asm("prmt.b32 %0, %1, %2, %3;"
            : "=r"(mask)
            : "r"(bits << (7 - i)), "r"(bits << (6 - i)), "r"(0x1100u * (12 + b) + 0x0011u * (8 + b)));
        w[j] &= mask;
    }
}

// What a head without memory has in TMEM or in a tile of what it does not remember becomes 0, whatever it was. Out of
// line: in the loops over columns that every head takes, a choice took up to 6 % of a walk.
__device__ __noinline__ void clear_columns(uint32_t at, int columns, bool keep) {
    for (int c = 0; c < columns; c += 16) {
        uint32_t r[16];
        tmem_ld16(at + c, r);
        tmem_wait_ld16(r);
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = keep ? r[j] : 0u;
        tmem_st16(at + c, r);
    }
    tmem_wait_st();
}
template <int T>
__device__ __noinline__ void clear_rows(uint8_t* tile, int thread, int but) {
    for (int e = thread; e < 8 * kChunk; e += 128)
        if (e / 8 != but)
#pragma unroll
            for (int t = 0; t < T / 64; ++t)
                *reinterpret_cast<uint4*>(tile + 16 * e + t * kAtomBytes) = make_uint4(0, 0, 0, 0);
}

// (W o X A^T) V has every token of a chunk in every output, those that do not count with a weight of 0, and 0 times an
// infinity or NaN is NaN. So where a warp's outputs from the chunk are NaN (TMEM tells with the load), its tokens' are
// made again one product after another, of the tokens that count alone: what is no number then reaches what it
// reaches in the recurrence. The weights, rounded as they were, take the place of the outputs in TMEM, two in a word.
// Such a chunk takes 0.3 ms at 64 channels, 0.75 at 128; others no more than before but for the code's place in
// registers: 3 % of the packed training, 4 of the prefill, none of the long backward. (With eight keys in flight it
// took half, but all others 1 to 6 % more; a look at the values before their product took 4 to 15 % of every walk,
// whichever warps did it.)
__device__ __forceinline__ const __nv_bfloat16* source(const Source& s, int b, int own_batch, int h, int group,
                                                       int64_t token) {
    return s.t + (int64_t)b * own_batch * s.b + (int64_t)(group ? h / group : 0) * s.h + token * s.n;
}
__device__ __forceinline__ void eight(const __nv_bfloat16* t, float* v) {
    const uint4 d = *reinterpret_cast<const uint4*>(t);
    const uint32_t w[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(w[j] << 16);
        v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
}
// One warp: lane's token i of the chunk that begins at `token`; `mine`: whether its outputs are written, into the tile
// row `stage` or to p.y + to; y_at, x_at: columns of outputs and of X S, which has the factor f.
__device__ __forceinline__ void outputs_again(const Walk& p, uint32_t y_at, uint32_t x_at, int b, int h, int token,
                                           int rows, int i, bool mine, float lg, float f, uint8_t* stage,
                                           int64_t to) {
    const bool alone = forgets(lg);
    auto counts = [&](int key) { return key < rows && (key == i || (!alone && (p.back ? key > i : key < i))); };
    const __nv_bfloat16* x = source(p.x, b, p.mx, h, p.gx, token + min(i, rows - 1));
    const __nv_bfloat16* a = source(p.a, b, p.ma, h, p.ga, token);
    const __nv_bfloat16* v = source(p.v, b, p.mv, h, p.gv, token);
#pragma unroll 1
    for (int key = 0; key < rows; key += 2) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (!counts(key + k)) continue;
            const __nv_bfloat16* row = a + (int64_t)(key + k) * p.a.n;
#pragma unroll 1
            for (int d = 0; d < p.Da; d += 8) {
                float u[8], w[8];
                eight(x + d, u);
                eight(row + d, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[k] = fmaf(u[j], w[j], s[k]);
            }
            s[k] *= exp2f(lg * abs(key + k - i)) * p.scale_p;
        }
        __syncwarp();
        tmem_st1(y_at + key / 2, bf16_pair(s[0], s[1]));
    }
    tmem_wait_st();
#pragma unroll 1
    for (int c = 0; c < p.Dv; c += 8) {
        float y[8];
        uint32_t s[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = 0.f;
#pragma unroll 1
        for (int key = 0; key < rows; key += 2) {
            const uint32_t w = tmem_ld1(y_at + key / 2);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (!counts(key + k)) continue;
                float u[8];
                eight(v + (int64_t)(key + k) * p.v.n + c, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = fmaf(__uint_as_float(k ? w & 0xffff0000u : w << 16), u[j], y[j]);
            }
            __syncwarp();
        }
        tmem_ld8(x_at + c, s);
        wait_ld8(s);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = fmaf(__uint_as_float(s[j]), f, y[j]);
        if (mine && p.y_f32 && !stage) {
            float4* d = reinterpret_cast<float4*>((float*)p.y + to + c);
            d[0] = make_float4(y[0], y[1], y[2], y[3]);
            d[1] = make_float4(y[4], y[5], y[6], y[7]);
        } else if (mine) {
            uint4* d = stage ? reinterpret_cast<uint4*>(stage + c / 64 * kAtomBytes + 16 * ((c % 64 / 8) ^ (i & 7)))
                             : reinterpret_cast<uint4*>((__nv_bfloat16*)p.y + to + c);
            *d = make_uint4(bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]),
                            bf16_pair(y[6], y[7]));
        }
        __syncwarp();
    }
}

// How many chunks a block walks.
template <bool STATES>
__device__ __noinline__ int count_chunks(const Walk& p) {
    Feed f;
    Piece x;
    int n = 0;
    begin_feed(p, blockIdx.x, gridDim.x, f);
    while (next_walked<STATES>(p, f, x)) n += x.c1 - x.c0;
    return n;
}

__device__ __forceinline__ uint32_t bf16_bits(uint32_t a, uint32_t b) {
    return bf16_pair(__uint_as_float(a), __uint_as_float(b));
}

template <int TK, int TV, bool STATES>
__global__ void __launch_bounds__(kThreads, 1)
    walk_kernel(const __grid_constant__ CUtensorMap tX, const __grid_constant__ CUtensorMap tA,
                const __grid_constant__ CUtensorMap tV, const __grid_constant__ CUtensorMap tY,
                const __grid_constant__ Walk p) {
    using C = Cfg<TK, TV, STATES>;
    constexpr uint32_t kSets = C::kSets;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBody);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t bar0 = smem_u32(bars);
    // Of each but the last two there are two, for even and odd chunks: whoever waits for chunk n's phase must
    // not find that of chunk n + 1 done too, and no barrier's phase n + 2 comes before all have seen n.
    const uint32_t s_ready = bar0 + 8u * C::kOther, p_ready = s_ready + 16, clean = s_ready + 32,
                   u_ready = s_ready + 48, y_ready = s_ready + 64, y_free = s_ready + 80;
    const uint32_t x_ready = s_ready + 96, made = s_ready + 112, b_ready = s_ready + 128, done = s_ready + 136;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kOther; ++s)
            mbar_init(bar0 + 8u * s, s >= C::kEmptyA && s < C::kEmptyV ? 2 : s >= C::kOut && s < C::kVFree ? 128 : 1);
        for (uint32_t s = 0; s < 16; s += 8) {
            mbar_init(s_ready + s, 1);
            mbar_init(p_ready + s, 256);
            mbar_init(clean + s, 128);
            mbar_init(u_ready + s, 1);
            mbar_init(y_ready + s, 1);
            mbar_init(y_free + s, 128);
            mbar_init(x_ready + s, 1);
            mbar_init(made + s, 128);
        }
        mbar_init(b_ready, TK);
        mbar_init(done, 2);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tX);
        prefetch_tmap(&tA);
        prefetch_tmap(&tV);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), C::kTmem);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_trigger();
    pdl_wait();

    Feed feed;
    Piece here;
    const int width = (p.Dv + 15) / 16 * 16;  // columns of the products
    const int steps = (p.Da + 15) / 16;       // steps of a product over Da
    // the barrier of chunk n, and its phase there
    auto of = [](uint32_t bar, uint32_t n) { return bar + 8u * (n & 1); };
    auto wait_chunk = [&](uint32_t bar, uint32_t n) {
        return wait_for(bar + 8u * (n & 1), (n >> 1) & 1, abort_flag, p.waits);
    };
    // a ring's barrier (of `size`, the first at `first`) for its n-th use, and a wait for that use
    auto ring = [&](int first, int size, uint32_t n) { return bar0 + 8u * (first + n % size); };
    auto wait_use = [&](int first, int size, uint32_t n) {
        return wait_for(bar0 + 8u * (first + n % size), n / size & 1, abort_flag, p.waits);
    };
    auto tile_a = [&](uint32_t n) { return smem + n % C::kA * C::kTileK; };
    auto tile_x = [&](uint32_t n) { return smem + C::kOffX + n % C::kX * C::kTileK; };
    auto tile_v = [&](uint32_t n) { return smem + C::kOffV + n % C::kV * C::kTileV; };

    if (warp == 0) {
        // ------------------------------------------------------------ loads: A, X, V
        uint32_t it = 0, n = 0, used_x = 0;  // tiles and chunks; those of X
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (ok && next_walked<STATES>(p, feed, here)) {
            const Piece x = here;
            const int b = p.cuts ? 0 : x.sequence, h = x.h;
            for (int c = x.c0; c < x.c1 && ok; ++c, ++n) {
                int rows;
                const int token = chunk_at(p, x, c, rows);
                auto load = [&](int full, int empty, int size, uint32_t bytes, auto&& issue) {
                    if (n >= (uint32_t)size && !wait_use(empty, size, n - size)) return false;
                    if (elect_one() && !(blockIdx.x == 0 && it == p.waits.withheld)) {
                        mbar_expect_tx(ring(full, size, n), bytes);
                        issue(ring(full, size, n));
                    }
                    __syncwarp();
                    ++it;
                    return true;
                };
                ok = load(C::kFullA, C::kEmptyA, C::kA, C::kTileK, [&](uint32_t bar) {
                    load_rows<TK>(smem_u32(tile_a(n)), &tA, token, p.ga ? h / p.ga : 0, b * p.ma, bar);
                });
                if (ok && !STATES) {
                    ok = load(C::kFullX, C::kEmptyX, C::kX, C::kTileK, [&](uint32_t bar) {
                        load_rows<TK>(smem_u32(tile_x(n)), &tX, token, p.gx ? h / p.gx : 0, b * p.mx, bar);
                    });
                    used_x += ok;
                }
                ok = ok && load(C::kFullV, C::kEmptyV, C::kV, C::kTileV, [&](uint32_t bar) {
                    load_rows<TV>(smem_u32(tile_v(n)), &tV, token, p.gv ? h / p.gv : 0, b * p.mv, bar);
                });
                if (!ok) break;  // (n stays this chunk's)
            }
        }
        if (!ok) {  // wait (bounded) until every copy issued has landed
            const uint64_t t0 = globaltimer_ns();
            const uint32_t per = STATES ? 2 : 3;
            const uint32_t uses[3] = {(it + per - 1) / per, used_x, it / per};
            const int first[3] = {C::kFullA, C::kFullX, C::kFullV}, size[3] = {C::kA, C::kX, C::kV};
            for (int k = 0; k < 3; ++k)
                for (uint32_t u = uses[k] < (uint32_t)size[k] ? 0 : uses[k] - size[k]; u < uses[k]; ++u)
                    while (!mbar_try_wait(ring(first[k], size[k], u), u / size[k] & 1) &&
                           globaltimer_ns() - t0 < kWaitLimitNs) {
                    }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ products: X A^T, and (W o X A^T) V
        // A tile is released by the warps that wait for its last product: a commit of its own
        // for each kept this warp from issuing for hundreds of cycles.
        const uint32_t scores = idesc_bf16_f32(128, 128, false, false);
        const uint32_t outs = idesc_bf16_f32(128, 16, false, true) + ((uint32_t)(width / 8 - 2) << 17);
        const int total = STATES ? 0 : count_chunks<STATES>(p);
        bool ok = true;
        // with two sets the scores of a chunk go ahead of the last chunk's outputs
        for (int m = 0; ok && m < total + (int)kSets - 1; ++m) {
            if (m < total) {
                const uint32_t n = m;
                // (the scores go over the W o scores that an earlier product has read: nothing orders the two
                // but its end)
                ok = wait_use(C::kFullA, C::kA, n) && wait_use(C::kFullX, C::kX, n) &&
                     (n < kSets || wait_chunk(y_ready, n - kSets));
                if (!ok) break;
                tc_fence_after();
                const uint32_t a = lower(smem_u32(tile_a(n)), 16), q = lower(smem_u32(tile_x(n)), 16);
                const uint32_t to = tmem + n % kSets * 128;
                if (elect_one()) {
#pragma unroll
                    for (int s = 0; s < TK / 16; ++s)
                        if (s < steps) product_ss(to, q + by_channel(s), a + by_channel(s), scores, s > 0);
                    mma_commit(of(s_ready, n));
                }
                __syncwarp();
            }
            if (m >= (int)kSets - 1) {
                const uint32_t n = m - (kSets - 1);
                ok = wait_use(C::kFullV, C::kV, n) && wait_chunk(clean, n) && wait_chunk(p_ready, n) &&
                     (n == 0 || wait_chunk(y_free, n - 1));
                if (!ok) break;
                tc_fence_after();
                const uint32_t v = lower(smem_u32(tile_v(n)), kAtomBytes), w = tmem + n % kSets * 128;
                if (elect_one()) {
#pragma unroll
                    for (int s = 0; s < kChunk / 16; ++s)
                        product_ts(tmem + C::kColY, w + s / 4 * 64 + s % 4 * 8, v + by_row(s), outs, s > 0);
                    mma_commit(of(y_ready, n));
                }
                __syncwarp();
            }
        }
        // no product and no arrival of one is in flight when the block ends
        if (elect_one()) mma_commit(done);
        __syncwarp();
        wait_for(done, 0, abort_flag, p.waits);
        if (!ok) linger();
    } else if (warp == 2) {
        // ------------------------------------------------------------ products: X S, then S += A^T (w o V)
        const uint32_t states = idesc_bf16_f32(128, 16, true, true) + ((uint32_t)(width / 8 - 2) << 17);
        const uint32_t outs = idesc_bf16_f32(128, 16, false, true) + ((uint32_t)(width / 8 - 2) << 17);
        const uint32_t s0 = lower(smem_u32(smem + C::kOffSt), TK * 128);
        const uint32_t total = count_chunks<STATES>(p);
        bool ok = true;
        uint32_t g = 0;  // parts
        for (uint32_t n = 0; ok && n < total; ++n) {
            const uint32_t a = lower(smem_u32(tile_a(n)), kAtomBytes), q = lower(smem_u32(tile_x(n)), 16);
            const uint32_t to = tmem + C::kColX + n % kSets * TV;
            auto states_of = [&]() {
                // (where TK is 64, A^T's rows from 64 on are whatever lies behind the tile: they are not used)
#pragma unroll 1
                for (int part = 0; part < C::kParts; ++part, ++g) {
                    if (!wait_use(C::kVFull, C::kBufs, g)) return false;
                    tc_fence_after();
                    const uint32_t v =
                        lower(smem_u32(smem + C::kOffVw + g % C::kBufs * 2 * C::kVw), C::kPart * 128);
                    const uint32_t ap = a + by_row(part * (C::kPart / 16));
                    if (elect_one()) {
#pragma unroll
                        for (int s = 0; s < C::kPart / 16; ++s) {
                            product_ss(tmem + C::kColS, ap + by_row(s), v + by_row(s), states, 1u);
                            product_ss(tmem + C::kColS, ap + by_row(s), v + (C::kVw >> 4) + by_row(s), states, 1u);
                        }
                        mma_commit(ring(C::kVFree, C::kBufs, g));
                        if (part == C::kParts - 1) {
                            if (STATES) {  // nobody else reads A and V
                                mma_commit(ring(C::kEmptyA, C::kA, n));
                                mma_commit(ring(C::kEmptyA, C::kA, n));
                                mma_commit(ring(C::kEmptyV, C::kV, n));
                            } else {
                                mma_commit(of(u_ready, n));
                            }
                        }
                    }
                    __syncwarp();
                }
                return true;
            };
            ok = wait_use(C::kFullA, C::kA, n);
            if (ok && STATES) {
                ok = (n > 0 || wait_for(b_ready, 0, abort_flag, p.waits)) && states_of();
            } else if (ok) {
                ok = wait_use(C::kFullX, C::kX, n) && (n < kSets || wait_chunk(y_free, n - kSets)) &&
                     wait_for(b_ready, n & 1, abort_flag, p.waits);
                if (!ok) break;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int s = 0; s < TK / 16; ++s)
                        if (s < steps) {
                            product_ss(to, q + by_channel(s), s0 + by_row(s), outs, s > 0);
                            if (C::kStTwo)
                                product_ss(to, q + by_channel(s), s0 + (C::kSt >> 4) + by_row(s), outs, 1u);
                        }
                    mma_commit(ring(C::kEmptyX, C::kX, n));
                    mma_commit(of(x_ready, n));
                }
                __syncwarp();
                ok = states_of();
            }
        }
        if (elect_one()) mma_commit(done);
        __syncwarp();
        wait_for(done, 0, abort_flag, p.waits);
        if (!ok) linger();
    } else if (warp == 3) {
        // ------------------------------------------------------------ stores of staged outputs
        // (a barrier a slot, which is released once it is stored: the outputs may be several chunks ahead; the
        // slots' phases count their staged uses alone)
        uint32_t n = 0, phases = 0;
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (ok && !STATES && next_piece(p, feed, here)) {
            const Piece x = here;
            const int b = p.cuts ? 0 : x.sequence, h = x.h;
            for (int c = x.c0; c < x.c1; ++c, ++n) {
                int rows;
                const int token = chunk_at(p, x, c, rows);
                if (!staged(p, rows)) continue;
                const uint32_t slot = n % C::kV;
                ok = wait_for(bar0 + 8u * (C::kOut + slot), phases >> slot & 1, abort_flag, p.waits);
                if (!ok) break;
                phases ^= 1u << slot;
                if (elect_one()) {
                    const uint32_t from = smem_u32(tile_v(n));
#pragma unroll
                    for (int t = 0; t < TV / 64; ++t)
                        if (64 * t < p.Dv) tma_store_4d(&tY, from + t * kAtomBytes, 64 * t, token, h, b);
                    bulk_commit();
                    bulk_wait_read();
                    mbar_arrive(ring(C::kEmptyV, C::kV, n));
                }
                __syncwarp();
            }
        }
        if (elect_one()) bulk_wait_all();
        __syncwarp();
    } else if (warp < 12) {
        // ------------------------------------------------------------ scores
        // Two warps share 32 tokens: one takes the keys 0 to 63, the other 64 to 127, 16 at a time, each
        // writing over columns that it has read itself.
        const int q = warp & 3, half = (warp - 4) >> 2, i = 32 * q + lane;  // the thread's token in the chunk
        const uint32_t at = tmem + ((uint32_t)(32 * q) << 16) + 64 * half;
        // its keys that count: from `low` to before `high`, whole sixteens
        const int edge = min(max(32 * q - 64 * half, 0), 64);
        const int low = p.back ? edge : 0, high = p.back ? 64 : min(max(32 * q + 32 - 64 * half, 0), 64);
        uint32_t n = 0;
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (ok && !STATES && next_piece(p, feed, here)) {
            const Piece x = here;
            const float lg = head_decay(p, x.h, false);
            // Powers of g along the keys, from the gaps of the first two on: times g^2 for each next two keys
            // backwards, times g^-2 forwards. (On the diagonal gaps may be below 0: those keys do not
            // count.) From g = 1/2 on the first power, g^127 at least, is one that float32 holds; below
            // that each takes an exponential of its own. So it does with a scale below 2^-40: the chain begins up to
            // 64 keys in front of those that count, at 2^-77 times the scale, and what float32 does not hold
            // there would be 0 where it counts. A table of powers in shared memory, which the products' operands
            // come from too, took longer than the chain.
            const float way = p.back ? lg : -lg;
            const int gap0 = p.back ? 64 * half + low - i : i - 64 * half - low;
            const bool gentle = lg > p.gentle, alone = forgets(lg);
            const float g2 = gentle ? exp2f(2.f * way) : 1.f;
            const uint64_t next = pair(g2, g2);
            const uint64_t first = pair(exp2f(lg * gap0) * p.scale_p, exp2f(lg * gap0 + way) * p.scale_p);
            for (int c = x.c0; c < x.c1; ++c, ++n) {
                int rows;
                chunk_at(p, x, c, rows);
                const uint32_t from = at + n % kSets * 128;
                ok = wait_chunk(s_ready, n);
                if (!ok) break;
                tc_fence_after();
                if (threadIdx.x == 128) {  // one of two that read A and X
                    mbar_arrive(ring(C::kEmptyA, C::kA, n));
                    mbar_arrive(ring(C::kEmptyX, C::kX, n));
                }
                uint64_t f = first;
#pragma unroll 1
                for (int t = low; t < high; t += 16) {
                    const int key = 64 * half + t;
                    uint32_t r[16], w[8];
                    tmem_ld16(from + t, r);
                    tmem_wait_ld16(r);
                    if (gentle) {
#pragma unroll
                        for (int j = 0; j < 16; j += 2, f = mul2(f, next))
                            w[j / 2] =
                                pack_bf16x2(mul2(pair(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), f));
                    } else {
                        const int gap = p.back ? key - i : i - key;
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            r[j] = __float_as_uint(
                                __uint_as_float(r[j]) *
                                (exp2f(lg * max(p.back ? gap + j : gap - j, 0)) * p.scale_p));
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = bf16_bits(r[2 * j], r[2 * j + 1]);
                    }
                    // on the diagonal, in a chunk that ends early and without memory, what does not count is 0
                    // whatever it was
                    if ((key >> 5) == q || key + 16 > rows || alone) {
                        const int least = p.back || alone ? i - key : 0;
                        const int most = min(p.back && !alone ? 16 : i + 1 - key, rows - key);
                        keep_keys(w, (most >= 16 ? 0xffffu : most <= 0 ? 0u : (1u << most) - 1u) &
                                         (least <= 0 ? ~0u : least >= 16 ? 0u : ~0u << least));
                    }
                    tmem_st8(from + t / 2, w);
                }
                {
                    uint32_t w[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = 0;
#pragma unroll 1
                    for (int t = p.back ? 0 : high; t < (p.back ? low : 64); t += 16)
                        tmem_st8(from + t / 2, w);
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(of(p_ready, n));
            }
        }
    } else if (warp < 16) {
        // ------------------------------------------------------------ outputs
        const int q = warp & 3, i = 32 * q + lane;  // the thread's token in the chunk
        const uint32_t at = tmem + ((uint32_t)(32 * q) << 16);
        uint32_t n = 0;
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (ok && !STATES && next_piece(p, feed, here)) {
            const Piece x = here;
            const int b = p.cuts ? 0 : x.sequence, h = x.h;
            const float lg = head_decay(p, h, false);
            for (int k = x.c0; k < x.c1; ++k, ++n) {
                int rows;
                const int token = chunk_at(p, x, k, rows);
                const int since = p.back ? rows - 1 - i : i;
                const float f = i < rows ? exp2f(lg * (since + p.lead)) * p.scale_r : 0.f;
                const int64_t to = b * p.yb + h * p.yh + (int64_t)(token + i) * p.yn;
                ok = wait_chunk(made, n) && wait_chunk(x_ready, n) && wait_chunk(y_ready, n);
                if (!ok) break;
                tc_fence_after();
                // V has been read, by the warps that decay it and by its product: the outputs go over it, from
                // where whole lines are stored. (Stores of a thread's own row, 16 bytes of 32 lines an
                // instruction, held up the state's through the pipe that they share: 241 us instead of 229
                // for the prefill, when this was chosen.)
                // (without memory the state in front is at most the first token's)
                if (forgets(lg)) clear_columns(at + C::kColX + n % kSets * TV, p.Dv, since + p.lead == 0);
                const bool staging = staged(p, rows);
                uint8_t* stage = tile_v(n) + i * 128;
                if (!staging && threadIdx.x == 384) mbar_arrive(ring(C::kEmptyV, C::kV, n));
                bool no_number = false;
#pragma unroll 1
                for (int c = 0; c < p.Dv; c += 16) {
                    uint32_t y[16], s[16];
                    float most = tmem_ldmaxnan16(at + C::kColY + c, y);
                    tmem_ld16(at + C::kColX + n % kSets * TV + c, s);
                    tmem_wait_ld16(y);
                    tmem_wait_ld16(s);
                    reg_after_wait16(y, most);
                    no_number = no_number || most != most;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        y[j] = __float_as_uint(fmaf(__uint_as_float(s[j]), f, __uint_as_float(y[j])));
                    if (staging) {
                        uint8_t* d = stage + c / 64 * kAtomBytes;
                        const int piece = c % 64 / 8;
                        *reinterpret_cast<uint4*>(d + 16 * (piece ^ (i & 7))) =
                            make_uint4(bf16_bits(y[0], y[1]), bf16_bits(y[2], y[3]), bf16_bits(y[4], y[5]),
                                       bf16_bits(y[6], y[7]));
                        *reinterpret_cast<uint4*>(d + 16 * ((piece + 1) ^ (i & 7))) =
                            make_uint4(bf16_bits(y[8], y[9]), bf16_bits(y[10], y[11]),
                                       bf16_bits(y[12], y[13]), bf16_bits(y[14], y[15]));
                    } else if (i < rows) {
                        const bool both = c + 8 < p.Dv;
                        if (p.y_f32) {
                            uint4* d = reinterpret_cast<uint4*>((float*)p.y + to + c);
                            d[0] = make_uint4(y[0], y[1], y[2], y[3]);
                            d[1] = make_uint4(y[4], y[5], y[6], y[7]);
                            if (both) d[2] = make_uint4(y[8], y[9], y[10], y[11]);
                            if (both) d[3] = make_uint4(y[12], y[13], y[14], y[15]);
                        } else {
                            uint4* d = reinterpret_cast<uint4*>((__nv_bfloat16*)p.y + to + c);
                            d[0] = make_uint4(bf16_bits(y[0], y[1]), bf16_bits(y[2], y[3]),
                                              bf16_bits(y[4], y[5]), bf16_bits(y[6], y[7]));
                            if (both)
                                d[1] = make_uint4(bf16_bits(y[8], y[9]), bf16_bits(y[10], y[11]),
                                                  bf16_bits(y[12], y[13]), bf16_bits(y[14], y[15]));
                        }
                    }
                    __syncwarp();
                }
                if (__builtin_expect(__any_sync(0xffffffffu, no_number && i < rows), 0))
                    outputs_again(p, at + C::kColY, at + C::kColX + n % kSets * TV, b, h, token, rows, i,
                                  no_number && i < rows, lg, f, staging ? stage : nullptr, to);
                tc_fence_before();
                mbar_arrive(of(y_free, n));
                if (staging) {
                    fence_proxy_async();
                    mbar_arrive(bar0 + 8u * (C::kOut + n % C::kV));
                }
            }
        }
    } else if (warp < 20) {
        // ------------------------------------------------------------ the state
        const int q = warp & 3, row = 32 * q + lane;  // the thread's row of it
        const bool keeps = 32 * q < p.Da;
        const uint32_t at = tmem + ((uint32_t)(32 * q) << 16) + C::kColS;
        uint32_t n = 0;
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (32 * q < TK && ok && next_walked<STATES>(p, feed, here)) {
            const Piece x = here;
            const int64_t own = ((int64_t)blockIdx.x * p.Da + row) * p.Dv;
            const int64_t kept = ((int64_t)x.sequence * p.Hq + x.h) * p.Da * p.Dv + row * p.row_stride;
            const float lg = head_decay(p, x.h, row == 0);
            const bool alone = forgets(lg);
            if (keeps) {  // the state in front of the piece
                const float* from = nullptr;
                int64_t step = 1;
                // (an empty sequence's places, in two blocks perhaps, all take `state` itself)
                if (!STATES && x.total > 0 && (x.begun || (p.state && x.c1 < x.total))) {
                    from = (x.begun ? p.slots : p.begins) + (int64_t)blockIdx.x * p.Da * p.Dv + row * p.slot_row;
                    step = p.slot_col;
                } else if (!STATES && p.state) {
                    from = p.state + kept;
                    step = p.col_stride;
                }
#pragma unroll 1
                for (int c = 0; c < width; c += 8) {
                    uint32_t r[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        r[j] = from && row < p.Da && c + j < p.Dv
                                   ? __float_as_uint(from[(c + j) * step]) : 0u;
                    tmem_st8(at + c, r);
                }
                tmem_wait_st();
            }
            if (STATES) {
                // (a block's one piece, without any decay between its chunks: the values' weights hold it)
                tc_fence_before();
                mbar_arrive(b_ready);
                ok = wait_for(done, 0, abort_flag, p.waits);
                tc_fence_after();
            }
            for (int k = x.c0; k < x.c1 && !STATES; ++k, ++n) {
                int rows;
                chunk_at(p, x, k, rows);
                if (keeps) {
                    const float g = exp2f(lg * rows);
                    const uint64_t g2 = pair(g, g);
#pragma unroll 1
                    for (int c = 0; c < p.Dv; c += 16) {
                        uint32_t r[16];
                        tmem_ld16(at + c, r);
                        tmem_wait_ld16(r);
                        // rows of 64 values, 16-byte pieces swapped as the tiles' are
                        uint8_t* d = smem + C::kOffSt + c / 64 * (TK * 128) + row * 128;
                        uint32_t hi[8], lo[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            hi[j] = split_pair(pair(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])),
                                               lo[j]);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint4* e = reinterpret_cast<uint4*>(d + 16 * ((c % 64 / 8 + j) ^ (row & 7)));
                            *e = make_uint4(hi[4 * j], hi[4 * j + 1], hi[4 * j + 2], hi[4 * j + 3]);
                            if (C::kStTwo)
                                e[C::kSt / 16] =
                                    make_uint4(lo[4 * j], lo[4 * j + 1], lo[4 * j + 2], lo[4 * j + 3]);
                        }
#pragma unroll
                        for (int j = 0; j < 16; j += 2) {
                            const float2 v =
                                halves(mul2(pair(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), g2));
                            r[j] = __float_as_uint(v.x);
                            r[j + 1] = __float_as_uint(v.y);
                        }
                        tmem_st16(at + c, r);
                    }
                    tmem_wait_st();
                    if (alone) clear_columns(at, p.Dv, false);
                }
                fence_proxy_async();
                tc_fence_before();
                mbar_arrive(b_ready);
                ok = wait_chunk(u_ready, n);
                if (!ok) break;
                tc_fence_after();
                if (row == 0) mbar_arrive(ring(C::kEmptyA, C::kA, n));  // the other of the two that read A
            }
            if (!ok) break;
            float* to = nullptr;
            int64_t step = 1;
            if (STATES) {
                to = p.slots_out + own;
            } else if (p.state_out && x.c1 == x.total) {
                to = p.state_out + kept;
                step = p.col_stride;
            }
            if (keeps && to)
#pragma unroll 1
                for (int c = 0; c < p.Dv; c += 8) {
                    uint32_t r[8];
                    tmem_ld8(at + c, r);
                    wait_ld8(r);
                    if (row < p.Da)
#pragma unroll
                        for (int j = 0; j < 8; ++j) to[(c + j) * step] = __uint_as_float(r[j]);
                    __syncwarp();
                }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------ decayed values
        const int maker = threadIdx.x - 640;
        // a row's 16-byte pieces of a tile of 64 channels that hold values: 8, or 4 where parts are whole chunks
        const int shift = C::kParts == 1 && width <= 32 ? 2 : 3;
        const int stride = 128 >> shift, turns = C::kPart / stride;  // of a part: the thread's tokens
        const int r0 = maker >> shift;
        uint32_t n = 0, g = 0;
        bool ok = true;
        begin_feed(p, blockIdx.x, gridDim.x, feed);
        while (ok && next_walked<STATES>(p, feed, here)) {
            const Piece x = here;
            const float lg = head_decay(p, x.h, false);
            // From the end of a part where its weights are largest on, each next one of the thread's tokens has
            // `ratio` times the last one's weight.
            const float ratio = exp2f(lg * stride);
            const bool alone = forgets(lg);
            for (int k = x.c0; k < x.c1; ++k, ++n) {
                int rows;
                chunk_at(p, x, k, rows);
                ok = wait_use(C::kFullA, C::kA, n) && wait_use(C::kFullV, C::kV, n) &&
                     (n < 2 || STATES || wait_chunk(y_free, n - 2));  // clean's and made's last phases are seen
                if (!ok) break;
                uint8_t* v = tile_v(n);
                if (rows < kChunk) {
                    // what lies behind the sequence may be another one, or no numbers at all
                    uint8_t* a = tile_a(n);
#pragma unroll 1
                    for (int e = 8 * rows + maker; e < 8 * kChunk; e += 128)
#pragma unroll
                        for (int t = 0; t < TV / 64; ++t)
                            *reinterpret_cast<uint4*>(v + 16 * e + t * kAtomBytes) = make_uint4(0, 0, 0, 0);
#pragma unroll 1
                    for (int e = 8 * rows + maker; e < 8 * kChunk; e += 128)
#pragma unroll
                        for (int t = 0; t < TK / 64; ++t)
                            *reinterpret_cast<uint4*>(a + 16 * e + t * kAtomBytes) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async();
                }
                // without outputs the state is not decayed from chunk to chunk: all of its decay is in the values
                const int behind = STATES ? (x.c1 - 1 - k) * kChunk : 0;
                // Without memory only a token whose weight is a power of 0 is left in the state, and of the others not
                // even what is not finite: their rows of A become 0, when the scores are made.
                const int last = !alone || p.back || behind ? -1 : rows - 1;
                if (alone) {
                    ok = STATES || wait_chunk(s_ready, n);
                    if (!ok) break;
                    clear_rows<TK>(tile_a(n), maker, last);
                    fence_proxy_async();
                }
                mbar_arrive(of(clean, n));
#pragma unroll 1
                for (int part = 0; part < C::kParts; ++part, ++g) {
                    ok = g < (uint32_t)C::kBufs || wait_use(C::kVFree, C::kBufs, g - C::kBufs);
                    if (!ok) break;
                    uint8_t* to = smem + C::kOffVw + g % C::kBufs * 2 * C::kVw;
                    // the thread's token with the part's largest weight, and where its piece lies: the tiles'
                    // pieces are swapped by the row's last three bits
                    const int row = p.back ? r0 : C::kPart - stride + r0;
                    int at = part * C::kPart + row;
                    int o = row * 128 + 16 * ((maker & ((1 << shift) - 1)) ^ (row & 7));
                    const uint8_t* from = v + part * C::kPart * 128;
                    const int step = p.back ? stride * 128 : -stride * 128;
                    if (rows == kChunk && !alone) {
                        float w = exp2f(lg * (behind + (p.back ? at + 1 - p.lead : kChunk - p.lead - at))) * p.scale_w;
#pragma unroll 1
                        for (int e = 0; e < turns; e += 4 / (TV / 64)) {
                            uint4 d[4];  // as many as fit, read before the first is worked on
#pragma unroll
                            for (int j = 0; j < 4; ++j)
                                d[j] = *reinterpret_cast<const uint4*>(
                                    from + o + j / (TV / 64) * step + j % (TV / 64) * kAtomBytes);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                uint8_t* dst = to + o + j / (TV / 64) * step + j % (TV / 64) * C::kPart * 128;
                                uint4 rest;
                                *reinterpret_cast<uint4*>(dst) = scaled(d[j], w, rest);
                                *reinterpret_cast<uint4*>(dst + C::kVw) = rest;
                                if (j % (TV / 64) == TV / 64 - 1) w *= ratio;
                            }
                            o += 4 / (TV / 64) * step;
                        }
                    } else {
#pragma unroll 1
                        for (int e = 0; e < turns; ++e, o += step, at += p.back ? stride : -stride) {
                            const float w =
                                exp2f(lg * (behind + (p.back ? at + 1 - p.lead : rows - p.lead - at))) * p.scale_w;
#pragma unroll
                            for (int t = 0; t < TV / 64; ++t) {
                                uint4 d = make_uint4(0, 0, 0, 0), rest = d;
                                if (alone ? at == last : at < rows)
                                    d = scaled(*reinterpret_cast<const uint4*>(from + o + t * kAtomBytes), w, rest);
                                *reinterpret_cast<uint4*>(to + o + t * C::kPart * 128) = d;
                                *reinterpret_cast<uint4*>(to + C::kVw + o + t * C::kPart * 128) = rest;
                            }
                        }
                    }
                    fence_proxy_async();
                    mbar_arrive(ring(C::kVFull, C::kBufs, g));
                }
                if (!ok) break;
                mbar_arrive(of(made, n));
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, C::kTmem);
}

// ------------------------------------------------------------------ packed sequences
// One block: the cuts, brought into 0 to N and never falling (each at least the largest before it), and the
// places before every sequence in the list of chunks, where each has some more in front (kDecayFront). And where
// every block's equal part of that list begins.
constexpr int kCutThreads = 1024;
__global__ void __launch_bounds__(kCutThreads)
    cut_kernel(const int32_t* offsets, int sequences, int N, int* first, int* cuts, int Hq, int blocks,
               int2* starts, int* status) {
    __shared__ int sm[2][kCutThreads / 32];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    bool bad = false;
    int base = 0, total = 0;  // the largest cut, the chunks so far
    for (int s0 = 0; s0 <= sequences; s0 += kCutThreads) {
        const int s = s0 + threadIdx.x;
        const int raw = s <= sequences ? offsets[s] : 0;
        int v = min(max(raw, 0), N);
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v = max(v, o);
        }
        if (lane == 31) sm[0][warp] = v;
        __syncthreads();
        for (int w = 0; w < kCutThreads / 32; ++w) {
            if (w == warp) v = max(v, base);
            base = max(base, sm[0][w]);
        }
        if (s <= sequences) {
            cuts[s] = v;
            bad = bad || v != raw;
        }
        __syncthreads();
    }
    if (bad) record_status(status, FLAREPP_ERR_INVALID_ARGUMENT);
    for (int s0 = 0; s0 < sequences; s0 += kCutThreads) {
        const int s = s0 + threadIdx.x;
        const int n = s < sequences ? kDecayFront + (cuts[s + 1] - cuts[s] + kChunk - 1) / kChunk : 0;
        int v = n;
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += o;
        }
        if (lane == 31) sm[1][warp] = v;
        __syncthreads();
        int at = v - n;
        for (int w = 0; w < kCutThreads / 32; ++w) {
            if (w == warp) at += total;
            total += sm[1][w];
        }
        if (s < sequences) first[s] = at;
        __syncthreads();
    }
    if (threadIdx.x == 0) first[sequences] = total;
    if (!starts) return;
    __syncthreads();
    const int all = total * Hq, share = (all + blocks - 1) / blocks;  // (the host has seen to 31 bits)
    for (int b = threadIdx.x; b < blocks && b * share < all; b += kCutThreads) {
        const int at = b * share;
        int low = 0, high = sequences;  // the last sequence that begins at this place or before
        while (high - low > 1) {
            const int mid = (low + high) / 2;
            if (first[mid] * Hq <= at) low = mid;
            else high = mid;
        }
        starts[b] = make_int2(low, (at - first[low] * Hq) / (first[low + 1] - first[low]));
    }
}

__global__ void __launch_bounds__(256)
    blank_kernel(const int* cuts, int sequences, int N, __nv_bfloat16* y, int64_t yh, int64_t yn, int H,
                 int D) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int a = cuts[0], b = cuts[sequences], v = D / 8;
    const int64_t n = (int64_t)(a + N - b) * H * v, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int64_t rh = i / v;
        const int row = (int)(rh / H), h = (int)(rh - (int64_t)row * H);
        const int64_t t = row < a ? row : b + (row - a);
        *reinterpret_cast<uint4*>(y + h * yh + t * yn + (i - rh * v) * 8) = make_uint4(0, 0, 0, 0);
    }
}

// ------------------------------------------------------------------ the join over a sequence's pieces
// In: the state that a block's last piece leaves from nothing, for blocks whose last piece's sequence goes on
// in the next block. Out: the state in front of every block's first chunk, and, in place of what the block left
// with which a sequence begins, the state in front of the sequence (if there is one: Walk::begins). A group of blocks
// (blockIdx.y) follows the sequence that begins in walk block y and goes on in the next, a thread one
// value of the state, kAhead blocks' values in flight.
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Walk p, float* left, float* slots,
                                                   int blocks) {
    tc::pdl_trigger();
    tc::pdl_wait();
    constexpr int kAhead = 8;
    const int e = blockIdx.x * 256 + threadIdx.x, size = p.Da * p.Dv, y = blockIdx.y;
    // what walk block y + 1 begins with, where its first place is in a sequence's head
    const Walk& q = p;
    Feed f;
    begin_feed(q, y + 1, blocks, f);
    if (f.at >= f.end) return;
    const int end = f.at, share = end / (y + 1);
    const int low = f.sequence, h = f.h, each = places_of(q, low), base = places_before(q, low) + h * each;
    if (base < y * share || base >= end || e >= size) return;  // begun before block y, or behind it
    bool bad = false;
    const float lg = decay_log2(q.log_decay[h], &bad);
    int start;
    const int tokens = tokens_of(q, low, start);
    // tokens of chunks c0 to c1, as walked, and the chunks up to a place
    const int total = (tokens + kChunk - 1) / kChunk, ragged = total * kChunk - tokens;
    auto rows_of = [&](int c0, int c1) {
        const bool holds = c0 < c1 && (q.back ? c0 == 0 : c1 == total);  // the chunk that ends early
        return (c1 - c0) * kChunk - (holds ? ragged : 0);
    };
    auto chunks_to = [&](int place) { return max(place - base - q.front, 0); };
    const int r = e / q.Dv, c = e - r * q.Dv;
    float run = q.state ? q.state[((int64_t)low * q.Hq + h) * size + r * q.row_stride + c * q.col_stride] : 0.f;
    const int last = (base + each - 1) / share;  // the walk block that ends the sequence
    const float begin = run;
    for (int k0 = y; k0 < last; k0 += kAhead) {
        float v[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (k0 + j < last) v[j] = left[(int64_t)(k0 + j) * size + e];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int k = k0 + j;
            if (k >= last) break;
            const int rows = rows_of(chunks_to(k * share), chunks_to((k + 1) * share));
            run = rows > 0 && forgets(lg) ? v[j] : fmaf(exp2f(lg * rows), run, v[j]);
            slots[(int64_t)(k + 1) * size + e] = run;
        }
        if (k0 == y && q.state) left[(int64_t)y * size + e] = begin;
    }
}

// ------------------------------------------------------------------ the sum over a group's heads
__global__ void __launch_bounds__(256)
    group_kernel(const float* sums, int64_t BN, int64_t N, int Hk, int group, int D, __nv_bfloat16* y,
                 int64_t yb, int64_t yh, int64_t yn) {
    tc::pdl_trigger();
    tc::pdl_wait();
    const int v = D / 8;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= BN * Hk * v) return;
    const int64_t rest = id / v;
    const int c = (int)(id - rest * v) * 8;
    const int64_t bh = rest / N, n = rest - bh * N, b = bh / Hk;
    const int h = (int)(bh - b * Hk);
    float a[8];
    for (int g = 0; g < group; ++g) {
        const float* x = sums + ((bh * group + g) * N + n) * D + c;
        const float4 lo = *reinterpret_cast<const float4*>(x);
        const float4 hi = *reinterpret_cast<const float4*>(x + 4);
        const float t[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = g ? a[j] + t[j] : t[j];
    }
    *reinterpret_cast<uint4*>(y + b * yb + h * yh + n * yn + c) =
        make_uint4(bf16_pair(a[0], a[1]), bf16_pair(a[2], a[3]), bf16_pair(a[4], a[5]),
                   bf16_pair(a[6], a[7]));
}

// ------------------------------------------------------------------ host side
size_t up(size_t n) { return (n + kWsAlign - 1) / kWsAlign * kWsAlign; }

template <typename... Args>
cudaError_t launch(void (*kernel)(Args...), int64_t blocks, int threads, size_t smem, cudaStream_t st,
                   const std::common_type_t<Args>&... args) {
    if (blocks <= 0 || blocks > INT32_MAX) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Args(args)...);
}

// bf16 [B, H, N, D]: boxes of 64 channels by 128 tokens, swizzled. A dimension whose values are the same
// place (stride 0) is one of size 1: *own_head and *own_batch say whether coordinates count.
bool map_of(CUtensorMap* m, const flarepp_heads& t, int64_t B, int64_t H, int64_t N, int64_t D,
            bool* own_head, bool* own_batch) {
    auto fn = encode_fn();
    if (!fn) return false;
    *own_head = H > 1 && t.stride_h > 0;
    *own_batch = B > 1 && t.stride_b > 0;
    const cuuint64_t row = (cuuint64_t)D * 2;
    cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)N, *own_head ? (cuuint64_t)H : 1,
                          *own_batch ? (cuuint64_t)B : 1};
    cuuint64_t strides[3] = {N > 1 ? (cuuint64_t)t.stride_n * 2 : row,
                             *own_head ? (cuuint64_t)t.stride_h * 2 : row,
                             *own_batch ? (cuuint64_t)t.stride_b * 2 : row};
    cuuint32_t box[4] = {64, kChunk, 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t.data, dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int TK, int TV, bool STATES>
cudaError_t launch_walk(const CUtensorMap* m, const Walk& p, int64_t blocks, cudaStream_t st) {
    using C = Cfg<TK, TV, STATES>;
    auto kernel = walk_kernel<TK, TV, STATES>;
    static std::atomic<uint64_t> ready{0};  // devices whose shared-memory limit is raised
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!(ready.load() >> dev & 1)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
        if (e != cudaSuccess) return e;
        ready.fetch_or(uint64_t(1) << dev);
    }
    return launch(kernel, blocks, kThreads, C::kSmem, st, m[0], m[1], m[2], m[3], p);
}

template <bool STATES>
cudaError_t launch_for(const CUtensorMap* m, const Walk& p, int64_t blocks, cudaStream_t st) {
    if (p.Da <= 64)
        return p.Dv <= 64 ? launch_walk<64, 64, STATES>(m, p, blocks, st)
                          : launch_walk<64, 128, STATES>(m, p, blocks, st);
    return p.Dv <= 64 ? launch_walk<128, 64, STATES>(m, p, blocks, st)
                      : launch_walk<128, 128, STATES>(m, p, blocks, st);
}

}  // namespace

cudaError_t take_decay_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

// Each of the card's blocks walks an equal part of the list of all sequences' heads' chunks, so that a sequence
// may be cut between two blocks or more, which costs a first walk over what lies in front of the cuts and two
// launches; or the list is one of whole sequences' heads, and nothing is cut. The cheaper one by the chunks that
// the busiest block has to do, those of the first walk as 0.8 (it reads half of the bytes, and may be
// as long again), the launches as ten. Whole and cut, us a forward in a graph: 128 heads of 8,192
// tokens and 128 channels 187 and 313; of 64 channels 160 of 4,096 116 and 126, 76 of 8,192 109 and 110, 128 of 1,024
// 22 and 52, 8 of 700 15 and 26, 8 of 1,200 22 and 28. (Lengths of packed sequences are not known here: the
// longest possible one counts.)
DecayPlan decay_plan(const flarepp_decay_shape& s, bool backward) {
    DecayPlan p{};
    p.sequences = s.sequences ? s.sequences : s.B;
    p.chunks = cdiv(s.N, kChunk);
    const int64_t heads = p.sequences * s.Hq;
    const int64_t places = s.sequences ? s.Hq * (p.chunks + kDecayFront * s.sequences) : heads * p.chunks;
    const int64_t whole = cdiv(heads, kNumSMs);  // heads of the busiest block
    const int64_t cut = cdiv(places, kNumSMs);   // chunks of every block
    p.whole = (double)(whole * p.chunks) <= (double)cut + 0.8 * (double)(cut < p.chunks ? cut : p.chunks) + 10;
    if (s.sequences) {
        p.blocks = p.whole && heads < kNumSMs ? heads : kNumSMs;
        p.share = p.whole ? cdiv(heads, p.blocks) : 0;
    } else {
        p.share = p.whole ? whole : cut;
        p.blocks = cdiv(p.whole ? heads : places, p.share);
    }
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    if (s.sequences) {
        p.off_first = place((p.sequences + 1) * 4);
        p.off_cuts = place((p.sequences + 1) * 4);
        if (!p.whole) p.off_starts = place(p.blocks * sizeof(int2));
    }
    if (!p.whole) {
        p.off_left = place((size_t)p.blocks * s.Dk * s.Dv * 4);
        p.off_slots = place((size_t)p.blocks * s.Dk * s.Dv * 4);
    }
    if (backward && s.Hq != s.Hk)
        p.off_sums = place((size_t)s.B * s.Hq * s.N * (s.Dk > s.Dv ? s.Dk : s.Dv) * 4);
    p.total = at;
    return p;
}

cudaError_t decay_cut(const flarepp_decay_shape& s, const DecayPlan& p, const int32_t* offsets, char* ws,
                      int32_t* status, cudaStream_t st) {
    return launch(cut_kernel, 1, kCutThreads, 0, st, offsets, (int)s.sequences, (int)s.N,
                  (int*)(ws + p.off_first), (int*)(ws + p.off_cuts), (int)s.Hq, (int)p.blocks,
                  p.whole ? (int2*)nullptr : (int2*)(ws + p.off_starts), (int*)status);
}

cudaError_t decay_blank(const flarepp_decay_shape& s, const DecayPlan& p, char* ws, const flarepp_heads& y,
                        int64_t heads, int64_t D, cudaStream_t st) {
    const int64_t most = cdiv(s.N * heads * D / 8, 256);
    return launch(blank_kernel, most < 2 * kNumSMs ? most : 2 * kNumSMs, 256, 0, st,
                  (const int*)(ws + p.off_cuts), (int)s.sequences, (int)s.N, (__nv_bfloat16*)y.data,
                  y.stride_h, y.stride_n, (int)heads, (int)D);
}

cudaError_t decay_walk(const DecayPlan& plan, char* ws, const DecayWalk& w, cudaStream_t st) {
    const flarepp_decay_shape& s = *w.shape;
    Walk p{};
    p.Hq = (int)s.Hq, p.N = (int)s.N, p.Da = (int)w.Da, p.Dv = (int)w.Dv;
    p.back = w.back;
    CUtensorMap m[4];
    const DecayOperand* of[3] = {&w.x, &w.a, &w.v};
    int* const group[3] = {&p.gx, &p.ga, &p.gv};
    int* const batch[3] = {&p.mx, &p.ma, &p.mv};
    for (int i = 0; i < 3; ++i) {
        bool own_head, own_batch;
        if (!map_of(&m[i], *of[i]->t, s.B, of[i]->heads, s.N, i == 2 ? w.Dv : w.Da, &own_head, &own_batch))
            return cudaErrorInvalidValue;
        *group[i] = own_head ? (int)(s.Hq / of[i]->heads) : 0;
        *batch[i] = own_batch;
    }
    m[3] = m[2];  // (float32 outputs are not staged)
    if (!w.y32) {
        bool own_head, own_batch;
        if (!map_of(&m[3], *w.y, s.B, s.Hq, s.N, w.Dv, &own_head, &own_batch)) return cudaErrorInvalidValue;
    }
    if (s.sequences) {
        p.cuts = (const int*)(ws + plan.off_cuts);
        p.first = (const int*)(ws + plan.off_first);
    }
    if (s.sequences && !plan.whole) {
        p.starts = (const int2*)(ws + plan.off_starts);
        p.front = kDecayFront;
    }
    p.whole = plan.whole;
    p.sequences = (int)plan.sequences;
    p.chunks = (int)plan.chunks;
    p.share = (int)plan.share;
    p.lead = w.back ? 0 : 1;
    p.scale_p = s.scale;
    p.gentle = fabsf(s.scale) >= 0x1p-40f || s.scale == 0.f ? -1.01f : 0.f;
    p.scale_w = w.back ? s.scale : 1.f;
    p.scale_r = w.back ? 1.f : s.scale;
    p.log_decay = w.log_decay;
    Source* const sources[3] = {&p.x, &p.a, &p.v};
    for (int i = 0; i < 3; ++i) {
        const flarepp_heads& t = *of[i]->t;
        *sources[i] = {(const __nv_bfloat16*)t.data, t.stride_b, t.stride_h, t.stride_n};
    }
    if (w.y32) {
        p.y = w.y32, p.y_f32 = 1;
        p.yn = w.Dv, p.yh = s.N * w.Dv, p.yb = s.Hq * p.yh;
    } else {
        p.y = w.y->data;
        p.yb = w.y->stride_b, p.yh = w.y->stride_h, p.yn = w.y->stride_n;
    }
    p.row_stride = w.turned ? 1 : w.Dv;
    p.col_stride = w.turned ? w.Da : 1;
    p.slot_row = w.again ? 1 : p.Dv;
    p.slot_col = w.again ? p.Da : 1;
    p.waits.status = w.status;
    test_fault_for(kDecayKernel, &p.waits.limit_ns, &p.waits.withheld);
    p.state = w.state;
    cudaError_t e = cudaSuccess;
    if (!plan.whole) {
        float* left = (float*)(ws + plan.off_left);
        float* slots = (float*)(ws + plan.off_slots);
        p.slots = slots;
        p.begins = left;
        if (w.again) {
            p.state_out = w.state_out;
            return launch_for<false>(m, p, plan.blocks, st);
        }
        Walk first = p;
        first.slots_out = left;
        e = launch_for<true>(m, first, plan.blocks, st);
        if (e != cudaSuccess) return e;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)cdiv((int64_t)p.Da * p.Dv, 256), (unsigned)plan.blocks);
        cfg.blockDim = dim3(256);
        cfg.stream = st;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        e = cudaLaunchKernelEx(&cfg, join_kernel, p, left, slots, (int)plan.blocks);
        if (e != cudaSuccess) return e;
    }
    p.state_out = w.state_out;
    return launch_for<false>(m, p, plan.blocks, st);
}

cudaError_t decay_group_sum(const flarepp_decay_shape& s, const float* sums, const flarepp_heads& y, int64_t D,
                            cudaStream_t st) {
    return launch(group_kernel, cdiv(s.B * s.N * s.Hk * (D / 8), 256), 256, 0, st, sums, s.B * s.N, s.N,
                  (int)s.Hk, (int)(s.Hq / s.Hk), (int)D, (__nv_bfloat16*)y.data, y.stride_b, y.stride_h,
                  y.stride_n);
}

}  // namespace flarepp
