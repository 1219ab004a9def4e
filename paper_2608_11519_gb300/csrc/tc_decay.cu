// The walk of the decay attention over a sequence (tcgen05 / TMEM / TMA): y_t = x_t S_t with
// S_t = g S_(t-1) + a_t v_t^T, in chunks of 128 tokens. Within a chunk, from the state S in front of it,
//   Y = (X A^T o W) V + r o (X S),   S' = g^n S + A^T (w o V)
// with W_ij = g^(i-j) for j <= i (0 above), r_i = g^(i+1), w_j = g^(n-1-j): four products of 128 rows. The
// same walk from the sequence's end makes the gradients of keys and values (DecayWalk says how).
//
// Bound by bytes at every width: a chunk reads three tiles and writes one, 64 KB at 64 channels, which the
// card takes 1.45 us for on each of its 152 SMs, and its four products some 0.35 us. So one block walks a
// piece of a sequence of one head, with the state staying in TMEM, and nothing is read twice; where heads
// and sequences are fewer than the SMs, sequences are cut into pieces, whose states a first walk
// (only A and V, only S) and a join over the pieces find.
//
// No power of g passes float32, whatever the decay: in blocks of 32 x 32 W is the product
// g^(i - last j of the block) g^(last j - j), a factor of the thread's and one of a table's, both at most 1
// below the diagonal; on it the first is g^-31 at most, and a strong decay takes an exponential each there.
// W o (X A^T), S and w o V are rounded to bf16 as operands; sums, states and what r multiplies are float32.
//
// Roles (24 warps, a block an SM): warp 0 loads tiles (A, X, V of each chunk, a ring), warps 1 and 2 issue the
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
constexpr int kTable = 160;                // powers of g: gaps of -32 to 127
constexpr int kPowers = 2 * kTable * 4;    // bytes of two such tables
constexpr size_t kWsAlign = 256;

// A piece of a sequence, as a block walks it.
struct Piece {
    int start, rows;  // tokens
    int sequence;
    int flags;  // kFirst: nothing before it in the sequence, kLast: nothing behind
};
enum { kFirst = 1, kLast = 2 };

struct Walk {
    int Hq, N, Da, Dv;
    int back, only_state;
    int gx, ga, gv;       // query heads that share a head of x, a, v
    int mx, ma, mv;       // whether a batch element has its own
    const Piece* pieces;  // packed sequences, else NULL
    const int* count;
    int n_pieces;
    int per_sequence, piece_rows;
    float scale_p, scale_w, scale_r;  // what scores, decayed values and X S are multiplied by
    int lead;                         // r_i = g^(i + lead), w_j = g^(n - lead - j)
    const float* log_decay;
    void* y;
    int64_t yb, yh, yn;
    int y_f32;
    const float* slots;   // the state in front of every piece [piece][Hq][Da][Dv], or NULL
    float* slots_out;     // with only_state: the state that a piece leaves
    const float* state;   // in front of every sequence, or NULL
    float* state_out;
    int64_t row_stride, col_stride;  // of a state between calls
    Waits waits;
};

template <int TK, int TV>
struct Cfg {
    static constexpr int kSlot = (TK > TV ? TK : TV) * kChunk * 2;
    // Values of up to 64 channels leave room for two sets of scores, of X S and of decayed values.
    static constexpr int kSets = TV == 64 ? 2 : 1;
    static constexpr int kVw = TV * kChunk * 2;
    static constexpr int kSt = TK * TV * 2;
    static constexpr uint32_t kColY = kSets * 128;  // from 0 on: scores, and W o scores as bf16 over them
    static constexpr uint32_t kColX = kColY + TV;
    static constexpr uint32_t kColS = kColX + kSets * TV;
    static constexpr uint32_t kTmem = 512;
    static constexpr int kRoom = kMaxSmem - 1024 - kPowers - kSets * kVw - kSt - 512;
    static constexpr int kSlots = kRoom / kSlot < 12 ? kRoom / kSlot : 12;
    static constexpr int kBars = 2 * kSlots + 15;
    static constexpr int kBody = kSlots * kSlot + kSets * kVw + kSt;
    static constexpr int kSmem = 1024 + kBody + kPowers + kBars * 8 + 16;
    static_assert(kSlots >= 5 && kBars * 8 + 16 <= 512 && kSmem <= kMaxSmem, "shared memory");
    static_assert(kColS + TV <= kTmem, "TMEM");
};

__device__ __forceinline__ Piece piece_of(const Walk& p, int i) {
    if (p.pieces) return p.pieces[i];
    Piece x;
    x.sequence = i / p.per_sequence;
    const int k = i - x.sequence * p.per_sequence;
    x.start = k * p.piece_rows;
    x.rows = min(p.piece_rows, p.N - x.start);
    x.flags = (k == 0 ? kFirst : 0) | (k == p.per_sequence - 1 ? kLast : 0);
    return x;
}
__device__ __forceinline__ bool ends(const Walk& p, const Piece& x) {
    return x.flags & (p.back ? kFirst : kLast);
}
__device__ __forceinline__ int chunks_of(const Walk& p, const Piece& x) {
    // the state of a sequence's last piece is not asked for by the first walk
    if (p.only_state && ends(p, x)) return 0;
    return (x.rows + kChunk - 1) / kChunk;
}
// The first token of the piece's k-th chunk, and its tokens.
__device__ __forceinline__ int chunk_at(const Walk& p, const Piece& x, int k, int n, int& rows) {
    const int c = p.back ? n - 1 - k : k;
    rows = min(kChunk, x.rows - c * kChunk);
    return x.start + c * kChunk;
}
__device__ __forceinline__ float head_decay(const Walk& p, int h, bool record) {
    bool bad = false;
    const float lg = decay_log2(p.log_decay[h], &bad);
    if (bad && record) record_status(p.waits.status, FLAREPP_ERR_INVALID_ARGUMENT);
    return lg;
}

// warp_wait whose tries sleep in the barrier (up to a millisecond each) instead of polling: most of a block's
// warps wait most of the time, and polling they took three of four issue slots from those that work.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                         const Waits& w) {
    bool got = mbar_sleep_wait(bar, parity, 1000000u);
    if (!got) {
        const uint64_t t0 = globaltimer_ns();
        const uint32_t nap = w.limit_ns < 4000000u ? (uint32_t)(w.limit_ns / 4) : 1000000u;
        while (!(got = mbar_sleep_wait(bar, parity, nap))) {
            if (*abort_flag) break;
            if (globaltimer_ns() - t0 > w.limit_ns) {
                *abort_flag = 1;
                record_status(w.status, FLAREPP_ERR_TIMEOUT);
                break;
            }
        }
    }
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

__device__ __forceinline__ uint4 scaled(uint4 d, float w) {
    const uint64_t w2 = pair(w, w);
    return make_uint4(pack_bf16x2(mul2(unpack_bf16x2(d.x), w2)), pack_bf16x2(mul2(unpack_bf16x2(d.y), w2)),
                      pack_bf16x2(mul2(unpack_bf16x2(d.z), w2)), pack_bf16x2(mul2(unpack_bf16x2(d.w), w2)));
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

// The chunks of a block's pieces, one after the other, for the roles that only count them.
struct Cursor {
    int u, left;
};
__device__ __forceinline__ bool next_chunk(const Walk& p, int units, Cursor& c) {
    while (c.left == 0) {
        if (c.u >= units) return false;
        c.left = chunks_of(p, piece_of(p, c.u / p.Hq));
        c.u += gridDim.x;
    }
    --c.left;
    return true;
}

__device__ __forceinline__ uint32_t bf16_bits(uint32_t a, uint32_t b) {
    return bf16_pair(__uint_as_float(a), __uint_as_float(b));
}

template <int TK, int TV>
__global__ void __launch_bounds__(kThreads, 1)
    walk_kernel(const __grid_constant__ CUtensorMap tX, const __grid_constant__ CUtensorMap tA,
                const __grid_constant__ CUtensorMap tV, const Walk p) {
    using C = Cfg<TK, TV>;
    constexpr int kSlots = C::kSlots;
    constexpr uint32_t kSets = C::kSets;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    uint8_t* vw = smem + kSlots * C::kSlot;
    uint8_t* st = vw + kSets * C::kVw;
    float* powers = reinterpret_cast<float*>(smem + C::kBody);  // [2][kTable]
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + C::kBody + kPowers);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    const uint32_t full0 = smem_u32(bars), empty0 = full0 + 8u * kSlots;
    // Of each but the last two there are two, for even and odd chunks: whoever waits for chunk n's phase must
    // not find that of chunk n + 1 done too, and no barrier's phase n + 2 comes before all have seen n.
    const uint32_t s_ready = empty0 + 8u * kSlots, p_ready = s_ready + 16, v_ready = s_ready + 32,
                   u_ready = s_ready + 48, y_ready = s_ready + 64, y_free = s_ready + 80;
    const uint32_t b_ready = s_ready + 96, done = s_ready + 104, t_ready = s_ready + 112;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(full0 + 8u * s, 1);
            mbar_init(empty0 + 8u * s, 2);
        }
        for (uint32_t s = 0; s < 16; s += 8) {
            mbar_init(s_ready + s, 1);
            mbar_init(p_ready + s, 256);
            mbar_init(v_ready + s, 128);
            mbar_init(u_ready + s, 1);
            mbar_init(y_ready + s, 1);
            mbar_init(y_free + s, 128);
        }
        mbar_init(b_ready, TK);
        mbar_init(done, 2);
        mbar_init(t_ready, 256);
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

    const int units = (p.pieces ? *p.count : p.n_pieces) * p.Hq;
    const int per = p.only_state ? 2 : 3;  // tiles of a chunk
    const int width = (p.Dv + 15) / 16 * 16;  // columns of the products
    const int steps = (p.Da + 15) / 16;       // steps of a product over Da
    // the barrier of chunk n, and its phase there
    auto of = [](uint32_t bar, uint32_t n) { return bar + 8u * (n & 1); };
    auto wait_chunk = [&](uint32_t bar, uint32_t n) {
        return wait_for(bar + 8u * (n & 1), (n >> 1) & 1, abort_flag, p.waits);
    };
    auto wait_tile = [&](uint32_t t) {
        return wait_for(full0 + 8u * (t % kSlots), (t / kSlots) & 1, abort_flag, p.waits);
    };
    auto tile = [&](uint32_t t) { return smem_u32(smem + t % kSlots * C::kSlot); };

    if (warp == 0) {
        // ------------------------------------------------------------ loads: A, X, V
        uint32_t it = 0;
        bool ok = true;
        for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
            const int i = u / p.Hq;
            const int h = u - i * p.Hq;
            const Piece x = piece_of(p, i);
            const int n = chunks_of(p, x), b = p.pieces ? 0 : x.sequence;
            for (int k = 0; k < n && ok; ++k) {
                int rows;
                const int token = chunk_at(p, x, k, n, rows);
                for (int j = 0; j < per; ++j, ++it) {
                    const int s = it % kSlots;
                    const uint32_t full = full0 + 8u * s;
                    if (it >= (uint32_t)kSlots &&
                        !wait_for(empty0 + 8u * s, (it / kSlots - 1) & 1, abort_flag, p.waits)) {
                        ok = false;
                        break;
                    }
                    if (elect_one() && !(blockIdx.x == 0 && it == p.waits.withheld)) {
                        const uint32_t dst = smem_u32(smem + s * C::kSlot);
                        const int what = p.only_state && j == 1 ? 2 : j;
                        mbar_expect_tx(full, (what == 2 ? TV : TK) * kChunk * 2);
                        if (what == 0)
                            load_rows<TK>(dst, &tA, token, p.ga ? h / p.ga : 0, b * p.ma, full);
                        else if (what == 1)
                            load_rows<TK>(dst, &tX, token, p.gx ? h / p.gx : 0, b * p.mx, full);
                        else
                            load_rows<TV>(dst, &tV, token, p.gv ? h / p.gv : 0, b * p.mv, full);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok) {  // wait (bounded) until every copy issued has landed
            const uint64_t t0 = globaltimer_ns();
            for (int s = 0; s < kSlots && (uint32_t)s < it; ++s) {
                const uint32_t last = it - 1 - ((it - 1 - s) % kSlots);
                while (!mbar_try_wait(full0 + 8u * s, (last / kSlots) & 1) &&
                       globaltimer_ns() - t0 < kWaitLimitNs) {
                }
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------ products: X A^T, and (W o X A^T) V
        // A tile is released by the warps that wait for its last product: a commit of its own
        // for each kept this warp from issuing for hundreds of cycles.
        const uint32_t scores = idesc_bf16_f32(128, 128, false, false);
        const uint32_t outs = idesc_bf16_f32(128, 16, false, true) + ((uint32_t)(width / 8 - 2) << 17);
        Cursor ahead{(int)blockIdx.x, 0}, here{(int)blockIdx.x, 0};
        bool ok = true;
        auto issue_scores = [&](uint32_t n) {
            if (!wait_tile(3 * n) || !wait_tile(3 * n + 1)) return false;
            tc_fence_after();
            const uint32_t a = lower(tile(3 * n), 16), x = lower(tile(3 * n + 1), 16);
            const uint32_t to = tmem + n % kSets * 128;
            if (elect_one()) {
#pragma unroll 1
                for (int s = 0; s < steps; ++s)
                    product_ss(to, x + by_channel(s), a + by_channel(s), scores, s > 0);
                mma_commit(of(s_ready, n));
            }
            __syncwarp();
            return true;
        };
        if (!p.only_state) {
            if (kSets == 2 && next_chunk(p, units, ahead)) ok = issue_scores(0);
            for (uint32_t n = 0; ok && next_chunk(p, units, here); ++n) {
                if (kSets == 1) ok = issue_scores(n);
                else if (next_chunk(p, units, ahead)) ok = issue_scores(n + 1);
                ok = ok && wait_chunk(v_ready, n) && wait_chunk(p_ready, n) &&
                     (n == 0 || wait_chunk(y_free, n - 1));
                if (!ok) break;
                tc_fence_after();
                const uint32_t v = lower(tile(3 * n + 2), kAtomBytes), w = tmem + n % kSets * 128;
                if (elect_one()) {
#pragma unroll 2
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
        const uint32_t s0 = lower(smem_u32(st), TK * 128);
        Cursor here{(int)blockIdx.x, 0};
        bool ok = true;
        for (uint32_t n = 0; next_chunk(p, units, here); ++n) {
            ok = wait_tile(per * n) && (p.only_state || wait_tile(3 * n + 1)) &&
                 (p.only_state || n < kSets || wait_chunk(y_free, n - kSets)) && wait_chunk(v_ready, n) &&
                 wait_for(b_ready, n & 1, abort_flag, p.waits);
            if (!ok) break;
            tc_fence_after();
            const uint32_t a = lower(tile(per * n), kAtomBytes), x = lower(tile(3 * n + 1), 16);
            const uint32_t v = lower(smem_u32(vw + n % kSets * C::kVw), kAtomBytes);
            const uint32_t to = tmem + C::kColX + n % kSets * TV;
            // (where TK is 64, A^T's rows from 64 on are whatever lies behind the tile: they are not used)
            if (elect_one()) {
                if (!p.only_state)
#pragma unroll 1
                    for (int s = 0; s < steps; ++s)
                        product_ss(to, x + by_channel(s), s0 + by_row(s), outs, s > 0);
#pragma unroll 2
                for (int s = 0; s < kChunk / 16; ++s)
                    product_ss(tmem + C::kColS, a + by_row(s), v + by_row(s), states, 1u);
                mma_commit(of(u_ready, n));
            }
            __syncwarp();
        }
        if (elect_one()) mma_commit(done);
        __syncwarp();
        wait_for(done, 0, abort_flag, p.waits);
        if (!ok) linger();
    } else if (warp == 3) {
        // (no role: the next four warps begin a warpgroup, whose warps are TMEM's four quarters)
    } else if (warp < 12) {
        // ------------------------------------------------------------ scores
        // Two warps share 32 tokens: one takes the keys 0 to 63, the other 64 to 127, 16 at a time, each
        // writing over columns that it has read itself.
        const int q = warp & 3, half = (warp - 4) >> 2, i = 32 * q + lane;  // the thread's token in the chunk
        const uint32_t at = tmem + ((uint32_t)(32 * q) << 16) + 64 * half;
        uint32_t n = 0, pieces = 0;
        bool ok = true;
        for (int u = blockIdx.x; !p.only_state && u < units && ok; u += gridDim.x) {
            const int item = u / p.Hq;
            const Piece x = piece_of(p, item);
            const int total = chunks_of(p, x);
            if (total == 0) continue;
            // The head's powers of g by gap, 0 for gaps below 0, in the order in which keys take them. A warp
            // that fills a table knows that all have left it: they have filled the other one since.
            float* table = powers + (pieces & 1) * kTable;
            {
                const float lg = head_decay(p, u - item * p.Hq, false);
                const int k = threadIdx.x - 128, gap = p.back ? k - 32 : 127 - k;
                if (k < kTable) table[k] = gap < 0 ? 0.f : exp2f(lg * gap) * p.scale_p;
            }
            mbar_arrive(t_ready);
            ok = wait_for(t_ready, pieces & 1, abort_flag, p.waits);
            ++pieces;
            if (!ok) break;
            const float* mine = table + (p.back ? 32 - i : 127 - i) + 64 * half;
            for (int k = 0; k < total; ++k, ++n) {
                int rows;
                chunk_at(p, x, k, total, rows);
                const uint32_t from = at + n % kSets * 128;
                ok = wait_chunk(s_ready, n);
                if (!ok) break;
                tc_fence_after();
                if (threadIdx.x == 128) {  // one of two that read A and X
                    mbar_arrive(empty0 + 8u * (3 * n % kSlots));
                    mbar_arrive(empty0 + 8u * ((3 * n + 1) % kSlots));
                }
#pragma unroll 1
                for (int c = 0; c < 64; c += 16) {
                    const int key = 64 * half + c;
                    uint32_t w[8];
                    if (p.back ? key + 15 < 32 * q : key > 32 * q + 31) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) w[j] = 0;
                    } else {
                        uint32_t r[16];
                        tmem_ld16(from + c, r);
                        tmem_wait_ld16(r);
                        const float* g = mine + c;
#pragma unroll
                        for (int j = 0; j < 16; j += 2)
                            w[j / 2] = pack_bf16x2(mul2(
                                pair(__uint_as_float(r[j]), __uint_as_float(r[j + 1])), pair(g[j], g[j + 1])));
                        // on the diagonal, and in a chunk that ends early, what does not count is 0
                        // whatever it was
                        if ((key >> 5) == q || key + 16 > rows) {
                            const int low = p.back ? i - key : 0;
                            const int high = min(p.back ? 16 : i + 1 - key, rows - key);
                            keep_keys(w, (high >= 16 ? 0xffffu : high <= 0 ? 0u : (1u << high) - 1u) &
                                             (low <= 0 ? ~0u : low >= 16 ? 0u : ~0u << low));
                        }
                    }
                    tmem_st8(from + c / 2, w);
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
        for (int u = blockIdx.x; !p.only_state && u < units && ok; u += gridDim.x) {
            const int item = u / p.Hq;
            const int h = u - item * p.Hq;
            const Piece x = piece_of(p, item);
            const int total = chunks_of(p, x), b = p.pieces ? 0 : x.sequence;
            if (total == 0) continue;
            const float lg = head_decay(p, h, false);
            for (int k = 0; k < total; ++k, ++n) {
                int rows;
                const int token = chunk_at(p, x, k, total, rows);
                const int since = p.back ? rows - 1 - i : i;
                const float f = i < rows ? exp2f(lg * (since + p.lead)) * p.scale_r : 0.f;
                const int64_t to = b * p.yb + h * p.yh + (int64_t)(token + i) * p.yn;
                ok = wait_chunk(u_ready, n) && wait_chunk(y_ready, n);
                if (!ok) break;
                tc_fence_after();
                if (threadIdx.x == 384)  // V has been read, by the warps that decay it and by its product
                    mbar_arrive_n(empty0 + 8u * ((3 * n + 2) % kSlots), 2);
#pragma unroll 1
                for (int c = 0; c < p.Dv; c += 16) {
                    uint32_t y[16], s[16];
                    tmem_ld16(at + C::kColY + c, y);
                    tmem_ld16(at + C::kColX + n % kSets * TV + c, s);
                    tmem_wait_ld16(y);
                    tmem_wait_ld16(s);
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        y[j] = __float_as_uint(fmaf(__uint_as_float(s[j]), f, __uint_as_float(y[j])));
                    if (i < rows) {
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
                tc_fence_before();
                mbar_arrive(of(y_free, n));
            }
        }
    } else if (warp < 20) {
        // ------------------------------------------------------------ the state
        const int q = warp & 3, row = 32 * q + lane;  // the thread's row of it
        const bool keeps = 32 * q < p.Da;
        const uint32_t at = tmem + ((uint32_t)(32 * q) << 16) + C::kColS;
        uint32_t n = 0;
        bool ok = true;
        for (int u = blockIdx.x; 32 * q < TK && u < units && ok; u += gridDim.x) {
            const int item = u / p.Hq;
            const int h = u - item * p.Hq;
            const Piece x = piece_of(p, item);
            const int total = chunks_of(p, x);
            const int64_t own = (int64_t)u * p.Da * p.Dv + (int64_t)row * p.Dv;
            const int64_t kept = ((int64_t)x.sequence * p.Hq + h) * p.Da * p.Dv + row * p.row_stride;
            const float lg = head_decay(p, h, row == 0);
            if (p.only_state && ends(p, x)) continue;
            if (keeps) {  // the state in front of the piece
                const float* from = nullptr;
                int64_t step = 1;
                if (!p.only_state && p.slots) {
                    from = p.slots + own;
                } else if (!p.only_state && p.state) {
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
            for (int k = 0; k < total; ++k, ++n) {
                int rows;
                chunk_at(p, x, k, total, rows);
                if (keeps) {
                    const float g = exp2f(lg * rows);
                    const uint64_t g2 = pair(g, g);
#pragma unroll 1
                    for (int c = 0; c < p.Dv; c += 16) {
                        uint32_t r[16];
                        tmem_ld16(at + c, r);
                        tmem_wait_ld16(r);
                        if (!p.only_state) {
                            // rows of 64 values, 16-byte pieces swapped as the tiles' are
                            uint8_t* d = st + c / 64 * (TK * 128) + row * 128;
#pragma unroll
                            for (int j = 0; j < 16; j += 8) {
                                const int piece = ((c % 64 + j) / 8) ^ (row & 7);
                                *reinterpret_cast<uint4*>(d + 16 * piece) = make_uint4(
                                    bf16_bits(r[j], r[j + 1]), bf16_bits(r[j + 2], r[j + 3]),
                                    bf16_bits(r[j + 4], r[j + 5]), bf16_bits(r[j + 6], r[j + 7]));
                            }
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
                }
                fence_proxy_async();
                tc_fence_before();
                mbar_arrive(b_ready);
                ok = wait_chunk(u_ready, n);
                if (!ok) break;
                tc_fence_after();
                if (row == 0) {  // the other of the two that read A and X; without outputs A and V
                    const uint32_t times = p.only_state ? 2 : 1;
                    mbar_arrive_n(empty0 + 8u * (per * n % kSlots), times);
                    mbar_arrive_n(empty0 + 8u * ((per * n + 1) % kSlots), times);
                }
            }
            if (!ok) break;
            float* to = nullptr;
            int64_t step = 1;
            if (p.only_state) {
                to = p.slots_out + own;
            } else if (p.state_out && ends(p, x)) {
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
        // a row's 16-byte pieces of a tile of 64 channels that hold values: 8 or 4
        const int shift = width > 32 ? 3 : 2, turns = 1 << shift;  // tokens of the thread
        uint32_t n = 0;
        bool ok = true;
        for (int u = blockIdx.x; u < units && ok; u += gridDim.x) {
            const int item = u / p.Hq;
            const Piece x = piece_of(p, item);
            const int total = chunks_of(p, x);
            if (total == 0) continue;
            const float lg = head_decay(p, u - item * p.Hq, false);
            // Of a whole chunk the thread takes a 16-byte piece of every 16th (or 32nd) token, from the one
            // with the largest weight on: each next one's is `ratio` times the last's.
            const int stride = 128 >> shift, r0 = p.back ? maker >> shift : 127 - (maker >> shift);
            const float heaviest = exp2f(lg * (p.back ? r0 + 1 - p.lead : kChunk - p.lead - r0)) * p.scale_w;
            const float ratio = exp2f(lg * stride);
            for (int k = 0; k < total; ++k, ++n) {
                int rows;
                chunk_at(p, x, k, total, rows);
                const uint32_t ia = per * n, iv = ia + per - 1;
                // the buffer's last product is done, and whoever waited for its last filling has seen it
                ok = wait_tile(iv) && (rows == kChunk || wait_tile(ia)) &&
                     (n < kSets || wait_chunk(u_ready, n - kSets)) &&
                     (n < 2 || p.only_state || wait_chunk(y_ready, n - 2));
                if (!ok) break;
                uint8_t* v = smem + iv % kSlots * C::kSlot;
                uint8_t* a = smem + ia % kSlots * C::kSlot;
                uint8_t* to = vw + n % kSets * C::kVw;
                if (rows == kChunk) {
                    float w = heaviest;
                    // the tiles' pieces are swapped by the row's last three bits
                    int o = r0 * 128 + 16 * ((maker & ((1 << shift) - 1)) ^ (r0 & 7));
                    const int step = p.back ? stride * 128 : -stride * 128;
#pragma unroll 2
                    for (int e = 0; e < turns; ++e, o += step, w *= ratio)
#pragma unroll
                        for (int t = 0; t < TV / 64; ++t)
                            *reinterpret_cast<uint4*>(to + o + t * kAtomBytes) =
                                scaled(*reinterpret_cast<const uint4*>(v + o + t * kAtomBytes), w);
                } else {
                    // what lies behind the sequence may be another one, or no numbers at all
#pragma unroll 1
                    for (int e = maker; e < TV * 16; e += 128) {
                        const int r = (e & 1023) >> 3;
                        const float w = exp2f(lg * (p.back ? r + 1 - p.lead : rows - p.lead - r)) * p.scale_w;
                        uint4 d = make_uint4(0, 0, 0, 0);
                        if (r < rows) d = scaled(*reinterpret_cast<const uint4*>(v + 16 * e), w);
                        else *reinterpret_cast<uint4*>(v + 16 * e) = d;
                        *reinterpret_cast<uint4*>(to + 16 * e) = d;
                    }
#pragma unroll 1
                    for (int e = maker; e < TK * 16; e += 128)
                        if (((e & 1023) >> 3) >= rows)
                            *reinterpret_cast<uint4*>(a + 16 * e) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async();
                mbar_arrive(of(v_ready, n));
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
// One block: the cuts, brought into 0 to N and never falling (each at least the largest before it), the
// first piece of every sequence, and the pieces.
constexpr int kCutThreads = 1024;
__global__ void __launch_bounds__(kCutThreads)
    cut_kernel(const int32_t* offsets, int sequences, int N, int piece_rows, Piece* pieces, int* first,
               int* cuts, int* status) {
    __shared__ int sm[kCutThreads / 32];
    tc::pdl_trigger();
    tc::pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    bool bad = false;
    int base = 0, total = 0;
    // the largest so far, 1,024 offsets at a time
    for (int s0 = 0; s0 <= sequences; s0 += kCutThreads) {
        const int s = s0 + threadIdx.x;
        const int raw = s <= sequences ? offsets[s] : 0;
        int v = min(max(raw, 0), N);
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v = max(v, o);
        }
        if (lane == 31) sm[warp] = v;
        __syncthreads();
        int before = base;
        for (int w = 0; w < warp; ++w) before = max(before, sm[w]);
        v = max(v, before);
        if (s <= sequences) {
            cuts[s] = v;
            bad = bad || v != raw;
        }
        for (int w = 0; w < kCutThreads / 32; ++w) base = max(base, sm[w]);
        __syncthreads();
    }
    if (bad) record_status(status, FLAREPP_ERR_INVALID_ARGUMENT);
    // the sums of the pieces so far
    for (int s0 = 0; s0 < sequences; s0 += kCutThreads) {
        const int s = s0 + threadIdx.x;
        int start = 0, rows = 0, n = 0;
        if (s < sequences) {
            start = cuts[s];
            rows = cuts[s + 1] - start;
            n = max(1, (rows + piece_rows - 1) / piece_rows);
        }
        int v = n;
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, v, d);
            if (lane >= d) v += o;
        }
        if (lane == 31) sm[warp] = v;
        __syncthreads();
        int at = total + v - n;
        for (int w = 0; w < warp; ++w) at += sm[w];
        for (int w = 0; w < kCutThreads / 32; ++w) total += sm[w];
        __syncthreads();
        if (s < sequences) {
            first[s] = at;
            for (int k = 0; k < n; ++k) {
                Piece x;
                x.start = start + k * piece_rows;
                x.rows = min(piece_rows, rows - k * piece_rows);
                x.sequence = s;
                x.flags = (k == 0 ? kFirst : 0) | (k == n - 1 ? kLast : 0);
                pieces[at + k] = x;
            }
        }
    }
    if (threadIdx.x == 0) first[sequences] = total;
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
// In: the state that every piece but a sequence's last leaves from nothing; out, in place: the state in
// front of every piece. A thread follows one value of a state, kAhead pieces' values in flight.
struct Join {
    int Hq, N, Da, Dv, back;
    const Piece* pieces;
    const int* first;
    int per_sequence, piece_rows;
    const float* log_decay;
    const float* state;
    int64_t row_stride, col_stride;
    float* slots;
};
__global__ void __launch_bounds__(256) join_kernel(const Join p, int blocks_per_state) {
    tc::pdl_trigger();
    tc::pdl_wait();
    constexpr int kAhead = 8;
    const int64_t sh = blockIdx.x / blocks_per_state;
    const int e = (int)(blockIdx.x - sh * blocks_per_state) * 256 + threadIdx.x, size = p.Da * p.Dv;
    if (e >= size) return;
    const int64_t s = sh / p.Hq;
    const int h = (int)(sh - s * p.Hq);
    bool bad = false;
    const float lg = decay_log2(p.log_decay[h], &bad);
    const int64_t i0 = p.pieces ? p.first[s] : s * p.per_sequence;
    const int n = p.pieces ? p.first[s + 1] - (int)i0 : p.per_sequence;
    const int r = e / p.Dv, c = e - r * p.Dv;
    float run = p.state ? p.state[sh * size + r * p.row_stride + c * p.col_stride] : 0.f;
    for (int k0 = 0; k0 < n; k0 += kAhead) {
        float v[kAhead], g[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int k = k0 + j;
            if (k >= n) break;
            const int pos = p.back ? n - 1 - k : k;
            v[j] = k < n - 1 ? p.slots[((i0 + pos) * p.Hq + h) * size + e] : 0.f;
            const int rows = p.pieces ? p.pieces[i0 + pos].rows
                                      : min(p.piece_rows, p.N - pos * p.piece_rows);
            g[j] = exp2f(lg * rows);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int k = k0 + j;
            if (k >= n) break;
            const int pos = p.back ? n - 1 - k : k;
            p.slots[((i0 + pos) * p.Hq + h) * size + e] = run;
            run = fmaf(g[j], run, v[j]);
        }
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

template <int TK, int TV>
cudaError_t launch_walk(const CUtensorMap* m, const Walk& p, int64_t units, cudaStream_t st) {
    using C = Cfg<TK, TV>;
    auto kernel = walk_kernel<TK, TV>;
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
    return launch(kernel, units < kNumSMs ? units : kNumSMs, kThreads, C::kSmem, st, m[0], m[1], m[2], p);
}

cudaError_t launch_for(const CUtensorMap* m, const Walk& p, int64_t units, cudaStream_t st) {
    if (p.Da <= 64)
        return p.Dv <= 64 ? launch_walk<64, 64>(m, p, units, st) : launch_walk<64, 128>(m, p, units, st);
    return p.Dv <= 64 ? launch_walk<128, 64>(m, p, units, st) : launch_walk<128, 128>(m, p, units, st);
}

}  // namespace

cudaError_t take_decay_status(int32_t* out, cudaStream_t st) { return take_library_status(out, st); }

// Where sequences and heads fill the card, a piece is a sequence; otherwise the cut is the one
// whose blocks have the least to do, a chunk of a cut sequence counting for the walk and for the
// states' (half as much). Lengths of packed sequences are not known here: pieces for twice the card.
DecayPlan decay_plan(const flarepp_decay_shape& s, bool backward) {
    DecayPlan p{};
    p.sequences = s.sequences ? s.sequences : s.B;
    const int64_t all = cdiv(s.N, kChunk), slots = kNumSMs;
    if (s.sequences) {
        const int64_t per = cdiv(all * s.Hq, 2 * slots);
        p.chunks = per < 4 ? 4 : per;
        if (p.chunks > all) p.chunks = all;
        p.per_sequence = 0;
        p.pieces = s.sequences + all / p.chunks;
        p.split = p.chunks < all;
    } else {
        const int64_t heads = p.sequences * s.Hq;
        int64_t best = 1;
        double least = 0.0;
        for (int64_t n = 1; n <= all && (n == 1 || n * heads <= 4 * slots); ++n) {
            const double cost =
                (double)cdiv(heads * n, slots) * (double)cdiv(all, n) * (n > 1 ? 1.5 : 1.0) + (n > 1 ? 4 : 0);
            if (n == 1 || cost < least) least = cost, best = n;
        }
        p.chunks = cdiv(all, best);
        p.per_sequence = cdiv(all, p.chunks);
        p.pieces = p.sequences * p.per_sequence;
        p.split = p.per_sequence > 1;
    }
    size_t at = 0;
    auto place = [&](size_t bytes) {
        const size_t here = at;
        at += up(bytes);
        return here;
    };
    if (s.sequences) {
        p.off_pieces = place(p.pieces * sizeof(Piece));
        p.off_first = place((p.sequences + 1) * 4);
        p.off_cuts = place((p.sequences + 1) * 4);
    }
    if (p.split) p.off_states = place((size_t)p.pieces * s.Hq * s.Dk * s.Dv * 4);
    if (backward && s.Hq != s.Hk)
        p.off_sums = place((size_t)s.B * s.Hq * s.N * (s.Dk > s.Dv ? s.Dk : s.Dv) * 4);
    p.total = at;
    return p;
}

cudaError_t decay_cut(const flarepp_decay_shape& s, const DecayPlan& p, const int32_t* offsets, char* ws,
                      int32_t* status, cudaStream_t st) {
    return launch(cut_kernel, 1, kCutThreads, 0, st, offsets, (int)s.sequences, (int)s.N,
                  (int)(p.chunks * kChunk), (Piece*)(ws + p.off_pieces), (int*)(ws + p.off_first),
                  (int*)(ws + p.off_cuts), (int*)status);
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
    CUtensorMap m[3];
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
    if (s.sequences) {
        p.pieces = (const Piece*)(ws + plan.off_pieces);
        p.count = (const int*)(ws + plan.off_first) + s.sequences;
    }
    p.n_pieces = (int)plan.pieces;
    p.per_sequence = (int)plan.per_sequence;
    p.piece_rows = (int)(plan.chunks * kChunk);
    p.lead = w.back ? 0 : 1;
    p.scale_p = s.scale;
    p.scale_w = w.back ? s.scale : 1.f;
    p.scale_r = w.back ? 1.f : s.scale;
    p.log_decay = w.log_decay;
    if (w.y32) {
        p.y = w.y32, p.y_f32 = 1;
        p.yn = w.Dv, p.yh = s.N * w.Dv, p.yb = s.Hq * p.yh;
    } else {
        p.y = w.y->data;
        p.yb = w.y->stride_b, p.yh = w.y->stride_h, p.yn = w.y->stride_n;
    }
    p.row_stride = w.turned ? 1 : w.Dv;
    p.col_stride = w.turned ? w.Da : 1;
    p.waits.status = w.status;
    test_fault_for(kDecayKernel, &p.waits.limit_ns, &p.waits.withheld);
    const int64_t units = plan.pieces * s.Hq;
    if (units > INT32_MAX - kNumSMs) return cudaErrorInvalidValue;
    cudaError_t e;
    if (plan.split) {
        float* slots = (float*)(ws + plan.off_states);
        Walk first = p;
        first.only_state = 1;
        first.slots_out = slots;
        e = launch_for(m, first, units, st);
        if (e != cudaSuccess) return e;
        Join j{};
        j.Hq = p.Hq, j.N = p.N, j.Da = p.Da, j.Dv = p.Dv, j.back = p.back;
        j.pieces = p.pieces;
        j.first = s.sequences ? (const int*)(ws + plan.off_first) : nullptr;
        j.per_sequence = p.per_sequence, j.piece_rows = p.piece_rows;
        j.log_decay = p.log_decay;
        j.state = w.state;
        j.row_stride = p.row_stride, j.col_stride = p.col_stride;
        j.slots = slots;
        const int blocks = (int)cdiv((int64_t)p.Da * p.Dv, 256);
        e = launch(join_kernel, plan.sequences * s.Hq * blocks, 256, 0, st, j, blocks);
        if (e != cudaSuccess) return e;
        p.slots = slots;
    }
    p.state = w.state;
    p.state_out = w.state_out;
    return launch_for(m, p, units, st);
}

cudaError_t decay_group_sum(const flarepp_decay_shape& s, const float* sums, const flarepp_heads& y, int64_t D,
                            cudaStream_t st) {
    return launch(group_kernel, cdiv(s.B * s.N * s.Hk * (D / 8), 256), 256, 0, st, sums, s.B * s.N, s.N,
                  (int)s.Hk, (int)(s.Hq / s.Hk), (int)D, (__nv_bfloat16*)y.data, y.stride_b, y.stride_h,
                  y.stride_n);
}

}  // namespace flarepp
