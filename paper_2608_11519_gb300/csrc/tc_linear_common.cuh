// What the tensor-core kernels of the linear layer share: the slices of a contraction and their tiles
// in shared memory, bounded waits, TMA maps. Each translation unit has its own copy.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>

#include <atomic>

#include "layer_status.cuh"
#include "linear_internal.h"
#include "tc_pair_ptx.cuh"

namespace flarepp {
namespace {

using namespace tc;

constexpr int kSlice = 64;  // contraction values per ring stage: one 128-byte row
constexpr int kATile = 128 * kSlice * 2;
constexpr int kMaxNT = 256;
constexpr uint32_t kTmemCols = 512;
constexpr uint64_t kWaitLimitNs = 2000000000ull;
constexpr int kBlockBytes = 32 * 32 * 2;  // what an epilogue warp stages at a time
constexpr int kMaxSmem = 232448;
// the launches' numbers for the test hook of the bounded waits (flarepp_test_wait_fault)
enum LinKernel { kProductKernel = 16, kFewKernel = 17, kFusedKernel = 18, kDecayKernel = 19 };

// The bound of every wait of a launch, where a wait that gave up is recorded (null: the library's word),
// and (for tests) the ring item that CTA 0's producer never loads, or -1.
struct Waits {
    uint64_t limit_ns;
    int* status;
    int64_t withheld;
};

template <int CG>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    return CG == 2 ? mbar_try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity);
}

// All lanes of a warp wait for a phase; false once this wait or another one of the CTA gave up.
template <int CG>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag,
                                          const Waits& w) {
    bool got = try_wait<CG>(bar, parity);
    if (!got) {
        const uint64_t t0 = globaltimer_ns();
        for (uint32_t i = 1;; ++i) {
            got = try_wait<CG>(bar, parity);
            if (got) break;
            if ((i & 63u) == 0) {
                if (*abort_flag) break;
                if (globaltimer_ns() - t0 > w.limit_ns) {
                    *abort_flag = 1;
                    record_status(w.status, FLAREPP_ERR_TIMEOUT);
                    break;
                }
            }
        }
    }
    return __all_sync(0xffffffffu, got);
}

// One operand's tile of `rows` rows for the slice at contraction index k: K-major as one box of
// 64 x rows, MN-major as boxes of 64 rows x 64 contraction values ("atoms").
template <int CG, bool MN>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* m, int row, int rows,
                                          int k, uint32_t bar) {
    if (!MN) {
        if (CG == 2) tma_load_2d_pair(dst, m, k, row, bar);
        else tma_load_2d(dst, m, k, row, bar);
    } else {
        for (int r = 0; r < rows; r += 64, dst += 64 * kSlice * 2) {
            if (CG == 2) tma_load_2d_pair(dst, m, row + r, k, bar);
            else tma_load_2d(dst, m, row + r, k, bar);
        }
    }
}

// The descriptor of the 16 contraction values at step s of a slice.
template <bool MN>
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, int s) {
    return MN ? smem_desc(addr + s * 16 * 128, 64 * kSlice * 2, 1024, kSw128)
              : smem_desc(addr + s * 32, 16, 1024, kSw128);
}

// Let a role's copies in flight land after a wait that gave up.
__device__ __forceinline__ void linger() {
    const uint64_t t0 = globaltimer_ns();
    while (globaltimer_ns() - t0 < 1000000ull) {
    }
}

// ------------------------------------------------------------------ host side

PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> fn{nullptr};
    PFN_cuTensorMapEncodeTiled_v12000 f = fn.load(std::memory_order_acquire);
    if (f) return f;
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
        fn.store(f = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p),
                 std::memory_order_release);
    return f;
}

// bf16 [lines][inner] with `pitch` elements from line to line, boxes of box_inner x box_lines,
// swizzled to their 128- or 64-byte lines
bool make_map(CUtensorMap* m, const void* base, int64_t inner, int64_t lines, int64_t pitch,
              int box_inner, int box_lines) {
    auto fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)lines};
    cuuint64_t strides[1] = {(cuuint64_t)pitch * 2};
    cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_lines};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box,
              estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              box_inner == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace flarepp
