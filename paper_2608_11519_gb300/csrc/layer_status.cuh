// Where the layers' kernels record what only they can see (a wait that gave up, an id beyond the
// table): the caller's status word, or, for calls that pass none, a word of the library's own on each
// device, which flarepp_layers_device_status asks for. Each translation unit has its own copy of the word:
// the kernels know its address, so that a call neither looks it up nor passes it.
#pragma once
#include <cuda_runtime.h>

#include "flarepp_internal.h"

namespace flarepp {
namespace {

__device__ int32_t library_status;

// The larger word stays: a call may record a wait that gave up, whose outputs are invalid, and in another block or a
// later launch an argument that it brought into its range, whose are not.
__device__ __forceinline__ void record_status(int32_t* status, flarepp_status what) {
    atomicMax(status ? status : &library_status, (int32_t)what);
}
static_assert(FLAREPP_ERR_TIMEOUT > FLAREPP_ERR_INVALID_ARGUMENT && FLAREPP_ERR_INVALID_ARGUMENT > FLAREPP_OK,
              "the worse word is the larger");

// The word of the current device once the work on `st` is done; FLAREPP_OK again afterwards.
cudaError_t take_library_status(int32_t* out, cudaStream_t st) {
    void* word = nullptr;
    cudaError_t e = cudaGetSymbolAddress(&word, library_status);
    if (e == cudaSuccess) e = cudaMemcpyAsync(out, word, 4, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess || *out == FLAREPP_OK) return e;
    e = cudaMemsetAsync(word, 0, 4, st);
    return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}
static_assert(FLAREPP_OK == 0, "a cleared word is FLAREPP_OK");

}  // namespace

// One for each translation unit whose kernels record.
cudaError_t take_product_status(int32_t* out, cudaStream_t st);    // tc_linear.cu
cudaError_t take_few_status(int32_t* out, cudaStream_t st);        // tc_linear_few.cu
cudaError_t take_fused_status(int32_t* out, cudaStream_t st);      // tc_linear_fused.cu
cudaError_t take_embedding_status(int32_t* out, cudaStream_t st);  // embedding.cu
cudaError_t take_decay_status(int32_t* out, cudaStream_t st);      // tc_decay.cu
cudaError_t take_decay_step_status(int32_t* out, cudaStream_t st); // decay_step.cu
cudaError_t take_norm_status(int32_t* out, cudaStream_t st);       // norm.cu

}  // namespace flarepp
