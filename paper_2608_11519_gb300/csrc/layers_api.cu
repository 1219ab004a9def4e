// What the layers around the mixer share at the C interface: the question for the status of calls that
// passed no status word.
#include "layer_status.cuh"

extern "C" flarepp_status flarepp_layers_device_status(void* stream, int32_t* status_out) {
    using namespace flarepp;
    if (!status_out) return FLAREPP_ERR_INVALID_ARGUMENT;
    *status_out = FLAREPP_OK;
    cudaError_t (*const take[])(int32_t*, cudaStream_t) = {take_embedding_status, take_product_status,
                                                           take_few_status, take_fused_status};
    for (auto* from : take) {  // a wait that gave up counts for more than an id beyond the table
        int32_t word = FLAREPP_OK;
        if (from(&word, (cudaStream_t)stream) != cudaSuccess) return FLAREPP_ERR_CUDA;
        if (word != FLAREPP_OK) *status_out = word;
    }
    return FLAREPP_OK;
}
