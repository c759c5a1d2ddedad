// Device-side status of the context-free kernels: one word per translation unit and device, which a kernel sets when one
// of its bounded waits has run out and abs_llm_check reads and clears.
#pragma once

#include <cuda_runtime.h>

#include "abs_sgd.h"

namespace abs_sgd {

static __device__ int g_llm_status;

__device__ __forceinline__ void report_timeout() { atomicExch(&g_llm_status, ABS_ETIMEOUT); }

// Blocks until `s` has finished; *status: the word, which is zero afterwards.
static inline cudaError_t take_status(int* status, cudaStream_t s) {
    const int zero = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(status, g_llm_status, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess && *status != 0) {
        e = cudaMemcpyToSymbolAsync(g_llm_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    }
    return e;
}

cudaError_t take_status_norm(int* status, cudaStream_t s);    // llm_norm.cu
cudaError_t take_status_loss(int* status, cudaStream_t s);    // llm_loss.cu

}  // namespace abs_sgd
