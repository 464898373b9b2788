// Beside fake_cudart.c: a driver entry point for tensor maps that encodes nothing.
#include <cuda.h>
#include <cuda_runtime_api.h>

static CUresult encode(void) { return CUDA_SUCCESS; }

cudaError_t cudaGetDriverEntryPointByVersion(const char *symbol, void **fn, unsigned int version, unsigned long long flags,
                                             enum cudaDriverEntryPointQueryResult *found) {
    (void)symbol, (void)version, (void)flags;
    *fn = (void *)encode;
    if (found) *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
