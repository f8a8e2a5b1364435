// Orthogonalisation of an update by Newton-Schulz products: what the host entry hands to the launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace gpga {

struct OrthParams {
    const void* m = nullptr;
    void* out = nullptr;
    int64_t ldm = 0, node_ldm = 0, ldo = 0, node_ldo = 0;
    int64_t nodes = 0, r = 0, c = 0, steps = 0;
    int dtype = 0;
    bool accumulate = false;
    double c1 = 0, c3 = 0, c5 = 0, scale = 1, eps = 0;
    char* scratch = nullptr;
};

int64_t orth_scratch_bytes(const OrthParams& p);
cudaError_t launch_orth(const OrthParams& p, cudaStream_t stream);
unsigned int* orth_gave_up();
cudaError_t launch_wait_selftest(cudaStream_t stream);

}  // namespace gpga
