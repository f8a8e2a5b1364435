// Gated feed-forward block: what its host entries hand to the launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace gpga {

struct Matrix {          // a row-major matrix per node
    void* p = nullptr;
    int64_t ld = 0, node = 0;
};

struct FeedForwardParams {
    Matrix x, y, g, u, dy, dx;           // activations: node stride = rows * ld
    Matrix gate, up, down, dgate, dup, ddown;
    int64_t nodes = 0, rows = 0, d = 0, f = 0;
    int dtype = 0, weight_dtype = 0, grad_dtype = 0, activation = 0;
    bool accumulate = false;
    char* scratch = nullptr;
};

int64_t ff_forward_scratch_bytes(const FeedForwardParams& p);
int64_t ff_backward_scratch_bytes(const FeedForwardParams& p);
cudaError_t launch_ff_forward(const FeedForwardParams& p, cudaStream_t stream);
cudaError_t launch_ff_backward(const FeedForwardParams& p, cudaStream_t stream);
unsigned int* ff_forward_gave_up();    // device addresses of the files' flags
unsigned int* ff_backward_gave_up();

}  // namespace gpga
