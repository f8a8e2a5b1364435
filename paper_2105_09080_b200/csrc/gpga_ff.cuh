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

// Tokens per node up to which the forward pass reads the weights where they lie, without the tensor memory path: up to
// there its time is that of reading them.
inline bool ff_few(const FeedForwardParams& p) { return p.rows <= (p.dtype == 0 ? 8 : 32); }
int64_t ff_few_scratch_bytes(const FeedForwardParams& p);
cudaError_t launch_ff_few(const FeedForwardParams& p, cudaStream_t stream);

int64_t ff_forward_scratch_bytes(const FeedForwardParams& p);
int64_t ff_backward_scratch_bytes(const FeedForwardParams& p);
cudaError_t launch_ff_forward(const FeedForwardParams& p, cudaStream_t stream);
cudaError_t launch_ff_backward(const FeedForwardParams& p, cudaStream_t stream);
unsigned int* ff_forward_gave_up();    // device addresses of the files' flags
unsigned int* ff_backward_gave_up();

}  // namespace gpga
