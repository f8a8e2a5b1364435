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

// Whether the forward pass reads the weights where they lie, without the tensor memory path: for few tokens its time is
// that of reading them.  Measured with either: 32 tokens, 2048 x 5632, 16-bit weights 30 us and 33 us, fp32 weights 39 us
// and 97 us; 24 tokens, 4096 x 11008, 16-bit weights 94 us and 81 us, 16 tokens 81 us and 81 us; 8 tokens in fp32, 1024 x 2816 36 us and
// 48 us, 2048 x 5632 98 us and 157 us.  The form ends at 32 tokens (8 in fp32), where fp32 weights would still gain by it; 16-bit
// ones do not from 17 tokens on where they are large: 20e6 lies between the two sizes above.
inline bool ff_few(const FeedForwardParams& p)
{
    if (p.dtype == 0) return p.rows <= 8;
    return p.rows <= 16 || (p.rows <= 32 && (p.weight_dtype == 0 || p.d * p.f <= 20'000'000));
}
// Whether fp32 operands are taken as pairs of fp16 values (three products of pieces, with passes for the powers of two of rows and
// columns) and not as three bfloat16 values (six products): where the products take long enough for the passes.  Measured with
// three values and with pairs: forward 442 x 221 x 602 on 3 nodes 41 us and 54 us, 4096 x 256 x 688 56 us and 57 us, 700 x 700 x
// 1500 60 us and 53 us, 1151 x 743 x 1901 118 us and 102 us; gradient 1024 x 512 x 1024 74 us and 79 us, 700 x 700 x 1500
// 100 us and 101 us, 1536 x 768 x 768 105 us and 101 us, 2048 x 768 x 2048 229 us and 197 us.
inline bool ff_pairs(const FeedForwardParams& p, bool backward)
{
    return p.dtype == 0 && (double)p.nodes * p.rows * p.d * p.f * (backward ? 12 : 6) >= (backward ? 10e9 : 4e9);
}
int64_t ff_few_scratch_bytes(const FeedForwardParams& p);
cudaError_t launch_ff_few(const FeedForwardParams& p, cudaStream_t stream);

int64_t ff_forward_scratch_bytes(const FeedForwardParams& p);
int64_t ff_backward_scratch_bytes(const FeedForwardParams& p);
cudaError_t launch_ff_forward(const FeedForwardParams& p, cudaStream_t stream);
cudaError_t launch_ff_backward(const FeedForwardParams& p, cudaStream_t stream);
unsigned int* ff_forward_gave_up();    // device addresses of the files' flags
unsigned int* ff_backward_gave_up();

}  // namespace gpga
