// Embedding lookup and its gradient: launch parameters (kernels in gpga_embed.cu).
#pragma once
#include "gpga_token.cuh"

namespace gpga {

struct LookupParams {
    const float* table;
    const void* tokens;
    void* out;
    int64_t ldt, node_ldt;   // row and node stride of the table
    int64_t ldo;             // row stride of out
    uint32_t nodes, rows, vocab;
    int32_t d;
    bool tokens64;
    float scale;
    Divisor stretches;       // of a row, set by the launch
};

struct LookupGradParams {
    const void* dout;
    const void* tokens;
    float* grad;
    int64_t ldo;             // row stride of dout
    int64_t ldg, node_ldg;   // row and node stride of grad
    uint32_t nodes, rows, vocab;
    int32_t d;
    bool tokens64, accumulate;
    float scale;
    char* scratch;
};

cudaError_t launch_lookup(const LookupParams& p, int dtype, cudaStream_t s);
cudaError_t launch_lookup_grad(const LookupGradParams& p, int dtype, cudaStream_t s);
int64_t lookup_grad_scratch_bytes(int64_t nodes, int64_t rows, int64_t d, int64_t vocab);

}  // namespace gpga
