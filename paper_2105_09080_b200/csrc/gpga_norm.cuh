// Dropout and layer norm: launch parameters (kernels in gpga_dropout.cu, gpga_norm.cu and gpga_norm_grad.cu).
#pragma once
#include "gpga_token.cuh"

namespace gpga {

struct DropoutParams {
    const void* x;
    void* y;
    int64_t ldx, ldy;        // row strides in elements
    uint32_t nodes, rows;    // rows per node
    int32_t d;
    Divisor chunks, stretches;   // set by the launch
    bool shifted;                // rows of x and y are off the 16-byte alignment alike
    DropMask mask;
};

struct NormForwardParams {
    const void *x, *residual;      // residual may be null
    const float *weight, *bias;    // may be null
    void *y, *z;                   // z may be null
    float *mean, *rstd;
    int64_t ldx, ldr, ldy, ldz, ldw;   // row strides; ldw: node stride of weight and bias
    uint32_t nodes, rows;
    int32_t d;
    float eps;
    bool wvec;               // weight and bias rows allow 128-bit accesses
    bool shifted;            // rows of all activations are off the 16-byte alignment alike
    DropMask mask;
};

struct NormBackwardParams {
    const void *dy, *z, *dz;       // dz may be null
    const float *mean, *rstd, *weight;
    void *dres, *dx;               // dx may be null (then there is no dropout)
    float *dweight, *dbias;        // may be null
    float* partial;                // (nodes, splits, 2, d)
    int64_t lddy, ldz, lddz, lddres, lddx, ldw, lddw;   // lddw: node stride of dweight and dbias
    uint32_t nodes, rows;
    int32_t d;
    int32_t splits;          // blocks per node
    bool wvec, accumulate;
    bool shifted;            // rows of all activations are off the 16-byte alignment alike
    DropMask mask;
};

// dtype: GPGA_DTYPE_*; vec: every activation pointer and stride allows 128-bit accesses and d % 8 == 0.
cudaError_t launch_dropout(const DropoutParams& p, int dtype, bool vec, cudaStream_t s);
cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, bool vec, cudaStream_t s);
// p.splits is chosen by norm_backward_splits; p.partial may be null when it is 1.
cudaError_t launch_norm_backward(const NormBackwardParams& p, int dtype, bool vec, cudaStream_t s);
int norm_backward_splits(int64_t nodes, int64_t rows, int64_t d);

}  // namespace gpga
