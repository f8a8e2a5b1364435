// Dropout from a counter-based generator and layer norm, forward and backward.
#include "../../include/gpga.h"
#include "gpga_launch.cuh"
#include "gpga_norm.cuh"

namespace gpga {

namespace {

constexpr int kSMs = 148;

// ---- sums over the TPR threads of a row -------------------------------------------------------------
// TPR <= 32: lanes of one warp (the other groups of the warp may have left).  Wider: the whole block, through
// shared memory; `part` holds 32 floats per call site and round, so that one barrier per sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part)
{
    if constexpr (TPR <= 32) {
        const unsigned mask = TPR == 32 ? 0xFFFFFFFFu : ((1u << (TPR & 31)) - 1u) << ((threadIdx.x & 31) / TPR * TPR);
#pragma unroll
        for (int o = TPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(mask, v, o);
        return v;
    } else {
        v = warp_sum_f(v);
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 32; ++w) s += part[w];
        return s;
    }
}

// ---- dropout ----------------------------------------------------------------------------------------
template <class T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const DropoutParams p)
{
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const uint64_t total = (uint64_t)p.nodes * p.rows * chunks;
    const uint64_t g = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (g >= total) return;
    const uint32_t row = (uint32_t)(g / chunks), chunk = (uint32_t)(g - (uint64_t)row * chunks);
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const int col = (int)chunk * kChunk;
    Raw8<T, VEC> raw;
    float v[8];
    raw.load(static_cast<const T*>(p.x) + (int64_t)row * p.ldx, col, p.d);
    raw.get(v);
    drop8(p.mask, t, node, chunks, chunk, v);
    store8<T, VEC>(static_cast<T*>(p.y) + (int64_t)row * p.ldy, col, p.d, v);
}

// ---- layer norm, forward ----------------------------------------------------------------------------
// z = residual + dropout(x) of one chunk in fp32.
template <class T, bool VEC>
__device__ __forceinline__ void mix8(const NormForwardParams& p, const Raw8<T, VEC>& rx, const Raw8<T, VEC>& rr, uint32_t t,
                                     uint32_t node, uint32_t chunks, uint32_t chunk, float* v)
{
    rx.get(v);
    if (p.mask.threshold) drop8(p.mask, t, node, chunks, chunk, v);
    if (p.residual) {
        float r[8];
        rr.get(r);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += r[j];
    }
}

template <class T, bool VEC>
__device__ __forceinline__ void norm_store8(const NormForwardParams& p, int64_t row, uint32_t node, int col, const float* v,
                                            float mean, float rstd)
{
    float w[8], b[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 1.f, b[j] = 0.f;
    if (p.weight) param8(p.weight + node * p.ldw, col, p.d, p.wvec, w);
    if (p.bias) param8(p.bias + node * p.ldw, col, p.d, p.wvec, b);
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = fmaf((v[j] - mean) * rstd, w[j], b[j]);
    if (p.z) store8<T, VEC>(static_cast<T*>(p.z) + row * p.ldz, col, p.d, v);
    store8<T, VEC>(static_cast<T*>(p.y) + row * p.ldy, col, p.d, y);
}

// TPR threads per row, NC chunks of eight columns per thread: the row stays in registers between the mean,
// the variance (a second pass over the registers, so no cancellation) and the output.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_forward_kernel(const NormForwardParams p)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, RPB = BLOCK / TPR;
    __shared__ float part[2][32];
    const int lane = threadIdx.x % TPR;
    const uint32_t row = blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= p.nodes * p.rows) return;   // whole groups only; with TPR > 32 a block is one row
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const T* x = static_cast<const T*>(p.x) + (int64_t)row * p.ldx;
    const T* r = static_cast<const T*>(p.residual) + (p.residual ? (int64_t)row * p.ldr : 0);
    Raw8<T, VEC> rx[NC], rr[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t chunk = lane + c * TPR;
        if (chunk < chunks) {
            rx[c].load(x, chunk * kChunk, p.d);
            if (p.residual) rr[c].load(r, chunk * kChunk, p.d);
        }
    }
    float v[NC][8];
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t chunk = lane + c * TPR;
        if (chunk < chunks) {
            mix8<T, VEC>(p, rx[c], rr[c], t, node, chunks, chunk, v[c]);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += v[c][j];   // columns from d on are zero
        }
    }
    const float mean = row_sum<TPR>(sum, part[0]) / (float)p.d;
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int col = (lane + c * TPR) * kChunk;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (VEC ? col < p.d : col + j < p.d) {
                const float e = v[c][j] - mean;
                sq = fmaf(e, e, sq);
            }
    }
    const float var = row_sum<TPR>(sq, part[1]) / (float)p.d;
    const float rstd = 1.f / sqrtf(var + p.eps);
    if (lane == 0) {
        p.mean[row] = mean;
        p.rstd[row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t chunk = lane + c * TPR;
        if (chunk < chunks) norm_store8<T, VEC>(p, row, node, chunk * kChunk, v[c], mean, rstd);
    }
}

// Rows of any width: one block per row, three passes over it (the second and third mostly from L2).
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(const NormForwardParams p)
{
    __shared__ float part[2][32];
    const uint32_t row = blockIdx.x;
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const T* x = static_cast<const T*>(p.x) + (int64_t)row * p.ldx;
    const T* r = static_cast<const T*>(p.residual) + (p.residual ? (int64_t)row * p.ldr : 0);
    auto chunk_of = [&](uint32_t chunk, float* v) {
        Raw8<T, VEC> rx, rr;
        rx.load(x, chunk * kChunk, p.d);
        if (p.residual) rr.load(r, chunk * kChunk, p.d);
        mix8<T, VEC>(p, rx, rr, t, node, chunks, chunk, v);
    };
    float v[8];
    float sum = 0.f;
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_of(chunk, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[j];
    }
    const float mean = row_sum<1024>(sum, part[0]) / (float)p.d;
    float sq = 0.f;
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_of(chunk, v);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((int)chunk * kChunk + j < p.d) sq = fmaf(v[j] - mean, v[j] - mean, sq);
    }
    const float rstd = 1.f / sqrtf(row_sum<1024>(sq, part[1]) / (float)p.d + p.eps);
    if (threadIdx.x == 0) {
        p.mean[row] = mean;
        p.rstd[row] = rstd;
    }
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_of(chunk, v);
        norm_store8<T, VEC>(p, row, node, chunk * kChunk, v, mean, rstd);
    }
}

// ---- layer norm, backward ---------------------------------------------------------------------------
// g = rstd (h - mean(h) - xh mean(h xh)) + dz of one chunk, h = w dy and xh = (z - mean) rstd given.
template <class T, bool VEC>
__device__ __forceinline__ void grad_store8(const NormBackwardParams& p, int64_t row, uint32_t t, uint32_t node, uint32_t chunks,
                                            uint32_t chunk, const float* h, const float* xh, float rstd, float mh, float mhx)
{
    const int col = chunk * kChunk;
    float g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = rstd * (h[j] - mh - xh[j] * mhx);
    if (p.dz) {
        Raw8<T, VEC> raw;
        float e[8];
        raw.load(static_cast<const T*>(p.dz) + row * p.lddz, col, p.d);
        raw.get(e);
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] += e[j];
    }
    store8<T, VEC>(static_cast<T*>(p.dres) + row * p.lddres, col, p.d, g);
    if (p.dx) {
        drop8(p.mask, t, node, chunks, chunk, g);
        store8<T, VEC>(static_cast<T*>(p.dx) + row * p.lddx, col, p.d, g);
    }
}

// A block takes every splits-th group of rows of one node; each thread keeps the column sums of its chunks
// (dw += dy xh, db += dy) in registers and the block leaves one pair of rows of partial sums.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_backward_kernel(const NormBackwardParams p)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, RPB = BLOCK / TPR;
    __shared__ float part[2][RPB > 1 ? RPB : 1][32];
    extern __shared__ float sums[];   // 2 x d, only when RPB > 1
    const int lane = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    const uint32_t node = blockIdx.y;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    float dw[NC][8], db[NC][8];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[c][j] = db[c][j] = 0.f;

    for (uint32_t t0 = blockIdx.x * RPB; t0 < p.rows; t0 += gridDim.x * RPB) {
        const uint32_t t = t0 + sub;
        const bool live = t < p.rows;
        const int64_t row = (int64_t)node * p.rows + t;
        if (TPR <= 32 && !live) continue;
        Raw8<T, VEC> rz[NC], rdy[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t chunk = lane + c * TPR;
            if (chunk < chunks) {
                rz[c].load(static_cast<const T*>(p.z) + row * p.ldz, chunk * kChunk, p.d);
                rdy[c].load(static_cast<const T*>(p.dy) + row * p.lddy, chunk * kChunk, p.d);
            }
        }
        const float mean = p.mean[row], rstd = p.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        float xh[NC][8], h[NC][8];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t chunk = lane + c * TPR;
            if (chunk < chunks) {
                float w[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) w[j] = 1.f;
                if (p.weight) param8(p.weight + node * p.ldw, chunk * kChunk, p.d, p.wvec, w);
                rz[c].get(xh[c]);
                rdy[c].get(h[c]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // columns from d on have dy = 0 and so add nothing anywhere
                    xh[c][j] = (xh[c][j] - mean) * rstd;
                    db[c][j] += h[c][j];
                    dw[c][j] = fmaf(h[c][j], xh[c][j], dw[c][j]);
                    h[c][j] *= w[j];
                    s1 += h[c][j];
                    s2 = fmaf(h[c][j], xh[c][j], s2);
                }
            }
        }
        const float mh = row_sum<TPR>(s1, part[0][0]) / (float)p.d;
        const float mhx = row_sum<TPR>(s2, part[1][0]) / (float)p.d;
        if (TPR > 32) __syncthreads();   // part is reused by the next row
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t chunk = lane + c * TPR;
            if (chunk < chunks) grad_store8<T, VEC>(p, row, t, node, chunks, chunk, h[c], xh[c], rstd, mh, mhx);
        }
    }
    if (!p.dweight && !p.dbias) return;

    // the block's sums: its groups of rows one after the other, then out
    if constexpr (RPB > 1) {
        for (int s = 0; s < RPB; ++s) {
            if (s) __syncthreads();
            if (sub == s)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int col = (lane + c * TPR) * kChunk + j;
                        if (col < p.d) {
                            sums[col] = (s ? sums[col] : 0.f) + dw[c][j];
                            sums[p.d + col] = (s ? sums[p.d + col] : 0.f) + db[c][j];
                        }
                    }
        }
        __syncthreads();
    }
    float *ow, *ob;
    bool add = false;
    if (p.splits > 1) {
        ow = p.partial + ((int64_t)node * p.splits + blockIdx.x) * 2 * p.d;
        ob = ow + p.d;
    } else {
        ow = p.dweight ? p.dweight + node * p.lddw : nullptr;
        ob = p.dbias ? p.dbias + node * p.lddw : nullptr;
        add = p.accumulate;
    }
    if constexpr (RPB > 1) {
        for (int col = threadIdx.x; col < p.d; col += BLOCK) {
            if (ow) ow[col] = (add ? ow[col] : 0.f) + sums[col];
            if (ob) ob[col] = (add ? ob[col] : 0.f) + sums[p.d + col];
        }
    } else {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int col = (lane + c * TPR) * kChunk + j;
                if (col < p.d) {
                    if (ow) ow[col] = (add ? ow[col] : 0.f) + dw[c][j];
                    if (ob) ob[col] = (add ? ob[col] : 0.f) + db[c][j];
                }
            }
    }
}

// Rows of any width: the gradient of z, one block per row, two passes over it.
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(const NormBackwardParams p)
{
    __shared__ float part[2][32];
    const uint32_t row = blockIdx.x;
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const float mean = p.mean[row], rstd = p.rstd[row];
    auto chunk_of = [&](uint32_t chunk, float* h, float* xh) {
        Raw8<T, VEC> rz, rdy;
        float w[8];
        rz.load(static_cast<const T*>(p.z) + (int64_t)row * p.ldz, chunk * kChunk, p.d);
        rdy.load(static_cast<const T*>(p.dy) + (int64_t)row * p.lddy, chunk * kChunk, p.d);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = 1.f;
        if (p.weight) param8(p.weight + node * p.ldw, chunk * kChunk, p.d, p.wvec, w);
        rz.get(xh);
        rdy.get(h);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            xh[j] = (xh[j] - mean) * rstd;
            h[j] *= w[j];
        }
    };
    float h[8], xh[8];
    float s1 = 0.f, s2 = 0.f;
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_of(chunk, h, xh);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s1 += h[j];
            s2 = fmaf(h[j], xh[j], s2);
        }
    }
    const float mh = row_sum<1024>(s1, part[0]) / (float)p.d;
    const float mhx = row_sum<1024>(s2, part[1]) / (float)p.d;
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_of(chunk, h, xh);
        grad_store8<T, VEC>(p, row, t, node, chunks, chunk, h, xh, rstd, mh, mhx);
    }
}

// The column sums alone, for the rows that the kernel above takes.  It runs before that kernel: an output may
// replace dy or z.
template <class T, bool VEC>
__global__ void __launch_bounds__(128) norm_columns_kernel(const NormBackwardParams p)
{
    const uint32_t node = blockIdx.z;
    const int col = (blockIdx.x * 128 + threadIdx.x) * kChunk;
    if (col >= p.d) return;
    float dw[8] = {}, db[8] = {};
    for (uint32_t t = blockIdx.y; t < p.rows; t += gridDim.y) {
        const int64_t row = (int64_t)node * p.rows + t;
        Raw8<T, VEC> rz, rdy;
        float z[8], dy[8];
        rz.load(static_cast<const T*>(p.z) + row * p.ldz, col, p.d);
        rdy.load(static_cast<const T*>(p.dy) + row * p.lddy, col, p.d);
        const float mean = p.mean[row], rstd = p.rstd[row];
        rz.get(z);
        rdy.get(dy);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dw[j] = fmaf(dy[j], (z[j] - mean) * rstd, dw[j]);
            db[j] += dy[j];
        }
    }
    const bool add = p.splits == 1 && p.accumulate;
    float* ow = p.splits > 1 ? p.partial + ((int64_t)node * p.splits + blockIdx.y) * 2 * p.d
                             : p.dweight ? p.dweight + node * p.lddw : nullptr;
    float* ob = p.splits > 1 ? ow + p.d : p.dbias ? p.dbias + node * p.lddw : nullptr;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (col + j < p.d) {
            if (ow) ow[col + j] = (add ? ow[col + j] : 0.f) + dw[j];
            if (ob) ob[col + j] = (add ? ob[col + j] : 0.f) + db[j];
        }
}

// dw and db from the blocks' partial sums: 32 columns per block, eight warps take every eighth partial, and
// their sums are added in the order of the warps.  Deterministic: no atomics.
__global__ void __launch_bounds__(256) norm_params_kernel(const NormBackwardParams p)
{
    __shared__ float part[8][32];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;   // over 2 d: dw, then db
    const uint32_t node = blockIdx.y;
    const int64_t d2 = 2 * (int64_t)p.d;
    grid_dependency_wait();
    float s = 0.f;
    if (col < d2) {
        const float* src = p.partial + (int64_t)node * p.splits * d2 + col;
#pragma unroll 8
        for (int b = wid; b < p.splits; b += 8) s += src[b * d2];
    }
    part[wid][lane] = s;
    __syncthreads();
    if (wid || col >= d2) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) s += part[w][lane];
    float* out = col < p.d ? p.dweight : p.dbias;
    if (!out) return;
    out += node * p.lddw + (col < p.d ? col : col - p.d);
    *out = (p.accumulate ? *out : 0.f) + s;
}

__global__ void zero_params_kernel(const NormBackwardParams p)
{
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= p.d) return;
    if (p.dweight) p.dweight[blockIdx.y * p.lddw + col] = 0.f;
    if (p.dbias) p.dbias[blockIdx.y * p.lddw + col] = 0.f;
}

// ---- launches ---------------------------------------------------------------------------------------
constexpr int kForwardWide = 16384, kBackwardWide = 8192;   // widest rows that stay in registers

template <class T, bool VEC, int TPR, int NC>
cudaError_t forward_as(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, RPB = BLOCK / TPR;
    const uint32_t rows = p.nodes * p.rows;
    norm_forward_kernel<T, VEC, TPR, NC><<<(rows + RPB - 1) / RPB, BLOCK, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t forward_of(const NormForwardParams& p, cudaStream_t s)
{
    if (p.d <= 64) return forward_as<T, VEC, 8, 1>(p, s);
    if (p.d <= 256) return forward_as<T, VEC, 32, 1>(p, s);
    if (p.d <= 512) return forward_as<T, VEC, 32, 2>(p, s);
    if (p.d <= 1024) return forward_as<T, VEC, 32, 4>(p, s);
    if (p.d <= 2048) return forward_as<T, VEC, 128, 2>(p, s);
    if (p.d <= 4096) return forward_as<T, VEC, 128, 4>(p, s);
    if (p.d <= 8192) return forward_as<T, VEC, 512, 2>(p, s);
    if (p.d <= kForwardWide) return forward_as<T, VEC, 512, 4>(p, s);
    norm_forward_wide_kernel<T, VEC><<<p.nodes * p.rows, 1024, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC, int TPR, int NC>
cudaError_t backward_as(const NormBackwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, RPB = BLOCK / TPR;
    norm_backward_kernel<T, VEC, TPR, NC><<<dim3(p.splits, p.nodes), BLOCK, RPB > 1 ? 2 * p.d * sizeof(float) : 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t backward_of(const NormBackwardParams& p, cudaStream_t s)
{
    if (p.d <= 64) return backward_as<T, VEC, 8, 1>(p, s);
    if (p.d <= 256) return backward_as<T, VEC, 32, 1>(p, s);
    if (p.d <= 512) return backward_as<T, VEC, 32, 2>(p, s);
    if (p.d <= 1024) return backward_as<T, VEC, 32, 4>(p, s);
    if (p.d <= 2048) return backward_as<T, VEC, 256, 1>(p, s);
    if (p.d <= 4096) return backward_as<T, VEC, 512, 1>(p, s);
    if (p.d <= kBackwardWide) return backward_as<T, VEC, 512, 2>(p, s);
    if (p.dweight || p.dbias) {
        norm_columns_kernel<T, VEC><<<dim3((p.d + 1023) / 1024, p.splits, p.nodes), 128, 0, s>>>(p);
        const cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    norm_backward_wide_kernel<T, VEC><<<p.nodes * p.rows, 1024, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace

#define GPGA_BY_TYPE(call)                                                              \
    (dtype == GPGA_DTYPE_F32    ? (vec ? call(float, true) : call(float, false))        \
     : dtype == GPGA_DTYPE_BF16 ? (vec ? call(__nv_bfloat16, true) : call(__nv_bfloat16, false)) \
                                : (vec ? call(__half, true) : call(__half, false)))

cudaError_t launch_dropout(const DropoutParams& p, int dtype, bool vec, cudaStream_t s)
{
    const uint64_t total = (uint64_t)p.nodes * p.rows * ((p.d + kChunk - 1) / kChunk);
    if (!total) return cudaSuccess;
    const unsigned grid = (unsigned)((total + 255) / 256);
#define GPGA_CALL(T, V) (dropout_kernel<T, V><<<grid, 256, 0, s>>>(p), cudaGetLastError())
    return GPGA_BY_TYPE(GPGA_CALL);
#undef GPGA_CALL
}

cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, bool vec, cudaStream_t s)
{
    if (!p.rows) return cudaSuccess;
#define GPGA_CALL(T, V) forward_of<T, V>(p, s)
    return GPGA_BY_TYPE(GPGA_CALL);
#undef GPGA_CALL
}

int norm_backward_splits(int64_t nodes, int64_t rows, int64_t d)
{
    if (rows < 1) return 1;
    // rows a block works on at a time, and blocks that fit an SM
    const int64_t rpb = d <= 64 ? 32 : d <= 1024 ? 8 : 1;
    const int64_t per_sm = d <= 512 ? 3 : d <= 4096 ? 2 : 1;
    int64_t splits = (kSMs * per_sm + nodes - 1) / nodes;
    const int64_t groups = (rows + rpb - 1) / rpb;
    if (splits > groups) splits = groups;
    return (int)(splits < 1 ? 1 : splits);
}

cudaError_t launch_norm_backward(const NormBackwardParams& p, int dtype, bool vec, cudaStream_t s)
{
    const bool params = p.dweight || p.dbias;
    if (!p.rows) {
        if (!params || p.accumulate) return cudaSuccess;
        zero_params_kernel<<<dim3((p.d + 255) / 256, p.nodes), 256, 0, s>>>(p);
        return cudaGetLastError();
    }
#define GPGA_CALL(T, V) backward_of<T, V>(p, s)
    const cudaError_t e = GPGA_BY_TYPE(GPGA_CALL);
#undef GPGA_CALL
    if (e != cudaSuccess || p.splits == 1 || !params) return e;
    norm_params_kernel<<<dim3((unsigned)((2 * (int64_t)p.d + 31) / 32), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

}  // namespace gpga
