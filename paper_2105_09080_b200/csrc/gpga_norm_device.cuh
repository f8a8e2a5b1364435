// What the dropout and layer norm kernels share: how a row is spread over threads, sums over them, dispatch by type.
#pragma once
#include "../../include/gpga.h"
#include "gpga_launch.cuh"
#include "gpga_norm.cuh"
#include "gpga_tma.cuh"

namespace gpga {

constexpr int kSMs = 148;

// Chunk c of a thread.  A group of at most 32 threads takes neighbouring chunks call by call; in wider groups every
// warp has NC * 32 neighbouring chunks, so that only its two ends meet other warps' columns.
template <int TPR, int NC>
__device__ __forceinline__ uint32_t chunk_of(int c)
{
    if (TPR <= 32) return threadIdx.x % TPR + c * TPR;
    return (threadIdx.x % TPR / 32 * NC + c) * 32 + threadIdx.x % 32;
}
// First chunk of the lanes that share a store with this thread, for its chunk c.
template <int TPR, int NC>
__device__ __forceinline__ uint32_t first_chunk_of(int c)
{
    return TPR <= 32 ? c * TPR : (threadIdx.x % TPR / 32 * NC + c) * 32;
}
// Threads of a block for groups of TPR: several groups of up to 64, one wider one.
__host__ __device__ constexpr int block_of(int tpr) { return tpr <= 64 ? 128 : tpr; }
__host__ __device__ constexpr int lanes_of(int tpr) { return tpr < 32 ? tpr : 32; }

// 16 bytes from memory to shared memory without a register; a thread waits for its own copies.
__device__ __forceinline__ void copy16_async(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Chunks of R rows on their way to a warp through its own places in shared memory, so that loads in flight take no registers;
// place: [tensor][r][c][warp][piece].  In fp32 a chunk is two 16-byte pieces (Q); lanes copy neighbouring pieces, so that
// whole sectors come at once, and the pieces lie exchanged in every other group of eight, so that a warp reads its chunks
// without bank conflicts.  A group's lanes synchronise between copies that have landed and reads, where Q > 1 or rows are shifted.
template <class T, bool SHIFT, int TPR, int NC, int R> struct Staged {
    static constexpr int BLOCK = block_of(TPR), LANES = lanes_of(TPR), Q = sizeof(T) / 2, E = 16 / sizeof(T);   // E: columns of a piece
    uint4* stage;
    int d, shift, lane;
    __device__ __forceinline__ uint4* place(int tensor, int r, int c, int piece) const
    {
        const int at = Q == 1 ? piece : piece ^ (piece >> 3 & 1);
        return stage + (((tensor * R + r) * NC + c) * BLOCK + (threadIdx.x - lane)) * Q + at;
    }
    // full: every chunk is there
    __device__ __forceinline__ void fetch(const T* row, const Span& s, int tensor, int r, bool full) const
    {
        const bool in = !SHIFT || inside(row, d, s);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int piece = q * LANES + lane, at = (int)first_chunk_of<TPR, NC>(c) * kChunk - shift + piece * E;
                if (!full && at >= d) continue;
                const T* from = row + at;
                uint4* to = place(tensor, r, c, piece);
                if (in || (at >= 0 && at + E <= d)) {
                    copy16_async(smem_u32(to), from);
                } else {   // the array's first and last rows
#pragma unroll 1
                    for (int e = 0; e < E; ++e) reinterpret_cast<T*>(to)[e] = at + e >= 0 && at + e < d ? from[e] : from_f32<T>(0.f);
                }
            }
    }
    __device__ __forceinline__ void chunk(int tensor, int r, int c, f32x2_t* v) const
    {
        Raw8<T, true> raw;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const uint4 x = *place(tensor, r, c, Q * lane + q);
            raw.w[4 * q] = x.x; raw.w[4 * q + 1] = x.y; raw.w[4 * q + 2] = x.z; raw.w[4 * q + 3] = x.w;
        }
        raw.get(v);
    }
};

// Sums of M values over L lanes; lane l is left with value l / (L / M).  M values take M - 1 shuffles to halve down to one
// per lane (a lane gives away the half it does not keep), the remaining steps on that one.
template <int L, int M>
__device__ __forceinline__ float lane_sums(float* v, unsigned mask)
{
    const int lane = threadIdx.x % L;
    int o = L / 2;
#pragma unroll
    for (int m = M / 2; m >= 1; m /= 2, o /= 2) {
        const bool upper = lane & o;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float give = upper ? v[i] : v[i + m], keep = upper ? v[i + m] : v[i];
            v[i] = keep + __shfl_xor_sync(mask, give, o);
        }
    }
#pragma unroll
    for (; o >= 1; o /= 2) v[0] += __shfl_xor_sync(mask, v[0], o);
    return v[0];
}
// Hands the M sums round: every lane gets them all.
template <int L, int M>
__device__ __forceinline__ void share_sums(float mine, float* v, unsigned mask)
{
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = M > 1 ? __shfl_sync(mask, mine, i * (L / M), L) : mine;
}

// Sums of M values over the TPR threads of a group; every thread gets them all: 17 shuffles for M = 8 in a warp instead of
// 40.  Wider groups go on through shared memory: one barrier; `part` ([warps][M], on 16 bytes) may be used again by the
// next call but one.  Up to seven warps' sums are read by every thread, more are added by the lanes once more (32 warps'
// pairs: 20 instructions instead of 130).
template <int TPR, int M>
__device__ __forceinline__ void group_sums(float* v, float* part)
{
    constexpr int L = lanes_of(TPR), W = TPR / 32;
    const unsigned mask = group_mask<TPR>();
    const float mine = lane_sums<L, M>(v, mask);
    if constexpr (TPR <= 32) {
        share_sums<L, M>(mine, v, mask);
    } else {
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, w0 = threadIdx.x / TPR * W;
        if (lane % (L / M) == 0) part[warp * M + lane / (L / M)] = mine;
        __syncthreads();
        if constexpr (W >= 8) {
#pragma unroll
            for (int i = 0; i < M; ++i) v[i] = lane < W ? part[(w0 + lane) * M + i] : 0.f;
            share_sums<32, M>(lane_sums<32, M>(v, mask), v, mask);
        } else if constexpr (M >= 4) {
            f32x2_t sum[M / 2];
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int i = 0; i < M / 4; ++i) {
                    const float4 q = reinterpret_cast<const float4*>(part)[(w0 + w) * (M / 4) + i];
                    sum[2 * i] = w ? add2(sum[2 * i], pack2(q.x, q.y)) : pack2(q.x, q.y);
                    sum[2 * i + 1] = w ? add2(sum[2 * i + 1], pack2(q.z, q.w)) : pack2(q.z, q.w);
                }
#pragma unroll
            for (int i = 0; i < M; ++i) v[i] = element(sum, i);
        } else {
#pragma unroll
            for (int i = 0; i < M; ++i) v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int i = 0; i < M; ++i) v[i] += part[(w0 + w) * M + i];
        }
    }
}

}  // namespace gpga

// call(type, vec) for the activation type `dtype` and the runtime `vec`.
#define GPGA_BY_TYPE(call)                                                              \
    (dtype == GPGA_DTYPE_F32    ? (vec ? call(float, true) : call(float, false))        \
     : dtype == GPGA_DTYPE_BF16 ? (vec ? call(__nv_bfloat16, true) : call(__nv_bfloat16, false)) \
                                : (vec ? call(__half, true) : call(__half, false)))
