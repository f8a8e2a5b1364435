// Dropout from a counter-based generator and layer norm, forward and backward.
#include "../../include/gpga.h"
#include "gpga_launch.cuh"
#include "gpga_norm.cuh"
#include "gpga_tma.cuh"

namespace gpga {

namespace {

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


// Sums of M values over the TPR threads of a group; every thread gets them all.  In a warp, M values take M - 1
// shuffles to halve down to one per lane (a lane gives away the half it does not keep), the remaining steps on that
// one, and M to hand the sums round: 17 for M = 8 instead of 40.  Wider groups go on through shared memory: one
// barrier; `part` ([warps][M], on 16 bytes) may be used again by the next call but one.
template <int TPR, int M>
__device__ __forceinline__ void group_sums(float* v, float* part)
{
    constexpr int L = lanes_of(TPR);
    const unsigned mask = group_mask<TPR>();
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
    // lane l now has value l / (L / M)
    if constexpr (TPR > 32) {
        const int warp = threadIdx.x / 32;
        if (lane % (L / M) == 0) part[warp * M + lane / (L / M)] = v[0];
        __syncthreads();
        const int w0 = threadIdx.x / TPR * (TPR / 32);
        if constexpr (M >= 4) {
            f32x2_t sum[M / 2];
#pragma unroll
            for (int w = 0; w < TPR / 32; ++w)
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
            for (int w = 0; w < TPR / 32; ++w)
#pragma unroll
                for (int i = 0; i < M; ++i) v[i] += part[(w0 + w) * M + i];
        }
    } else if constexpr (M > 1) {
        const float mine = v[0];
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] = __shfl_sync(mask, mine, i * (L / M), L);
    }
}

// ---- dropout ----------------------------------------------------------------------------------------
// Both tensors dense and aligned: U chunks per thread, 256 apart, their loads in flight together; no index arithmetic per
// chunk but an addition (with a division by the row's length and 64-bit products it took 134 instructions per chunk instead
// of 97, and issue slots bounded it).  Bound: HBM.  8 x 4096 x 4096 bf16 80 us = 6.7 TB/s, one chunk per thread 118 us.
template <class T, int U>
__global__ void __launch_bounds__(256) dropout_dense_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, total = p.rows * p.chunks.d;
    const T* x = static_cast<const T*>(p.x) + (int64_t)node * total * kChunk;
    T* y = static_cast<T*>(p.y) + (int64_t)node * total * kChunk;
    const uint32_t f0 = blockIdx.x * (256 * U) + threadIdx.x;   // the host keeps total + 256 U below 2^32
    Raw8<T, true> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (f0 + u * 256 < total) raw[u].load(x + (int64_t)f0 * kChunk, u * 256 * kChunk, p.d, Span());
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (f0 + u * 256 >= total) return;
        f32x2_t v[4];
        raw[u].get(v);
        drop8(p.mask, f0 + u * 256, node, v);
        store8<T>(y + (int64_t)f0 * kChunk + u * 256 * kChunk, v);
    }
}

// Otherwise TPR lanes take a stretch of NC * TPR chunks of one row.
template <class T, bool VEC, int TPR, int NC>
__global__ void __launch_bounds__(256) dropout_rows_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, chunks = p.chunks.d;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const uint32_t first = (g - t * p.stretches.d) * (NC * TPR);
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)node * p.rows + t;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
    const Span span = span_of<T>(p.x, p.ldx, (int64_t)p.nodes * p.rows, p.d);
    Raw8<T, VEC> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (!VEC || first + c * TPR + lane < chunks) raw[c].load(x, (int)(first + c * TPR + lane) * kChunk, p.d, span);
    RowStore<T, VEC, TPR> store;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t base = first + c * TPR, chunk = base + lane;
        if (base >= chunks) break;
        f32x2_t v[4];
        if (!VEC || chunk < chunks) {
            raw[c].get(v);
            drop8(p.mask, t * chunks + chunk, node, v);
        }
        store.store(y, (int)chunk * kChunk, p.d, v, lane, group_mask<TPR>(), c + 1 == NC || base + TPR >= chunks);
    }
}

// Rows of x and y off the alignment alike: shifted chunks.  p.stretches counts those of the widest shift.  8 x 4096 rows
// of 2001 bf16 columns 70 us (cut chunks 93 us, single elements 157 us; an aligned row's rate would be 40 us): the words of
// a neighbour's generator call, shuffled and cut, are what it pays.
template <class T, int TPR, int NC>
__global__ void __launch_bounds__(256) dropout_shifted_kernel(const DropoutParams p)
{
    const uint32_t node = blockIdx.y, chunks = p.chunks.d;
    const uint32_t g = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    const uint32_t t = divide(g, p.stretches);
    if (t >= p.rows) return;
    const int64_t row = (int64_t)node * p.rows + t;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    T* y = static_cast<T*>(p.y) + row * p.ldy;
    const int lane = threadIdx.x % TPR, shift = shift_of(x);
    const uint32_t first = (g - t * p.stretches.d) * (NC * TPR);
    if ((int)first * kChunk - shift >= p.d) return;
    __shared__ __align__(16) T slots[256 / TPR][16];
    const Span span = span_of<T>(p.x, p.ldx, (int64_t)p.nodes * p.rows, p.d);
    auto col = [&](int c) { return (int)(first + c * TPR + lane) * kChunk - shift; };
    Raw8<T, true> raw[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c)
        if (col(c) < p.d) load_shifted(x, col(c), p.d, span, raw[c], slots[threadIdx.x / TPR]);
    const uint32_t groups = t * chunks + first;
    uint4 before = make_uint4(0, 0, 0, 0);
    if (p.mask.on && shift) before = drop_words(p.mask, groups - 1, node);
    f32x2_t v[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        raw[c].get(v[c]);
        if (p.mask.on) {
            const uint4 own = drop_words(p.mask, groups + c * TPR + lane, node);
            const uint4 left = shfl4(group_mask<TPR>(), own, (lane + TPR - 1) % TPR, TPR);
            uint32_t word[4];
            shifted_words(lane ? left : before, own, shift, word);
            before = left;   // lane 0 has the last lane's
            drop8_by(p.mask, word, v[c]);
        }
    }
    store_shifted<T, TPR, NC>(y, col(0), p.d, shift, v, slots[threadIdx.x / TPR], lane, group_mask<TPR>());
}

// ---- layer norm, forward ----------------------------------------------------------------------------
// (z - mean) rstd w + b
__device__ __forceinline__ void scale8(const f32x2_t* v, float mean, float rstd, const f32x2_t* w, const f32x2_t* b, f32x2_t* y)
{
    const f32x2_t m = both(mean), s = both(rstd);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fma2(mul2(sub2(v[j], m), s), w[j], b[j]);
}

__device__ __forceinline__ f32x2_t sum4(const f32x2_t* v) { return add2(add2(v[0], v[1]), add2(v[2], v[3])); }

// Sum of (v - mean)^2 over the columns of a chunk at column `col` that lie in the row; EDGE: some may not.
template <bool EDGE>
__device__ __forceinline__ f32x2_t squares8(const f32x2_t* v, float mean, int col, int d)
{
    const f32x2_t m = both(mean);
    f32x2_t e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = sub2(v[j], m);
    if (EDGE) keep_columns(e, columns_there(col, d));
    f32x2_t s = mul2(e[0], e[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) s = fma2(e[j], e[j], s);
    return s;
}

// s / n for a row's mean: one multiplication by fl(1 / n), corrected by the exact remainder.  (A constant row's mean is
// exact this way, as by a division, which takes several times the instructions.)
__device__ __forceinline__ float mean_of(float s, float n, float inv_n)
{
    const float m = s * inv_n;
    const float fixed = fmaf(fmaf(-m, n, s), inv_n, m);
    return fabsf(fixed) <= 3.4e38f ? fixed : m;   // an infinite sum has no remainder
}

// Statistics of R rows that a group of TPR threads holds in registers (columns and rows that are not there: zero).  The
// variance is a second pass over the registers, so that nothing cancels.  FULL: every chunk is there; EDGE: chunks may be
// partial.  Chunk m starts at column 8 m - shift.
template <bool FULL, bool EDGE, int TPR, int NC, int R>
__device__ __forceinline__ void row_statistics(const f32x2_t (*v)[NC][4], int d, int shift, float eps, float* part, float* mean, float* rstd)
{
    const float n = (float)d, inv_n = 1.f / n;
    float s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        f32x2_t sum = sum4(v[r][0]);
#pragma unroll
        for (int c = 1; c < NC; ++c) sum = add2(sum, sum4(v[r][c]));
        s[r] = sum2(sum);
    }
    group_sums<TPR, R>(s, part);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mean[r] = mean_of(s[r], n, inv_n);
        f32x2_t sum = both(0.f);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int col = (int)chunk_of<TPR, NC>(c) * kChunk - shift;
            if (FULL || col < d) sum = add2(sum, squares8<EDGE>(v[r][c], mean[r], col, d));
        }
        s[r] = sum2(sum);
    }
    group_sums<TPR, R>(s, part + 32 * R);
#pragma unroll
    for (int r = 0; r < R; ++r) rstd[r] = rsqrtf(fmaf(s[r], inv_n, eps));   // within 2 ulp
}

// z = residual + dropout(x) of R rows from row t of a node on, in fp32; zero where there is no row or chunk.  The
// branches are the same for the whole launch and stand outside the loops.
template <class T, bool FULL, bool VEC, int TPR, int NC, int R>
__device__ __forceinline__ void load_mixed(const NormForwardParams& p, uint32_t node, uint32_t t, f32x2_t (*v)[NC][4])
{
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const int64_t all = (int64_t)p.nodes * p.rows, row0 = (int64_t)node * p.rows + t;
    const Span sx = span_of<T>(p.x, p.ldx, all, p.d), sr = span_of<T>(p.residual, p.ldr, all, p.d);
    Raw8<T, VEC> rx[R][NC], rr[R][NC];
    const T* x = static_cast<const T*>(p.x) + row0 * p.ldx;
    const T* res = static_cast<const T*>(p.residual) + (p.residual ? row0 * p.ldr : 0);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if (FULL || (t + r < p.rows && chunk_of<TPR, NC>(c) < chunks)) rx[r][c].load(x + r * p.ldx, chunk_of<TPR, NC>(c) * kChunk, p.d, sx);
    if (p.residual)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (FULL || (t + r < p.rows && chunk_of<TPR, NC>(c) < chunks))
                    rr[r][c].load(res + r * p.ldr, chunk_of<TPR, NC>(c) * kChunk, p.d, sr);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if (FULL || (t + r < p.rows && chunk_of<TPR, NC>(c) < chunks)) rx[r][c].get(v[r][c]);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) v[r][c][j] = both(0.f);
        }
    if (p.mask.on)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) drop8(p.mask, (t + r) * chunks + chunk_of<TPR, NC>(c), node, v[r][c]);
    if (p.residual)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (FULL || (t + r < p.rows && chunk_of<TPR, NC>(c) < chunks)) {
                    f32x2_t e[4];
                    rr[r][c].get(e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][c][j] = add2(v[r][c][j], e[j]);
                }
}

// Everything aligned, weight and bias there: a group of TPR threads takes R rows, NC chunks of eight columns per
// thread, all loads first.  FULL: the block's rows and every thread's chunks are all there, nothing is tested.
// Bound: HBM.  8 x 4096 rows of 1024, residual and dropout, bf16 43 us = 6.2 TB/s, fp32 without dropout 83 us = 6.5 TB/s.  A
// warp per row and a block per four rows: persistent blocks with the next row on its way in registers took 67 us (16 to 20
// warps per SM instead of 24 to 28), and tests inside the loops over chunks twice the instructions.
template <class T, bool FULL, int TPR, int NC, int R>
__device__ __forceinline__ void norm_forward(const NormForwardParams& p, float* part)
{
    constexpr int G = (TPR < 128 ? 128 : TPR) / TPR;
    const uint32_t node = blockIdx.y, chunks = (uint32_t)p.d / kChunk;
    const uint32_t t = (blockIdx.x * G + threadIdx.x / TPR) * R;
    const int64_t row0 = (int64_t)node * p.rows + t;
    f32x2_t v[R][NC][4];
    load_mixed<T, FULL, true, TPR, NC, R>(p, node, t, v);
    float mean[R], rstd[R];
    row_statistics<FULL, false, TPR, NC, R>(v, p.d, 0, p.eps, part, mean, rstd);
    if (threadIdx.x % TPR == 0)
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (FULL || t + r < p.rows) {
                p.mean[row0 + r] = mean[r];
                p.rstd[row0 + r] = rstd[r];
            }
    if (p.z) {
        T* z = static_cast<T*>(p.z) + row0 * p.ldz;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (FULL || (t + r < p.rows && chunk_of<TPR, NC>(c) < chunks)) store8<T>(z + r * p.ldz + chunk_of<TPR, NC>(c) * kChunk, v[r][c]);
    }
    T* y = static_cast<T*>(p.y) + row0 * p.ldy;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const uint32_t chunk = chunk_of<TPR, NC>(c);
        if (!FULL && chunk >= chunks) continue;
        f32x2_t w[4], b[4];
        param8(p.weight + node * p.ldw, chunk * kChunk, p.d, true, w);
        param8(p.bias + node * p.ldw, chunk * kChunk, p.d, true, b);
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (FULL || t + r < p.rows) {
                f32x2_t out[4];
                scale8(v[r][c], mean[r], rstd[r], w, b, out);
                store8<T>(y + r * p.ldy + chunk * kChunk, out);
            }
    }
}

template <class T, int TPR, int NC, int R>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_forward_kernel(const NormForwardParams p)
{
    constexpr int G = (TPR < 128 ? 128 : TPR) / TPR;
    __shared__ __align__(16) float part[2 * 32 * R];
    if (p.d == TPR * NC * kChunk && (blockIdx.x + 1) * (G * R) <= p.rows) norm_forward<T, true, TPR, NC, R>(p, part);
    else norm_forward<T, false, TPR, NC, R>(p, part);
}

// A node's weight and bias (one and zero where there is none) laid out in shared memory, chunk m from column 8 m - shift
// on, zero beside the row; each chunk's two halves in planes of their own (no bank conflicts).
template <int BLOCK>
__device__ __forceinline__ void stage_params(const NormForwardParams& p, uint32_t node, int shift, uint32_t chunks, float4* params)
{
    for (uint32_t at = threadIdx.x; at < chunks * kChunk; at += BLOCK) {
        const int col = (int)at - shift;
        const bool in = col >= 0 && col < p.d;
        float* to = reinterpret_cast<float*>(params + (at >> 2 & 1) * chunks + (at >> 3)) + (at & 3);
        to[0] = !in ? 0.f : p.weight ? p.weight[node * p.ldw + col] : 1.f;
        to[8 * chunks] = in && p.bias ? p.bias[node * p.ldw + col] : 0.f;
    }
    __syncthreads();
}
__device__ __forceinline__ void staged_params(const float4* params, uint32_t chunks, uint32_t chunk, f32x2_t* w, f32x2_t* b)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float4 qw = params[h * chunks + chunk], qb = params[(2 + h) * chunks + chunk];
        w[2 * h] = pack2(qw.x, qw.y); w[2 * h + 1] = pack2(qw.z, qw.w);
        b[2 * h] = pack2(qb.x, qb.y); b[2 * h + 1] = pack2(qb.z, qb.w);
    }
}

// Rows off the alignment all alike: shifted chunks, which are aligned memory in every array.  A block takes sets of rows
// that have one shift, and lays out the node's parameters for it once.  Bound: latency of a row's two sums at 16 to 20 warps
// per SM, then issue slots.  2 x 5001 rows of 1023 f16 19 us (cut chunks 27 us, single elements 39 us), 4 x 8000 rows of 1001
// bf16 with residual and dropout 85 us (121, 175), fp32 without dropout 94 us (130, 227).
template <class T, int TPR, int NC, int R>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, (NC < 3 ? 640 : 512) / (TPR < 128 ? 128 : TPR)) norm_forward_shifted_kernel(const NormForwardParams p)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, G = BLOCK / TPR, LANES = lanes_of(TPR);
    constexpr uint32_t P = kShiftRows<T>;
    extern __shared__ float4 params[];
    __shared__ __align__(16) float part[2 * 32 * R];
    __shared__ __align__(16) T slots[BLOCK / LANES][16];
    const uint32_t node = blockIdx.y, chunks = (uint32_t)(p.d + kChunk - 1) / kChunk, first_row = blockIdx.x % P;
    const uint32_t rows = p.rows > first_row ? (p.rows - first_row + P - 1) / P : 0;   // first_row + P i
    const int64_t all = (int64_t)p.nodes * p.rows, row0 = (int64_t)node * p.rows + first_row;
    const int shift = shift_of(static_cast<const T*>(p.x) + row0 * p.ldx), lane = threadIdx.x % LANES;
    const uint32_t shifted = (uint32_t)(p.d + shift + kChunk - 1) / kChunk;   // chunks of a row
    const Span sx = span_of<T>(p.x, p.ldx, all, p.d), sr = span_of<T>(p.residual, p.ldr, all, p.d);
    const int col0 = (int)chunk_of<TPR, NC>(0) * kChunk - shift;
    auto col = [&](int c) { return col0 + c * LANES * kChunk; };
    T* own_slots = slots[threadIdx.x / LANES];
    uint32_t there[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) there[c] = columns_there(col(c), p.d);
    stage_params<BLOCK>(p, node, shift, shifted, params);
    const uint32_t step = gridDim.x / P * (G * R);
    uint32_t i0 = blockIdx.x / P * (G * R), i = i0 + (G == 1 ? 0 : threadIdx.x / TPR * R);
    Raw8<T, true> rx[R][NC], rr[R][NC];
    auto load = [&](uint32_t from) {   // rows first_row + P from, ...
        const int64_t at = row0 + (int64_t)from * P;
        const T* x = static_cast<const T*>(p.x) + at * p.ldx;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (from + r < rows)
#pragma unroll
                for (int c = 0; c < NC; ++c)
                    if (there[c]) load_shifted(x + r * P * p.ldx, col(c), p.d, sx, rx[r][c], own_slots);
        if (p.residual) {
            const T* res = static_cast<const T*>(p.residual) + at * p.ldr;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (from + r < rows)
#pragma unroll
                    for (int c = 0; c < NC; ++c)
                        if (there[c]) load_shifted(res + r * P * p.ldr, col(c), p.d, sr, rr[r][c], own_slots);
        }
    };
    load(i);
    for (; i0 < rows; i0 += step, i += step) {
        const int64_t at = row0 + (int64_t)i * P;   // pointers from here: fewer registers than ones that are carried along
        f32x2_t v[R][NC][4];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) rx[r][c].get(v[r][c]);
        if (p.mask.on) {
            // lane r works out the words before the warp's first chunk in row r
            const uint32_t t_edge = first_row + (i + (lane < R ? lane : 0)) * P;
            const uint4 edge = drop_words(p.mask, t_edge * chunks + first_chunk_of<TPR, NC>(0) - 1, node);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint4 before = shfl4(group_mask<TPR>(), edge, r, LANES);
                const uint32_t groups = (first_row + (i + r) * P) * chunks;
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    const uint4 own = drop_words(p.mask, groups + chunk_of<TPR, NC>(c), node);
                    const uint4 left = shfl4(group_mask<TPR>(), own, (lane + LANES - 1) % LANES, LANES);
                    uint32_t word[4];
                    shifted_words(lane ? left : before, own, shift, word);
                    before = left;   // lane 0 has the last lane's
                    drop8_by(p.mask, word, v[r][c]);
                }
            }
        }
        if (p.residual)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    f32x2_t e[4];
                    rr[r][c].get(e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][c][j] = add2(v[r][c][j], e[j]);
                }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) keep_columns(v[r][c], i + r < rows ? there[c] : 0u);   // the rest was never loaded, or lies beside the row
        load(i + step);   // on their way during the sums
        float mean[R], rstd[R];
        row_statistics<false, true, TPR, NC, R>(v, p.d, shift, p.eps, part, mean, rstd);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (i + r >= rows) continue;
            if (threadIdx.x % TPR == 0) {
                p.mean[at + r * P] = mean[r];
                p.rstd[at + r * P] = rstd[r];
            }
            if (p.z) store_shifted<T, LANES, NC>(static_cast<T*>(p.z) + (at + r * P) * p.ldz, col0, p.d, shift, v[r], own_slots, lane, group_mask<TPR>());
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (there[c]) {
                    f32x2_t w[4], b[4];
                    staged_params(params, shifted, chunk_of<TPR, NC>(c), w, b);
                    scale8(v[r][c], mean[r], rstd[r], w, b, v[r][c]);
                }
            store_shifted<T, LANES, NC>(static_cast<T*>(p.y) + (at + r * P) * p.ldy, col0, p.d, shift, v[r], own_slots, lane, group_mask<TPR>());
        }
    }
}

// Otherwise (rows off the alignment in different ways, or aligned ones whose parameters are not): by blocks that take
// every gridDim.x-th set of rows of one node, each chunk cut out of the pieces of memory it lies in.
template <class T, bool VEC, int TPR, int NC, int R>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, 512 / (TPR < 128 ? 128 : TPR)) norm_forward_odd_kernel(const NormForwardParams p)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, G = BLOCK / TPR, LANES = lanes_of(TPR);
    extern __shared__ float4 params[];   // weight, bias: two planes of `chunks` each
    __shared__ __align__(16) float part[2 * 32 * R];
    const int lane = threadIdx.x % LANES;
    const uint32_t node = blockIdx.y;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    stage_params<BLOCK>(p, node, 0, chunks, params);
    // all groups of a block go round equally often (barriers inside)
    for (uint32_t t0 = blockIdx.x * (G * R); t0 < p.rows; t0 += gridDim.x * (G * R)) {
        const uint32_t t = t0 + threadIdx.x / TPR * R;
        const int64_t row0 = (int64_t)node * p.rows + t;
        f32x2_t v[R][NC][4];
        load_mixed<T, false, VEC, TPR, NC, R>(p, node, t, v);
        float mean[R], rstd[R];
        row_statistics<false, !VEC, TPR, NC, R>(v, p.d, 0, p.eps, part, mean, rstd);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (t + r >= p.rows) continue;
            if (threadIdx.x % TPR == 0) {
                p.mean[row0 + r] = mean[r];
                p.rstd[row0 + r] = rstd[r];
            }
            T* y = static_cast<T*>(p.y) + (row0 + r) * p.ldy;
            T* z = static_cast<T*>(p.z) + (p.z ? (row0 + r) * p.ldz : 0);
            RowStore<T, VEC, LANES> to_y, to_z;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint32_t first = first_chunk_of<TPR, NC>(c), chunk = chunk_of<TPR, NC>(c);
                if (first >= chunks) break;
                const bool last = c + 1 == NC || first + LANES >= chunks;
                if (p.z) to_z.store(z, chunk * kChunk, p.d, v[r][c], lane, group_mask<TPR>(), last);
                f32x2_t out[4];
                if (chunk < chunks) {
                    f32x2_t w[4], b[4];
                    staged_params(params, chunks, chunk, w, b);
                    scale8(v[r][c], mean[r], rstd[r], w, b, out);
                }
                to_y.store(y, chunk * kChunk, p.d, out, lane, group_mask<TPR>(), last);
            }
        }
    }
}

// Rows of any width: one block per row, three passes over it (the second and third mostly from L2).
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) norm_forward_wide_kernel(const NormForwardParams p)
{
    __shared__ __align__(16) float part[2][32];
    const uint32_t row = blockIdx.x;
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const T* x = static_cast<const T*>(p.x) + (int64_t)row * p.ldx;
    const T* r = static_cast<const T*>(p.residual) + (p.residual ? (int64_t)row * p.ldr : 0);
    const int64_t all = (int64_t)p.nodes * p.rows;
    const Span sx = span_of<T>(p.x, p.ldx, all, p.d), sr = span_of<T>(p.residual, p.ldr, all, p.d);
    auto chunk_at = [&](uint32_t chunk, f32x2_t* v) {
        Raw8<T, VEC> rx, rr;
        rx.load(x, chunk * kChunk, p.d, sx);
        if (p.residual) rr.load(r, chunk * kChunk, p.d, sr);
        rx.get(v);
        drop8(p.mask, t * chunks + chunk, node, v);
        if (p.residual) {
            f32x2_t e[4];
            rr.get(e);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = add2(v[j], e[j]);
        }
    };
    f32x2_t v[4];
    float sum[1] = {0.f};
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_at(chunk, v);
        sum[0] += sum2(sum4(v));
    }
    group_sums<1024, 1>(sum, part[0]);
    const float mean = mean_of(sum[0], (float)p.d, 1.f / (float)p.d);
    float sq[1] = {0.f};
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_at(chunk, v);
        sq[0] += sum2(squares8<!VEC>(v, mean, (int)chunk * kChunk, p.d));
    }
    group_sums<1024, 1>(sq, part[1]);
    const float rstd = rsqrtf(sq[0] / (float)p.d + p.eps);   // within 2 ulp
    if (threadIdx.x == 0) {
        p.mean[row] = mean;
        p.rstd[row] = rstd;
    }
    T* y = static_cast<T*>(p.y) + (int64_t)row * p.ldy;
    T* z = static_cast<T*>(p.z) + (p.z ? (int64_t)row * p.ldz : 0);
    const int lane = threadIdx.x & 31;
    for (uint32_t first = threadIdx.x - lane; first < chunks; first += 1024) {
        const uint32_t chunk = first + lane;
        f32x2_t out[4];
        if (chunk < chunks) {
            f32x2_t w[4], b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = both(1.f), b[j] = both(0.f);
            if (p.weight) param8(p.weight + node * p.ldw, chunk * kChunk, p.d, p.wvec, w);
            if (p.bias) param8(p.bias + node * p.ldw, chunk * kChunk, p.d, p.wvec, b);
            chunk_at(chunk, v);
            scale8(v, mean, rstd, w, b, out);
        }
        RowStore<T, VEC, 32> to_y, to_z;
        if (p.z) to_z.store(z, chunk * kChunk, p.d, v, lane, 0xFFFFFFFFu, true);
        to_y.store(y, chunk * kChunk, p.d, out, lane, 0xFFFFFFFFu, true);
    }
}

// ---- layer norm, backward ---------------------------------------------------------------------------
// g = rstd (w dy - mean(h) - xh mean(h xh)) of one chunk, xh = (z - mean) rstd.
__device__ __forceinline__ void grad8(const f32x2_t* z, const f32x2_t* dy, const f32x2_t* w, float mean, float rstd, float mh, float mhx,
                                      f32x2_t* g)
{
    const f32x2_t m = both(mean), s = both(rstd), a = both(-mh), c = both(-mhx);
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = mul2(s, fma2(mul2(sub2(z[j], m), s), c, fma2(dy[j], w[j], a)));
}

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// 16 bytes from memory to shared memory without a register; a thread waits for its own copies.
__device__ __forceinline__ void copy16_async(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The block's column sums: its groups of threads one after the other, then out, to the node's gradients or to the block's
// row of partial sums.  `sums` (2 * TPR * NC * 8 floats) is used where the block has several groups.  col0(c): first
// column of the thread's chunk c.
template <int TPR, int NC, class Col0>
__device__ __forceinline__ void write_column_sums(const NormBackwardParams& p, uint32_t node, f32x2_t (*dw)[4], f32x2_t (*db)[4], float* sums,
                                                  Col0 col0)
{
    constexpr int G = block_of(TPR) / TPR;
    if (!p.dweight && !p.dbias) return;
    const int sub = threadIdx.x / TPR;
    if constexpr (G > 1) {
        constexpr int D = TPR * NC * 8;
        for (int g = 0; g < G; ++g) {
            __syncthreads();
            if (sub == g)
#pragma unroll
                for (int c = 0; c < NC; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        f32x2_t* at = reinterpret_cast<f32x2_t*>(sums) + chunk_of<TPR, NC>(c) * 4 + j;
                        if (g) dw[c][j] = add2(at[0], dw[c][j]), db[c][j] = add2(at[D / 2], db[c][j]);
                        at[0] = dw[c][j];
                        at[D / 2] = db[c][j];
                    }
        }
        if (sub != G - 1) return;   // the last group has added itself last and holds the sums
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
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int col = col0(c) + j;
            if (col >= 0 && col < p.d) {
                if (ow) ow[col] = (add ? ow[col] : 0.f) + element(dw[c], j);
                if (ob) ob[col] = (add ? ob[col] : 0.f) + element(db[c], j);
            }
        }
}

// Rows aligned, or (SHIFT) off the alignment all alike.  A block takes sets of rows of one node, R rows per group of TPR
// threads at a time, so that 2 R row sums share the shuffles and the barrier.  Each thread has the same NC chunks of
// columns in every row and so keeps the column sums (dw += dy xh, db += dy) in registers.  The rows' chunks come to a warp
// through its own places in shared memory, one set ahead, so that the loads in flight take no registers (four rows of
// three tensors in registers: 75 us for 8 x 4096 rows of 1024 bf16 columns instead of 63); the second pass reads them
// there again.  In fp32 a chunk is two 16-byte pieces; lanes copy neighbouring pieces, so that whole sectors come at once,
// and the pieces lie exchanged in every other group of eight, so that a warp reads its chunks without bank conflicts.
// Bound: issue slots (56 % busy at 16 warps per SM) beside HBM.  8 x 4096 rows of 1024 bf16, residual and dropout 63 us =
// 5.3 TB/s, without either 41 us; fp32 130 us = 5.2 TB/s; 2000 rows of 8192 fp32 58 us = 3.4 TB/s, bound by the chain of one
// row per SM; shifted rows of 1001 bf16 (4 x 8000) 132 us against 184 us when cut.
// kSets: sets of rows in shared memory, one worked on, the others on their way.
template <class T, bool SHIFT, int TPR, int NC, int R, int kSets, int kPerSM>
__global__ void __launch_bounds__(block_of(TPR), kPerSM) norm_backward_kernel(const NormBackwardParams p)
{
    constexpr int BLOCK = block_of(TPR), G = BLOCK / TPR, LANES = lanes_of(TPR), Q = sizeof(T) / 2;   // Q: 16-byte pieces of a chunk
    constexpr uint32_t P = SHIFT ? kShiftRows<T> : 1;
    constexpr int E = 16 / sizeof(T);   // columns of a piece
    extern __shared__ uint4 stage[];   // two sets of [tensor][r][c][warp][piece]
    __shared__ __align__(16) float part[2][BLOCK / 32 * 2 * R];
    __shared__ __align__(16) T slots[SHIFT ? BLOCK / LANES : 1][16];
    T* own_slots = slots[SHIFT ? threadIdx.x / LANES : 0];
    const int sub = G == 1 ? 0 : threadIdx.x / TPR, tensors = p.dz ? 3 : 2;
    const uint32_t node = blockIdx.y, chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const uint32_t first_row = SHIFT ? blockIdx.x % P : 0;   // the block's rows: first_row + P i
    const uint32_t rows = p.rows > first_row ? (p.rows - first_row + P - 1) / P : 0;
    const int64_t all = (int64_t)p.nodes * p.rows, row0 = (int64_t)node * p.rows + first_row;
    const int shift = SHIFT ? shift_of(static_cast<const T*>(p.z) + row0 * p.ldz) : 0;
    const Span sz = span_of<T>(p.z, p.ldz, all, p.d), sy = span_of<T>(p.dy, p.lddy, all, p.d), se = span_of<T>(p.dz, p.lddz, all, p.d);
    auto col = [&](int c) { return (int)chunk_of<TPR, NC>(c) * kChunk - shift; };
    auto mine = [&](int c) { return col(c) < p.d; };
    const int lane = threadIdx.x % LANES;
    auto place = [&](int buf, int tensor, int r, int c, int piece) {
        const int at = Q == 1 ? piece : piece ^ (piece >> 3 & 1);
        return stage + ((((buf * 3 + tensor) * R + r) * NC + c) * BLOCK + (threadIdx.x - lane)) * Q + at;
    };

    uint32_t there[NC];
    f32x2_t w[NC][4], dw[NC][4], db[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        there[c] = SHIFT ? columns_there(col(c), p.d) : 0xFFu;
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[c][j] = db[c][j] = both(0.f), w[c][j] = both(1.f);
        if (p.weight && mine(c)) {
            const float* pw = p.weight + node * p.ldw;
            if (!SHIFT && p.wvec) {
                param8(pw, col(c), p.d, true, w[c]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int a = col(c) + 2 * j, b = a + 1;
                    w[c][j] = pack2(a >= 0 && a < p.d ? pw[a] : 0.f, b >= 0 && b < p.d ? pw[b] : 0.f);
                }
            }
        }
    }
    // rows of the current set start here, the next set's `ahead` elements further on; strides between neighbouring rows
    const uint32_t step = gridDim.x / P * (G * R);
    uint32_t i0 = blockIdx.x / P * (G * R), i = i0 + sub * R;
    const int64_t at = row0 + (int64_t)i * P;
    const T *z = static_cast<const T*>(p.z) + at * p.ldz, *dy = static_cast<const T*>(p.dy) + at * p.lddy;
    const T* dz = static_cast<const T*>(p.dz) + at * p.lddz;
    T *dres = static_cast<T*>(p.dres) + at * p.lddres, *dx = static_cast<T*>(p.dx) + at * p.lddx;
    const float *means = p.mean + at, *rstds = p.rstd + at;
    const int64_t row_z = p.ldz * P, row_y = p.lddy * P, row_e = p.lddz * P, row_g = p.lddres * P, row_x = p.lddx * P;
    const bool all_columns = p.d == TPR * NC * kChunk;   // with no shift: every thread has all its chunks

    auto fetch_one = [&](const T* row, const Span& s, int tensor, int buf, int r, bool full) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int piece = q * LANES + lane, at = (int)first_chunk_of<TPR, NC>(c) * kChunk - shift + piece * E;
                if (!full && at >= p.d) continue;
                const T* from = row + at;
                uint4* to = place(buf, tensor, r, c, piece);
                if (!SHIFT || (at >= 0 && at + E <= p.d) || (reinterpret_cast<const char*>(from) >= s.lo && reinterpret_cast<const char*>(from + E) <= s.hi)) {
                    copy16_async(smem_u32(to), from);
                } else {   // the array's first or last row
#pragma unroll 1
                    for (int e = 0; e < E; ++e) reinterpret_cast<T*>(to)[e] = at + e >= 0 && at + e < p.d ? from[e] : from_f32<T>(0.f);
                }
            }
    };
    // the set whose first row is `set` rows behind the current pointers; n: rows that it has
    auto fetch_rows = [&](uint32_t set, int buf, uint32_t n, bool full) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (full || (uint32_t)r < n) {
                fetch_one(z + (int64_t)(set + r) * row_z, sz, 0, buf, r, full);
                fetch_one(dy + (int64_t)(set + r) * row_y, sy, 1, buf, r, full);
            }
        if (tensors == 3)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (full || (uint32_t)r < n) fetch_one(dz + (int64_t)(set + r) * row_e, se, 2, buf, r, full);
    };
    auto fetch = [&](uint32_t set, int buf) {
        const uint32_t from = i + set, n = from < rows ? min((uint32_t)R, rows - from) : 0;
        if (!SHIFT && all_columns && i0 + set + G * R <= rows) fetch_rows(set, buf, R, true);
        else fetch_rows(set, buf, n, false);
        copies_commit();
    };
    auto chunk_in = [&](int buf, int tensor, int r, int c, f32x2_t* v) {
        Raw8<T, true> raw;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const uint4 x = *place(buf, tensor, r, c, Q * lane + q);
            raw.w[4 * q] = x.x; raw.w[4 * q + 1] = x.y; raw.w[4 * q + 2] = x.z; raw.w[4 * q + 3] = x.w;
        }
        raw.get(v);
    };
    const float inv_d = 1.f / (float)p.d;
    float mean_next[R], rstd_next[R];   // of the next set
    auto fetch_statistics = [&](uint32_t set) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            mean_next[r] = rstd_next[r] = 0.f;
            if (i + set + r < rows) {
                mean_next[r] = means[(int64_t)(set + r) * P];
                rstd_next[r] = rstds[(int64_t)(set + r) * P];
            }
        }
    };
    // one set; full: all its rows and chunks are there
    auto work = [&](int buf, int odd, const float* mean, const float* rstd, auto full_) {
        constexpr bool FULL = decltype(full_)::value;
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f32x2_t s1 = both(0.f), s2 = both(0.f);
            if (FULL || i + r < rows) {
                const f32x2_t m = both(mean[r]), q = both(rstd[r]);
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (!FULL && !mine(c)) continue;
                    f32x2_t vz[4], vy[4];
                    chunk_in(buf, 0, r, c, vz);
                    chunk_in(buf, 1, r, c, vy);
                    if (SHIFT) {   // what lies beside the row; the second pass does not store it
                        keep_columns(vz, there[c]);
                        keep_columns(vy, there[c]);
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // columns that are not there have dy = 0 and so add nothing
                        const f32x2_t xh = mul2(sub2(vz[j], m), q), h = mul2(vy[j], w[c][j]);
                        db[c][j] = add2(db[c][j], vy[j]);
                        dw[c][j] = fma2(vy[j], xh, dw[c][j]);
                        s1 = add2(s1, h);
                        s2 = fma2(h, xh, s2);
                    }
                }
            }
            s[2 * r] = sum2(s1);
            s[2 * r + 1] = sum2(s2);
        }
        group_sums<TPR, 2 * R>(s, part[odd]);
        asm volatile("" ::: "memory");   // the chunks are read again, not kept
        uint4 edge = make_uint4(0, 0, 0, 0);   // SHIFT: lane r has the words before the warp's first chunk in row r
        if (SHIFT && p.dx && p.mask.on) {
            const uint32_t t = first_row + (i + (lane < R ? lane : 0)) * P;
            edge = drop_words(p.mask, t * chunks + first_chunk_of<TPR, NC>(0) - 1, node);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!FULL && i + r >= rows) continue;
            f32x2_t g[NC][4];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (!FULL && !mine(c)) continue;
                f32x2_t vz[4], vy[4];
                chunk_in(buf, 0, r, c, vz);
                chunk_in(buf, 1, r, c, vy);
                grad8(vz, vy, w[c], mean[r], rstd[r], s[2 * r] * inv_d, s[2 * r + 1] * inv_d, g[c]);
            }
            if (tensors == 3)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (!FULL && !mine(c)) continue;
                    f32x2_t e[4];
                    chunk_in(buf, 2, r, c, e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[c][j] = add2(g[c][j], e[j]);
                }
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (!SHIFT && (FULL || mine(c))) store8<T>(dres + r * row_g + col(c), g[c]);
            if (SHIFT) store_shifted<T, LANES, NC>(dres + r * row_g, col(0), p.d, shift, g, own_slots, lane, group_mask<TPR>());
            if (!p.dx) continue;
            const uint32_t groups = (first_row + (i + r) * P) * chunks;
            uint4 before = SHIFT ? shfl4(group_mask<TPR>(), edge, r, LANES) : edge;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const uint32_t group = groups + chunk_of<TPR, NC>(c);
                if constexpr (SHIFT) {
                    if (!p.mask.on) continue;   // a probability that rounds to zero
                    const uint4 own = drop_words(p.mask, group, node);
                    const uint4 left = shfl4(group_mask<TPR>(), own, (lane + LANES - 1) % LANES, LANES);
                    uint32_t word[4];
                    shifted_words(lane ? left : before, own, shift, word);
                    before = left;   // lane 0 has the last lane's
                    drop8_by(p.mask, word, g[c]);
                } else {
                    if (!FULL && !mine(c)) continue;
                    drop8(p.mask, group, node, g[c]);
                    store8<T>(dx + r * row_x + col(c), g[c]);
                }
            }
            if (SHIFT) store_shifted<T, LANES, NC>(dx + r * row_x, col(0), p.d, shift, g, own_slots, lane, group_mask<TPR>());
        }
    };
#pragma unroll
    for (int k = 0; k < kSets - 1; ++k) fetch(k * step, k);
    fetch_statistics(0);
    for (int buf = 0, odd = 0; i0 < rows; buf = buf + 1 == kSets ? 0 : buf + 1, odd ^= 1) {
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) mean[r] = mean_next[r], rstd[r] = rstd_next[r];
        if (Q > 1 || SHIFT) __syncwarp(group_mask<TPR>());   // the other lanes have read what these copies replace
        fetch((kSets - 1) * step, buf ? buf - 1 : kSets - 1);
        fetch_statistics(step);
        copies_wait<kSets - 1>();
        if (Q > 1 || SHIFT) __syncwarp(group_mask<TPR>());   // and their copies of this set are there
        if (!SHIFT && all_columns && i0 + G * R <= rows) work(buf, odd, mean, rstd, Yes());
        else work(buf, odd, mean, rstd, No());
        i0 += step, i += step;
        z += step * row_z, dy += step * row_y, dz += step * row_e, dres += step * row_g, dx += step * row_x;
        means += (int64_t)step * P, rstds += (int64_t)step * P;
    }
    copies_wait<0>();
    __syncthreads();
    write_column_sums<TPR, NC>(p, node, dw, db, reinterpret_cast<float*>(stage), col);
}

// Rows that are off the alignment in different ways: each chunk is cut out of the pieces of memory it lies in.
template <class T, int TPR, int NC>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_backward_odd_kernel(const NormBackwardParams p)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, G = BLOCK / TPR, LANES = lanes_of(TPR);
    __shared__ __align__(16) float part[2][BLOCK / 32 * 2];
    __shared__ float sums[G > 1 ? 2 * TPR * NC * 8 : 1];
    const uint32_t node = blockIdx.y, chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const int64_t all = (int64_t)p.nodes * p.rows;
    const Span sz = span_of<T>(p.z, p.ldz, all, p.d), sy = span_of<T>(p.dy, p.lddy, all, p.d), se = span_of<T>(p.dz, p.lddz, all, p.d);
    auto col = [&](int c) { return (int)chunk_of<TPR, NC>(c) * kChunk; };
    f32x2_t w[NC][4], dw[NC][4], db[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
        for (int j = 0; j < 4; ++j) dw[c][j] = db[c][j] = both(0.f), w[c][j] = both(1.f);
        if (p.weight) param8(p.weight + node * p.ldw, col(c), p.d, false, w[c]);
    }
    const float inv_d = 1.f / (float)p.d;
    int buf = 0;
    for (uint32_t t0 = blockIdx.x * G; t0 < p.rows; t0 += gridDim.x * G, buf ^= 1) {
        const uint32_t t = t0 + threadIdx.x / TPR;
        const bool live = t < p.rows;
        const int64_t row = (int64_t)node * p.rows + t;
        Raw8<T, false> rz[NC], ry[NC];
        f32x2_t s1 = both(0.f), s2 = both(0.f);
        float mean = 0.f, rstd = 0.f;
        if (live) {
            mean = p.mean[row], rstd = p.rstd[row];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                rz[c].load(static_cast<const T*>(p.z) + row * p.ldz, col(c), p.d, sz);
                ry[c].load(static_cast<const T*>(p.dy) + row * p.lddy, col(c), p.d, sy);
            }
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                f32x2_t z[4], dy[4];
                rz[c].get(z);
                ry[c].get(dy);
                if (col(c) >= p.d) continue;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2_t xh = mul2(sub2(z[j], both(mean)), both(rstd)), h = mul2(dy[j], w[c][j]);
                    db[c][j] = add2(db[c][j], dy[j]);
                    dw[c][j] = fma2(dy[j], xh, dw[c][j]);
                    s1 = add2(s1, h);
                    s2 = fma2(h, xh, s2);
                }
            }
        }
        float s[2] = {sum2(s1), sum2(s2)};
        group_sums<TPR, 2>(s, part[buf]);
        if (!live) continue;
        T* dres = static_cast<T*>(p.dres) + row * p.lddres;
        T* dx = static_cast<T*>(p.dx) + (p.dx ? row * p.lddx : 0);
        RowStore<T, false, LANES> to_res, to_x;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const uint32_t first = first_chunk_of<TPR, NC>(c);
            if (first >= chunks) break;
            const bool last = c + 1 == NC || first + LANES >= chunks;
            f32x2_t z[4], dy[4], g[4];
            rz[c].unpack_again();
            ry[c].unpack_again();
            rz[c].get(z);
            ry[c].get(dy);
            grad8(z, dy, w[c], mean, rstd, s[0] * inv_d, s[1] * inv_d, g);
            if (p.dz) {
                Raw8<T, false> re;
                f32x2_t e[4];
                re.load(static_cast<const T*>(p.dz) + row * p.lddz, col(c), p.d, se);
                re.get(e);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = add2(g[j], e[j]);
            }
            to_res.store(dres, col(c), p.d, g, threadIdx.x % LANES, group_mask<TPR>(), last);
            if (p.dx) {
                drop8(p.mask, t * chunks + chunk_of<TPR, NC>(c), node, g);
                to_x.store(dx, col(c), p.d, g, threadIdx.x % LANES, group_mask<TPR>(), last);
            }
        }
    }
    write_column_sums<TPR, NC>(p, node, dw, db, sums, col);
}

// Rows of any width: the gradient of z, one block per row, two passes over it.
template <class T, bool VEC>
__global__ void __launch_bounds__(1024) norm_backward_wide_kernel(const NormBackwardParams p)
{
    __shared__ float part[32 * 2];
    const uint32_t row = blockIdx.x;
    const uint32_t node = row / p.rows, t = row - node * p.rows;
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const float mean = p.mean[row], rstd = p.rstd[row];
    const int64_t all = (int64_t)p.nodes * p.rows;
    const Span sz = span_of<T>(p.z, p.ldz, all, p.d), sy = span_of<T>(p.dy, p.lddy, all, p.d), se = span_of<T>(p.dz, p.lddz, all, p.d);
    auto chunk_at = [&](uint32_t chunk, f32x2_t* z, f32x2_t* dy, f32x2_t* w) {
        Raw8<T, VEC> rz, rdy;
        rz.load(static_cast<const T*>(p.z) + (int64_t)row * p.ldz, chunk * kChunk, p.d, sz);
        rdy.load(static_cast<const T*>(p.dy) + (int64_t)row * p.lddy, chunk * kChunk, p.d, sy);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = both(1.f);
        if (p.weight) param8(p.weight + node * p.ldw, chunk * kChunk, p.d, p.wvec, w);
        rz.get(z);
        rdy.get(dy);
    };
    f32x2_t z[4], dy[4], w[4];
    f32x2_t s1 = both(0.f), s2 = both(0.f);
    for (uint32_t chunk = threadIdx.x; chunk < chunks; chunk += 1024) {
        chunk_at(chunk, z, dy, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x2_t h = mul2(dy[j], w[j]);
            s1 = add2(s1, h);
            s2 = fma2(h, mul2(sub2(z[j], both(mean)), both(rstd)), s2);
        }
    }
    float s[2] = {sum2(s1), sum2(s2)};
    group_sums<1024, 2>(s, part);
    T* dres = static_cast<T*>(p.dres) + (int64_t)row * p.lddres;
    T* dx = static_cast<T*>(p.dx) + (p.dx ? (int64_t)row * p.lddx : 0);
    const int lane = threadIdx.x & 31;
    for (uint32_t first = threadIdx.x - lane; first < chunks; first += 1024) {
        const uint32_t chunk = first + lane;
        f32x2_t g[4];
        if (chunk < chunks) {
            chunk_at(chunk, z, dy, w);
            grad8(z, dy, w, mean, rstd, s[0] / (float)p.d, s[1] / (float)p.d, g);
            if (p.dz) {
                Raw8<T, VEC> re;
                f32x2_t e[4];
                re.load(static_cast<const T*>(p.dz) + (int64_t)row * p.lddz, chunk * kChunk, p.d, se);
                re.get(e);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] = add2(g[j], e[j]);
            }
        }
        RowStore<T, VEC, 32> to_res, to_x;
        to_res.store(dres, chunk * kChunk, p.d, g, lane, 0xFFFFFFFFu, true);
        if (p.dx) {
            if (chunk < chunks) drop8(p.mask, t * chunks + chunk, node, g);
            to_x.store(dx, chunk * kChunk, p.d, g, lane, 0xFFFFFFFFu, true);
        }
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
    const int64_t all = (int64_t)p.nodes * p.rows;
    const Span sz = span_of<T>(p.z, p.ldz, all, p.d), sy = span_of<T>(p.dy, p.lddy, all, p.d);
    f32x2_t dw[4], db[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) dw[j] = db[j] = both(0.f);
    for (uint32_t t = blockIdx.y; t < p.rows; t += gridDim.y) {
        const int64_t row = (int64_t)node * p.rows + t;
        Raw8<T, VEC> rz, rdy;
        f32x2_t z[4], dy[4];
        rz.load(static_cast<const T*>(p.z) + row * p.ldz, col, p.d, sz);
        rdy.load(static_cast<const T*>(p.dy) + row * p.lddy, col, p.d, sy);
        const f32x2_t m = both(p.mean[row]), q = both(p.rstd[row]);
        rz.get(z);
        rdy.get(dy);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            dw[j] = fma2(dy[j], mul2(sub2(z[j], m), q), dw[j]);
            db[j] = add2(db[j], dy[j]);
        }
    }
    const bool add = p.splits == 1 && p.accumulate;
    float* ow = p.splits > 1 ? p.partial + ((int64_t)node * p.splits + blockIdx.y) * 2 * p.d
                             : p.dweight ? p.dweight + node * p.lddw : nullptr;
    float* ob = p.splits > 1 ? ow + p.d : p.dbias ? p.dbias + node * p.lddw : nullptr;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (col + j < p.d) {
            if (ow) ow[col + j] = (add ? ow[col + j] : 0.f) + element(dw, j);
            if (ob) ob[col + j] = (add ? ob[col + j] : 0.f) + element(db, j);
        }
}

// 3 us for 576 blocks' sums of 1024 columns, its launch hidden behind the kernel before it.
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
constexpr int kForwardWide = 16384, kForwardOddWide = 8192, kBackwardWide = 8192;   // widest rows that stay in registers

// Blocks of a kernel that an SM holds, from its registers (looked up once) and shared memory.
template <class Kernel>
int blocks_per_sm(Kernel kernel, int block, size_t smem, int& regs)
{
    if (!regs) {
        cudaFuncAttributes at;
        regs = cudaFuncGetAttributes(&at, kernel) == cudaSuccess && at.numRegs > 0 ? at.numRegs : 128;
    }
    int n = 65536 / ((regs + 7) / 8 * 8 * block);
    if (n > 2048 / block) n = 2048 / block;
    const int by_smem = (int)(227 * 1024 / (smem + 2048));
    if (n > by_smem) n = by_smem;
    return n < 1 ? 1 : n;
}

template <class T, bool VEC, int TPR, int NC>
cudaError_t dropout_rows(DropoutParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((p.chunks.d + NC * TPR - 1) / (NC * TPR));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    dropout_rows_kernel<T, VEC, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC>
cudaError_t dropout_shifted(DropoutParams& p, cudaStream_t s)
{
    p.stretches = make_divisor((p.d + kShiftRows<T> - 1 + NC * TPR * kChunk - 1) / (NC * TPR * kChunk));
    const uint64_t groups = (uint64_t)p.rows * p.stretches.d;
    dropout_shifted_kernel<T, TPR, NC><<<dim3((unsigned)((groups + 256 / TPR - 1) / (256 / TPR)), p.nodes), 256, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t dropout_of(DropoutParams p, cudaStream_t s)
{
    const uint32_t chunks = (uint32_t)(p.d + kChunk - 1) / kChunk;
    const uint64_t total = (uint64_t)p.rows * chunks;   // per node, below 2^32
    p.chunks = make_divisor(chunks);
    if constexpr (VEC) {
        if (p.ldx == p.d && p.ldy == p.d && total < (uint64_t(1) << 32) - 1024) {
            // four chunks per thread where that still fills the SMs with blocks
            if (p.nodes * total < 148 * 8 * 1024) dropout_dense_kernel<T, 1><<<dim3((unsigned)((total + 255) / 256), p.nodes), 256, 0, s>>>(p);
            else dropout_dense_kernel<T, 4><<<dim3((unsigned)((total + 1023) / 1024), p.nodes), 256, 0, s>>>(p);
            return cudaGetLastError();
        }
    }
    if (!VEC && p.shifted) {
        const int d = p.d + (int)kShiftRows<T> - 1;
        return d <= 64    ? dropout_shifted<T, 8, 1>(p, s)
               : d <= 256 ? dropout_shifted<T, 32, 1>(p, s)
               : d <= 512 ? dropout_shifted<T, 32, 2>(p, s)
                          : dropout_shifted<T, 32, 4>(p, s);
    }
    return chunks <= 8    ? dropout_rows<T, VEC, 8, 1>(p, s)
           : chunks <= 32 ? dropout_rows<T, VEC, 32, 1>(p, s)
           : chunks <= 64 ? dropout_rows<T, VEC, 32, 2>(p, s)
                          : dropout_rows<T, VEC, 32, 4>(p, s);
}

template <class T, bool VEC, int TPR, int NC, int R>
cudaError_t forward_odd(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, SET = BLOCK / TPR * R;
    const size_t smem = (size_t)((p.d + kChunk - 1) / kChunk) * 64;
    const auto kernel = norm_forward_odd_kernel<T, VEC, TPR, NC, R>;
    if (smem > 47 * 1024) {
        static unsigned long long limit_set = 0;
        const cudaError_t e = ensure_smem_limit(kernel, kForwardOddWide * 8, limit_set);
        if (e != cudaSuccess) return e;
    }
    static int regs = 0;
    const uint32_t sets = (p.rows + SET - 1) / SET;
    const uint32_t room = (uint32_t)(kSMs * blocks_per_sm(kernel, BLOCK, smem, regs)) / p.nodes;
    kernel<<<dim3(sets < room ? sets : room ? room : 1, p.nodes), BLOCK, smem, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC, int R>
cudaError_t forward_shifted(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, SET = BLOCK / TPR * R;
    constexpr uint32_t P = kShiftRows<T>;
    const size_t smem = (size_t)((p.d + P + kChunk - 1) / kChunk) * 64;
    const auto kernel = norm_forward_shifted_kernel<T, TPR, NC, R>;
    if (smem > 47 * 1024) {
        static unsigned long long limit_set = 0;
        const cudaError_t e = ensure_smem_limit(kernel, (kForwardOddWide + 16) * 8, limit_set);
        if (e != cudaSuccess) return e;
    }
    static int regs = 0;
    // as many blocks as fit, in whole classes of rows
    const uint32_t sets = ((p.rows + P - 1) / P + SET - 1) / SET;
    const uint32_t room = (uint32_t)(kSMs * blocks_per_sm(kernel, BLOCK, smem, regs)) / (p.nodes * P);
    kernel<<<dim3(P * (sets < room ? sets : room ? room : 1), p.nodes), BLOCK, smem, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC, int R>
cudaError_t forward_as(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, SET = BLOCK / TPR * R;
    norm_forward_kernel<T, TPR, NC, R><<<dim3((p.rows + SET - 1) / SET, p.nodes), BLOCK, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool VEC>
cudaError_t forward_of(const NormForwardParams& p, cudaStream_t s)
{
    if constexpr (VEC)
        if (p.weight && p.bias && p.wvec) {
            if (p.d <= 64) return forward_as<T, 8, 1, 4>(p, s);
            if (p.d <= 128) return forward_as<T, 16, 1, 4>(p, s);
            if (p.d <= 256) return forward_as<T, 32, 1, 4>(p, s);
            if (p.d <= 512) return forward_as<T, 32, 2, 2>(p, s);
            if (p.d <= 1024) return forward_as<T, 32, 4, 1>(p, s);
            if (p.d <= 2048) return forward_as<T, 128, 2, 2>(p, s);
            if (p.d <= 4096) return forward_as<T, 128, 4, 1>(p, s);
            if (p.d <= 8192) return forward_as<T, 512, 2, 1>(p, s);
            if (p.d <= kForwardWide) return forward_as<T, 512, 4, 1>(p, s);
        }
    if constexpr (!VEC)
        if (p.shifted) {
            const int d = p.d + (int)kShiftRows<T> - 1;
            if (d <= 64) return forward_shifted<T, 8, 1, 2>(p, s);
            if (d <= 128) return forward_shifted<T, 16, 1, 2>(p, s);
            if (d <= 256) return forward_shifted<T, 32, 1, 2>(p, s);
            if (d <= 512) return forward_shifted<T, 32, 2, 1>(p, s);
            if (d <= 1024) return forward_shifted<T, 64, 2, 1>(p, s);
            if (d <= 1536) return forward_shifted<T, 64, 3, 1>(p, s);
            if (d <= 2048) return forward_shifted<T, 128, 2, 1>(p, s);
            if (d <= 4096) return forward_shifted<T, 256, 2, 1>(p, s);
            if (d <= kForwardOddWide) return forward_shifted<T, 512, 2, 1>(p, s);
        }
    if (p.d <= 64) return forward_odd<T, VEC, 8, 1, 2>(p, s);
    if (p.d <= 256) return forward_odd<T, VEC, 32, 1, 2>(p, s);
    if (p.d <= 512) return forward_odd<T, VEC, 32, 2, 1>(p, s);
    if (p.d <= 1024) return forward_odd<T, VEC, 64, 2, 1>(p, s);
    if (p.d <= 2048) return forward_odd<T, VEC, 128, 2, 1>(p, s);
    if (p.d <= 4096) return forward_odd<T, VEC, 256, 2, 1>(p, s);
    if (p.d <= kForwardOddWide) return forward_odd<T, VEC, 512, 2, 1>(p, s);
    norm_forward_wide_kernel<T, VEC><<<p.nodes * p.rows, 1024, 0, s>>>(p);
    return cudaGetLastError();
}

template <class T, bool SHIFT, int TPR, int NC, int R, int kSets, int kPerSM>
cudaError_t backward_as(const NormBackwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = block_of(TPR), G = BLOCK / TPR;
    constexpr size_t kStage = (size_t)kSets * 3 * R * NC * 8 * sizeof(T) * BLOCK, kSums = G > 1 ? (size_t)2 * TPR * NC * 8 * 4 : 0;
    constexpr size_t smem = kStage > kSums ? kStage : kSums;
    const auto kernel = norm_backward_kernel<T, SHIFT, TPR, NC, R, kSets, kPerSM>;
    static unsigned long long limit_set = 0;
    const cudaError_t e = ensure_smem_limit(kernel, (int)smem, limit_set);
    if (e != cudaSuccess) return e;
    kernel<<<dim3(p.splits, p.nodes), BLOCK, smem, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC>
cudaError_t backward_odd(const NormBackwardParams& p, cudaStream_t s)
{
    norm_backward_odd_kernel<T, TPR, NC><<<dim3(p.splits, p.nodes), TPR < 128 ? 128 : TPR, 0, s>>>(p);
    return cudaGetLastError();
}

// Where a row's columns and its shift fit a group's chunks: the kernels above; rows of up to kBackwardWide columns.
template <class T, bool SHIFT>
cudaError_t backward_by_width(const NormBackwardParams& p, cudaStream_t s)
{
    // Rows at a time and sets of them in shared memory, 36 or 48 KB for 128 threads.  Four bf16 rows and two sets against
    // two rows and three sets: 64 and 70 us for 8 x 4096 rows of 1024 columns, 62 and 65 us for 4 x 16000 rows of 512, but
    // 44 and 37 us for 4 x 60000 rows of 64.
    constexpr int R = sizeof(T) == 4 ? 2 : 4;
    const int d = p.d + (SHIFT ? (int)kShiftRows<T> - 1 : 0);
    if (d <= 64) return backward_as<T, SHIFT, 8, 1, R / 2, 3, 5>(p, s);
    if (d <= 128) return backward_as<T, SHIFT, 16, 1, R / 2, 3, 5>(p, s);
    if (d <= 256) return backward_as<T, SHIFT, 32, 1, R / 2, 3, 5>(p, s);
    if (d <= 512) return backward_as<T, SHIFT, 64, 1, R, 2, 4>(p, s);
    if (d <= 768) return backward_as<T, SHIFT, 96, 1, R, 2, 5>(p, s);
    if (d <= 1024) return backward_as<T, SHIFT, 128, 1, R, 2, 4>(p, s);
    if (d <= 1280) return backward_as<T, SHIFT, 160, 1, R, 2, 3>(p, s);
    if (d <= 1536) return backward_as<T, SHIFT, 192, 1, R, 2, SHIFT ? 2 : 3>(p, s);
    if (d <= 2048) return backward_as<T, SHIFT, 256, 1, R, 2, 2>(p, s);
    if (d <= 2560) return backward_as<T, SHIFT, 320, 1, R / 2, 3, SHIFT ? 1 : 2>(p, s);
    if (d <= 4096) return backward_as<T, SHIFT, 512, 1, R, 2, 1>(p, s);
    // (a shifted row's kernel does not fit the 64 registers of 1024 threads)
    if constexpr (SHIFT) return backward_as<T, SHIFT, 512, 2, 1, 2, 1>(p, s);
    else return backward_as<T, SHIFT, 1024, 1, R / 2, 2, 1>(p, s);
}

template <class T, bool VEC>
cudaError_t backward_of(const NormBackwardParams& p, cudaStream_t s)
{
    const bool shifted = !VEC && p.shifted && p.splits % (int)kShiftRows<T> == 0;
    if (p.d + (shifted ? (int)kShiftRows<T> - 1 : 0) <= kBackwardWide) {
        if constexpr (VEC) return backward_by_width<T, false>(p, s);
        else {
            if (shifted) return backward_by_width<T, true>(p, s);
            if (p.d <= 64) return backward_odd<T, 8, 1>(p, s);
            if (p.d <= 256) return backward_odd<T, 32, 1>(p, s);
            if (p.d <= 512) return backward_odd<T, 64, 1>(p, s);
            if (p.d <= 1024) return backward_odd<T, 128, 1>(p, s);
            if (p.d <= 2048) return backward_odd<T, 256, 1>(p, s);
            if (p.d <= 4096) return backward_odd<T, 512, 1>(p, s);
            return backward_odd<T, 512, 2>(p, s);
        }
    }
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
    if (!p.rows) return cudaSuccess;
#define GPGA_CALL(T, V) dropout_of<T, V>(p, s)
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
    // Blocks that an SM holds (four or five of 128 threads by their shared memory), and no more than sets of four rows per
    // group; a multiple of eight where there are as many, since blocks of shifted rows take every eighth row (a fourth in fp32).
    const int64_t set = 4 * (d <= 64 ? 16 : d <= 128 ? 8 : d <= 256 ? 4 : d <= 512 ? 2 : 1);
    const int64_t per_sm = d <= 256 ? 5 : d <= 512 ? 4 : d <= 768 ? 5 : d <= 1024 ? 4 : d <= 1536 ? 3 : d <= 2560 ? 2 : 1;
    int64_t splits = (kSMs * per_sm) / nodes;
    const int64_t groups = (rows + set - 1) / set;
    if (splits > groups) splits = groups;
    if (groups <= 2) splits = 1;   // one launch: 8 rows of 1024 one set after the other 4.8 us, 32 rows in two launches 5.3 us
    if (splits >= 8) splits = splits / 8 * 8;
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
    return launch_after_trigger(norm_params_kernel, dim3((unsigned)((2 * (int64_t)p.d + 31) / 32), p.nodes), dim3(256), 0, s, true, p);
}

}  // namespace gpga
