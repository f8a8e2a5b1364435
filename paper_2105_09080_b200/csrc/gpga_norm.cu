// Layer norm of residual + dropout(x).
#include "gpga_norm_device.cuh"

namespace gpga {

namespace {

// (z - mean) rstd w + b
__device__ __forceinline__ void scale8(const f32x2_t* v, float mean, float rstd, const f32x2_t* w, const f32x2_t* b, f32x2_t* y)
{
    const f32x2_t m = both(mean), s = both(rstd);
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = fma2(mul2(sub2(v[j], m), s), w[j], b[j]);
}

__device__ __forceinline__ f32x2_t sum4(const f32x2_t* v) { return add2(add2(v[0], v[1]), add2(v[2], v[3])); }

// Sum of (v - mean)^2 over the columns of a chunk that lie in the row (a bit each); EDGE: some may not.
template <bool EDGE>
__device__ __forceinline__ f32x2_t squares8(const f32x2_t* v, float mean, uint32_t there)
{
    const f32x2_t m = both(mean);
    f32x2_t e[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = sub2(v[j], m);
    if (EDGE) keep_columns(e, there);
    f32x2_t s = mul2(e[0], e[0]);
#pragma unroll
    for (int j = 1; j < 4; ++j) s = fma2(e[j], e[j], s);
    return s;
}

// s / n for a row's mean: one multiplication by fl(1 / n), corrected by the exact remainder: as good as a division, which
// takes several times the instructions.  (A constant row's mean is exact where the sum s is, otherwise off by the sum's rounding:
// of 200 random constants 69 at 1000 columns, none at 1024 or 4096.)
__device__ __forceinline__ float mean_of(float s, float n, float inv_n)
{
    const float m = s * inv_n;
    const float fixed = fmaf(fmaf(-m, n, s), inv_n, m);
    return fabsf(fixed) <= 3.4e38f ? fixed : m;   // an infinite sum has no remainder
}

// Statistics of R rows that a group of TPR threads holds in registers (columns and rows that are not there: zero).  The
// variance is a second pass over the registers, so that nothing cancels.  FULL: every chunk is there; EDGE: chunks may be
// partial.  there(c): the columns of chunk c that lie in the row, a bit each.
template <bool FULL, bool EDGE, int TPR, int NC, int R, class There>
__device__ __forceinline__ void row_statistics(const f32x2_t (*v)[NC][4], const There& there, int d, float eps, float* part, float* mean, float* rstd)
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
        for (int c = 0; c < NC; ++c)
            if (FULL || there(c)) sum = add2(sum, squares8<EDGE>(v[r][c], mean[r], there(c)));
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
    row_statistics<FULL, false, TPR, NC, R>(v, [&](int c) { return chunk_of<TPR, NC>(c) < chunks; }, p.d, p.eps, part, mean, rstd);
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
// that have one shift, and lays out the node's parameters for it once.  The next set is on its way, to shared memory (STAGED)
// or to registers.  Bound: issue slots (55 %) and latency at 16 to 20 warps per SM.  2 x 5001 rows of 1023 f16 19 us (cut
// chunks 27 us, single elements 39 us), 4 x 8000 rows of 1001 bf16 with residual and dropout 69 us (121, 175), fp32 without
// dropout 94 us (130, 227).  The generator call before a warp's first chunk is made for a row per lane at a time (a call
// for each row, of which one lane's words are used: 85 us instead of 75, at two chunks per lane).
template <class T, int TPR, int NC, int R, bool STAGED>
__global__ void __launch_bounds__(block_of(TPR), (STAGED && NC < 4 ? 640 : 512) / block_of(TPR)) norm_forward_shifted_kernel(const NormForwardParams p)
{
    constexpr int BLOCK = block_of(TPR), G = BLOCK / TPR, LANES = lanes_of(TPR);
    constexpr uint32_t P = kShiftRows<T>;
    extern __shared__ float4 params[];
    __shared__ __align__(16) float part[2 * 32 * R];
    __shared__ __align__(128) T slots[BLOCK / LANES][2][16];
    const uint32_t node = blockIdx.y, chunks = (uint32_t)(p.d + kChunk - 1) / kChunk, first_row = blockIdx.x % P;
    const uint32_t rows = p.rows > first_row ? (p.rows - first_row + P - 1) / P : 0;   // first_row + P i
    const int64_t all = (int64_t)p.nodes * p.rows, row0 = (int64_t)node * p.rows + first_row;
    const int shift = shift_of(static_cast<const T*>(p.x) + row0 * p.ldx), lane = threadIdx.x % LANES;
    const uint32_t shifted = (uint32_t)(p.d + shift + kChunk - 1) / kChunk;   // chunks of a row
    const Span sx = span_of<T>(p.x, p.ldx, all, p.d), sr = span_of<T>(p.residual, p.ldr, all, p.d);
    const int col0 = (int)chunk_of<TPR, NC>(0) * kChunk - shift;
    auto col = [&](int c) { return col0 + c * LANES * kChunk; };
    __shared__ uint4 edges[BLOCK];
    const Staged<T, true, TPR, NC, R> staged{reinterpret_cast<uint4*>(params + 4 * shifted), p.d, shift, lane};
    uint4* own_edges = edges + threadIdx.x / LANES * LANES;
    ShiftedStore<T, LANES, NC> to(col0, p.d, shift, slots[threadIdx.x / LANES][0], lane);
    uint32_t there[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) there[c] = columns_there(col(c), p.d);
    stage_params<BLOCK>(p, node, shift, shifted, params);
    const uint32_t step = gridDim.x / P * (G * R);
    uint32_t i0 = blockIdx.x / P * (G * R), i = i0 + (G == 1 ? 0 : threadIdx.x / TPR * R);
    __shared__ __align__(16) T load_slots[STAGED ? 1 : BLOCK / LANES][16];
    Raw8<T, true> rx[STAGED ? 1 : R][NC], rr[STAGED ? 1 : R][NC];
    auto fetch_row = [&](const T* row, const Span& s, int place, int r, Raw8<T, true>* raw) {
        if constexpr (STAGED) {
            staged.fetch(row, s, place, r, false);
        } else {
            const bool in = inside(row, p.d, s);
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (there[c]) load_shifted(row, col(c), in || there[c] == 0xFFu, p.d, raw[c], load_slots[threadIdx.x / LANES]);
        }
    };
    auto fetch = [&](uint32_t from, int buf) {   // rows first_row + P from, ...
        const int64_t at = row0 + (int64_t)from * P;
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (from + r < rows) {
                const int q = STAGED ? 0 : r;
                fetch_row(static_cast<const T*>(p.x) + (at + r * P) * p.ldx, sx, 2 * buf, r, rx[q]);
                if (p.residual) fetch_row(static_cast<const T*>(p.residual) + (at + r * P) * p.ldr, sr, 2 * buf + 1, r, rr[q]);
            }
        if (STAGED) copies_commit();
    };
    fetch(i, 0);
    for (uint32_t set = 0; i0 < rows; ++set, i0 += step, i += step) {
        const int64_t at = row0 + (int64_t)i * P;   // pointers from here: fewer registers than ones that are carried along
        const int buf = set & 1;
        if constexpr (STAGED) {
            __syncwarp(group_mask<TPR>());   // the other lanes have read what these copies replace
            fetch(i + step, buf ^ 1);
            copies_wait<1>();
            __syncwarp(group_mask<TPR>());   // the other lanes' copies of this set are there
        }
        f32x2_t v[R][NC][4];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if constexpr (STAGED) staged.chunk(2 * buf, r, c, v[r][c]);
                else rx[r][c].get(v[r][c]);
        if (p.mask.on) {
            if (set % (LANES / R) == 0) {   // lane l works out the words before the warp's first chunk, in row l % R of set l / R from here
                __syncwarp(group_mask<TPR>());
                own_edges[lane] = drop_words(p.mask, (first_row + (i + lane / R * step + lane % R) * P) * chunks + first_chunk_of<TPR, NC>(0) - 1, node);
                __syncwarp(group_mask<TPR>());
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint4 before = own_edges[set % (LANES / R) * R + r];
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
                    if constexpr (STAGED) staged.chunk(2 * buf + 1, r, c, e);
                    else rr[r][c].get(e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][c][j] = add2(v[r][c][j], e[j]);
                }
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < NC; ++c) keep_columns(v[r][c], i + r < rows ? there[c] : 0u);   // the rest was never loaded, or lies beside the row
        float mean[R], rstd[R];
        if constexpr (!STAGED) fetch(i + step, 0);   // on their way during the sums
        row_statistics<false, true, TPR, NC, R>(v, [&](int c) { return there[c]; }, p.d, p.eps, part, mean, rstd);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (i + r >= rows) continue;
            if (threadIdx.x % TPR == 0) {
                p.mean[at + r * P] = mean[r];
                p.rstd[at + r * P] = rstd[r];
            }
            if (p.z) to.store(static_cast<T*>(p.z) + (at + r * P) * p.ldz, col0, v[r], lane, group_mask<TPR>());
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (there[c]) {
                    f32x2_t w[4], b[4];
                    staged_params(params, shifted, chunk_of<TPR, NC>(c), w, b);
                    scale8(v[r][c], mean[r], rstd[r], w, b, v[r][c]);
                }
            to.store(static_cast<T*>(p.y) + (at + r * P) * p.ldy, col0, v[r], lane, group_mask<TPR>());
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
        row_statistics<false, !VEC, TPR, NC, R>(v, [&](int c) { return columns_there((int)chunk_of<TPR, NC>(c) * kChunk, p.d); }, p.d, p.eps, part, mean, rstd);
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
        sq[0] += sum2(squares8<!VEC>(v, mean, columns_there((int)chunk * kChunk, p.d)));
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

// ---- launches ---------------------------------------------------------------------------------------
constexpr int kForwardWide = 16384, kForwardOddWide = 8192;   // widest rows that stay in registers

// What a block of a kernel takes of an SM beside its dynamic shared memory; looked up once, by the initialiser of a static
// (host threads that come first together wait for it).
struct KernelUse {
    int regs;      // per thread
    size_t smem;   // static
};
template <class Kernel>
KernelUse use_of(Kernel kernel)
{
    cudaFuncAttributes at = {};
    if (cudaFuncGetAttributes(&at, kernel) != cudaSuccess) (void)cudaGetLastError();   // the launch will say what is wrong
    return {at.numRegs > 0 ? at.numRegs : 128, at.sharedSizeBytes};
}
// Blocks that an SM holds.
int blocks_per_sm(const KernelUse& use, int block, size_t smem)
{
    int n = 65536 / ((use.regs + 7) / 8 * 8 * block);
    if (n > 2048 / block) n = 2048 / block;
    const int by_smem = (int)(227 * 1024 / (smem + use.smem + 1024));
    if (n > by_smem) n = by_smem;
    return n < 1 ? 1 : n;
}

template <class T, bool VEC, int TPR, int NC, int R>
cudaError_t forward_odd(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, SET = BLOCK / TPR * R;
    const size_t smem = (size_t)((p.d + kChunk - 1) / kChunk) * 64;
    const auto kernel = norm_forward_odd_kernel<T, VEC, TPR, NC, R>;
    if (smem > 47 * 1024) {
        static std::atomic<unsigned long long> limit_set{0};
        const cudaError_t e = ensure_smem_limit(kernel, kForwardOddWide * 8, limit_set);
        if (e != cudaSuccess) return e;
    }
    static const KernelUse use = use_of(kernel);
    const uint32_t sets = (p.rows + SET - 1) / SET;
    const uint32_t room = (uint32_t)(kSMs * blocks_per_sm(use, BLOCK, smem)) / p.nodes;
    kernel<<<dim3(sets < room ? sets : room ? room : 1, p.nodes), BLOCK, smem, s>>>(p);
    return cudaGetLastError();
}

template <class T, int TPR, int NC, int R, bool STAGED>
cudaError_t forward_shifted(const NormForwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = block_of(TPR), SET = BLOCK / TPR * R;
    constexpr uint32_t P = kShiftRows<T>;
    constexpr int kStage = !STAGED ? 0 : 4 * R * NC * BLOCK * kChunk * (int)sizeof(T);
    const size_t smem = (size_t)((p.d + P + kChunk - 1) / kChunk) * 64 + kStage;
    const auto kernel = norm_forward_shifted_kernel<T, TPR, NC, R, STAGED>;
    static std::atomic<unsigned long long> limit_set{0};
    const cudaError_t e = ensure_smem_limit(kernel, (TPR * NC + 2) * kChunk * 8 + kStage, limit_set);
    if (e != cudaSuccess) return e;
    static const KernelUse use = use_of(kernel);
    // as many blocks as fit, in whole classes of rows
    const uint32_t sets = ((p.rows + P - 1) / P + SET - 1) / SET;
    const uint32_t room = (uint32_t)(kSMs * blocks_per_sm(use, BLOCK, smem)) / (p.nodes * P);
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
            // Chunks per thread, threads per row, and whether rows are staged: narrow rows gain from few lanes (4 x 30000 rows of 203
            // bf16 64 us, a chunk for each of 32 lanes 82 us), wide ones lose warps to the shared memory of two sets (4 x 1500
            // rows of 5001 fp32 staged 155 us, in registers 122 us; 4 x 8000 of 1001 bf16 staged 69 us, in registers 77 us).
            constexpr bool W = sizeof(T) == 4;
            const int d = p.d + (int)kShiftRows<T> - 1;
            if (d <= 64) return forward_shifted<T, 8, 1, 2, true>(p, s);
            if (d <= 128) return forward_shifted<T, 8, 2, 1, true>(p, s);
            if (d <= 256) return forward_shifted<T, W ? 16 : 8, W ? 2 : 4, 1, true>(p, s);
            if (d <= 512) return forward_shifted<T, W ? 32 : 16, W ? 2 : 4, 1, true>(p, s);
            if (d <= 768) return forward_shifted<T, 32, 3, 1, false>(p, s);
            if (d <= 1024) return forward_shifted<T, W ? 64 : 32, W ? 2 : 4, 1, !W>(p, s);
            if constexpr (!W)
                if (d <= 1280) return forward_shifted<T, 32, 5, 1, true>(p, s);
            if (d <= 1536) return forward_shifted<T, W ? 96 : 64, W ? 2 : 3, 1, false>(p, s);
            if (d <= 2048) return forward_shifted<T, W ? 128 : 64, W ? 2 : 4, 1, !W>(p, s);
            if (d <= 2560) return forward_shifted<T, W ? 160 : 128, W ? 2 : 3, 1, false>(p, s);
            if (d <= 4096) return forward_shifted<T, 256, 2, 1, false>(p, s);
            if (d <= 6144) return forward_shifted<T, 256, 3, 1, false>(p, s);
            if (d <= kForwardOddWide) return forward_shifted<T, W ? 512 : 256, W ? 2 : 4, 1, false>(p, s);
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

}  // namespace

cudaError_t launch_norm_forward(const NormForwardParams& p, int dtype, bool vec, cudaStream_t s)
{
    if (!p.rows) return cudaSuccess;
#define GPGA_CALL(T, V) forward_of<T, V>(p, s)
    return GPGA_BY_TYPE(GPGA_CALL);
#undef GPGA_CALL
}

}  // namespace gpga
