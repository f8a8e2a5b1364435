// Gradient of the layer norm of residual + dropout(x): of z and x row by row, of the weight and the bias over the rows.
#include <type_traits>
#include "gpga_norm_device.cuh"

namespace gpga {

namespace {

// g = rstd (w dy - mean(h) - xh mean(h xh)) of one chunk, xh = (z - mean) rstd.
__device__ __forceinline__ void grad8(const f32x2_t* z, const f32x2_t* dy, const f32x2_t* w, float mean, float rstd, float mh, float mhx,
                                      f32x2_t* g)
{
    const f32x2_t m = both(mean), s = both(rstd), a = both(-mh), c = both(-mhx);
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] = mul2(s, fma2(mul2(sub2(z[j], m), s), c, fma2(dy[j], w[j], a)));
}

struct NoStore {   // in a kernel's aligned form, in place of a ShiftedStore
    __device__ __forceinline__ NoStore(int, int, int, const void*, int) {}
};
struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

// The block's column sums: its groups of threads one after the other, then out, to the node's gradients or to the block's
// row of partial sums.  `sums` (2 * TPR * NC * 4 pairs) is used where the block has several groups.  col0(c): first
// column of the thread's chunk c.
template <int TPR, int NC, class Col0>
__device__ __forceinline__ void write_column_sums(const NormBackwardParams& p, uint32_t node, f32x2_t (*dw)[4], f32x2_t (*db)[4], f32x2_t* sums,
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
                        f32x2_t* at = sums + chunk_of<TPR, NC>(c) * 4 + j;
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
// there again.
// Bound: neither issue slots (56 % busy) nor HBM alone, but latency at 16 warps per SM beside both.  8 x 4096 rows of 1024
// bf16, residual and dropout 63 us = 5.3 TB/s in a graph (whole calls 69 us), without either 41 us; fp32 130 us = 5.2 TB/s; 2000 rows of 8192 fp32 58 us = 3.4 TB/s, bound by the chain of one
// row per SM; shifted rows of 1001 bf16 (4 x 8000) 115 us against 184 us when cut, and
// 123 us with a test for every row and chunk of every set.
// kSets: sets of rows in shared memory, one worked on, the others on their way.
template <class T, bool SHIFT, int TPR, int NC, int R, int kSets, int kPerSM>
__global__ void __launch_bounds__(block_of(TPR), kPerSM) norm_backward_kernel(const NormBackwardParams p)
{
    constexpr int BLOCK = block_of(TPR), G = BLOCK / TPR, LANES = lanes_of(TPR), Q = sizeof(T) / 2;
    constexpr uint32_t P = SHIFT ? kShiftRows<T> : 1;
    extern __shared__ uint4 stage[];   // two sets of [tensor][r][c][warp][piece]
    __shared__ __align__(16) float part[2][BLOCK / 32 * 2 * R];
    __shared__ __align__(128) T slots[SHIFT ? BLOCK / LANES : 1][2][16];
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
    const Staged<T, SHIFT, TPR, NC, R> staged{stage, p.d, shift, lane};
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

    // the set whose first row is `set` rows behind the current pointers; n: rows that it has
    auto fetch_rows = [&](uint32_t set, int buf, uint32_t n, bool full) {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (full || (uint32_t)r < n) {
                staged.fetch(z + (int64_t)(set + r) * row_z, sz, buf * 3 + 0, r, full);
                staged.fetch(dy + (int64_t)(set + r) * row_y, sy, buf * 3 + 1, r, full);
            }
        if (tensors == 3)
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (full || (uint32_t)r < n) staged.fetch(dz + (int64_t)(set + r) * row_e, se, buf * 3 + 2, r, full);
    };
    auto fetch = [&](uint32_t set, int buf) {
        const uint32_t from = i + set, n = from < rows ? min((uint32_t)R, rows - from) : 0;
        if (!SHIFT && all_columns && i0 + set + G * R <= rows) fetch_rows(set, buf, R, true);
        else fetch_rows(set, buf, n, false);
        copies_commit();
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
    std::conditional_t<SHIFT, ShiftedStore<T, LANES, NC>, NoStore> to(col(0), p.d, shift, slots[SHIFT ? threadIdx.x / LANES : 0][0], lane);
    uint32_t set = 0;
    __shared__ uint4 edges[SHIFT ? BLOCK : 1];
    uint4* own_edges = edges + (SHIFT ? threadIdx.x - lane : 0);
    // one set; full: all its rows are there, and all chunks or (SHIFT) zeroes in place of what is not
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
                    staged.chunk(buf * 3 + 0, r, c, vz);
                    staged.chunk(buf * 3 + 1, r, c, vy);
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
        if (SHIFT && p.dx && p.mask.on && set % (LANES / R) == 0) {   // lane l works out the words before the warp's first chunk, in row l % R of set l / R from here
            __syncwarp(group_mask<TPR>());
            own_edges[lane] = drop_words(p.mask, (first_row + (i + lane / R * step + lane % R) * P) * chunks + first_chunk_of<TPR, NC>(0) - 1, node);
            __syncwarp(group_mask<TPR>());
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (!FULL && i + r >= rows) continue;
            f32x2_t g[NC][4];
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if (!FULL && !mine(c)) continue;
                f32x2_t vz[4], vy[4];
                staged.chunk(buf * 3 + 0, r, c, vz);
                staged.chunk(buf * 3 + 1, r, c, vy);
                grad8(vz, vy, w[c], mean[r], rstd[r], s[2 * r] * inv_d, s[2 * r + 1] * inv_d, g[c]);
            }
            if (tensors == 3)
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    if (!FULL && !mine(c)) continue;
                    f32x2_t e[4];
                    staged.chunk(buf * 3 + 2, r, c, e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[c][j] = add2(g[c][j], e[j]);
                }
#pragma unroll
            for (int c = 0; c < NC; ++c)
                if (!SHIFT && (FULL || mine(c))) store8<T>(dres + r * row_g + col(c), g[c]);
            if constexpr (SHIFT) to.store(dres + r * row_g, col(0), g, lane, group_mask<TPR>());
            if (!p.dx) continue;
            const uint32_t groups = (first_row + (i + r) * P) * chunks;
            uint4 before = make_uint4(0, 0, 0, 0);
            if (SHIFT) before = own_edges[set % (LANES / R) * R + r];
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
            if constexpr (SHIFT) to.store(dx + r * row_x, col(0), g, lane, group_mask<TPR>());
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
        if ((SHIFT || all_columns) && i0 + G * R <= rows) work(buf, odd, mean, rstd, Yes());
        else work(buf, odd, mean, rstd, No());
        ++set, i0 += step, i += step;
        z += step * row_z, dy += step * row_y, dz += step * row_e, dres += step * row_g, dx += step * row_x;
        means += (int64_t)step * P, rstds += (int64_t)step * P;
    }
    copies_wait<0>();
    __syncthreads();
    write_column_sums<TPR, NC>(p, node, dw, db, reinterpret_cast<f32x2_t*>(stage), col);
}

// Rows that are off the alignment in different ways: each chunk is cut out of the pieces of memory it lies in.
template <class T, int TPR, int NC>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) norm_backward_odd_kernel(const NormBackwardParams p)
{
    constexpr int BLOCK = TPR < 128 ? 128 : TPR, G = BLOCK / TPR, LANES = lanes_of(TPR);
    __shared__ __align__(16) float part[2][BLOCK / 32 * 2];
    __shared__ f32x2_t sums[G > 1 ? 2 * TPR * NC * 4 : 1];
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
    __shared__ __align__(16) float part[32 * 2];
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
constexpr int kBackwardWide = 8192;   // widest rows whose column sums stay in registers

template <class T, bool SHIFT, int TPR, int NC, int R, int kSets, int kPerSM>
cudaError_t backward_as(const NormBackwardParams& p, cudaStream_t s)
{
    constexpr int BLOCK = block_of(TPR), G = BLOCK / TPR;
    constexpr size_t kStage = (size_t)kSets * 3 * R * NC * 8 * sizeof(T) * BLOCK, kSums = G > 1 ? (size_t)2 * TPR * NC * 8 * 4 : 0;
    constexpr size_t smem = kStage > kSums ? kStage : kSums;
    const auto kernel = norm_backward_kernel<T, SHIFT, TPR, NC, R, kSets, kPerSM>;
    static std::atomic<unsigned long long> limit_set{0};
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
